// The 4-bit form of a KV block and the arithmetic of one row, shared by the kernels that write and read it.
//
// A block is [Hkv][B / 16 tiles][2560 bytes], the whole rounded up to a multiple of 4096 bytes (the recall moves
// 4096-byte pieces).  A tile holds 16 tokens of one KV head and is contiguous, so that one warp fetches what it
// works on next in one burst:
//     [   0) K codes  [16 tokens][64 B]
//     [1024) V codes  [16 tokens][64 B]
//     [2048) K scales [16 tokens][4 groups]{scale, minimum} bf16
//     [2304) V scales [16 tokens][4 groups]{scale, minimum} bf16
// Every row of 128 channels is cut into 4 groups of 32:
//     minimum = min x,  scale = bf16((max x - min x) / 15),  code = round((x - minimum) / scale) in 0..15,
//     value = scale * code + minimum.
// The minimum is one of the (bf16) inputs and therefore exact; the scale is rounded BEFORE the codes are taken, so
// that writer and reader use the same number.  Non-finite inputs make their group of 32 read back as NaN.
//
// The order of the codes is the order in which the attention kernel's matrix instructions take them:
//     K row, channel 32 j + 8 c + i (j, c < 4, i < 8): nibble i of the 32-bit word at byte 16 c + 4 j
//     V row, channel 32 j + 4 r + i (r < 8, i < 4):    nibble i of the 16-bit word at byte 8 r + 2 j
#pragma once

#include "pi_common.cuh"

#define KV4_TILE_BYTES 2560
#define KV4_V_CODES 1024
#define KV4_K_SCALES 2048
#define KV4_V_SCALES 2304

static inline int64_t kv4_block_bytes(int n_kv_heads, int block_tokens) {
    return (static_cast<int64_t>(n_kv_heads) * block_tokens * 160 + 4095) / 4096 * 4096;
}

#ifdef __CUDACC__
// Codes and scale word of one row; 16 neighbouring lanes (aligned) hold the row, lane l of them channels 8 l .. 8 l + 7
// in `x`.  codes: nibble i = channel 8 l + i.  sz: scale | minimum << 16 of the lane's group (lanes 4 j .. 4 j + 3).
// All 32 lanes must call.
__device__ __forceinline__ void kv4_quantise(uint4 x, uint32_t& codes, uint32_t& sz) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&x);
    const __nv_bfloat162 mn2 = __hmin2_nan(__hmin2_nan(h[0], h[1]), __hmin2_nan(h[2], h[3]));
    const __nv_bfloat162 mx2 = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
    // {minimum, maximum} of the lane, then of the group's four lanes
    __nv_bfloat162 mm = __halves2bfloat162(__hmin_nan(__low2bfloat16(mn2), __high2bfloat16(mn2)),
                                           __hmax_nan(__low2bfloat16(mx2), __high2bfloat16(mx2)));
#pragma unroll
    for (int o = 1; o <= 2; o <<= 1) {
        const __nv_bfloat162 other = __shfl_xor_sync(0xffffffffu, mm, o);
        mm = __halves2bfloat162(__hmin_nan(__low2bfloat16(mm), __low2bfloat16(other)),
                                __hmax_nan(__high2bfloat16(mm), __high2bfloat16(other)));
    }
    const float lo = __low2float(mm);
    const __nv_bfloat16 sb = __float2bfloat16_rn(__fdiv_rn(__fsub_rn(__high2float(mm), lo), 15.f));
    const float s = __bfloat162float(sb);
    const __nv_bfloat162 pair = __halves2bfloat162(sb, __low2bfloat16(mm));
    sz = *reinterpret_cast<const uint32_t*>(&pair);
    codes = 0;
    if (__all_sync(0xffffffffu, s == 0.f || (s >= 0x1p-100f && s <= 0x1p100f))) {
        // Correctly rounded quotients by one divisor, after Markstein (Computation of elementary functions on the IBM RISC
        // System/6000 processor, 1990): q = d r with r = 1/s rounded, then q + (d - q s) r, the bracket being exact in a
        // fused operation.  Seven operations a value where a division of its own takes three times as many; the sum with
        // 1.5 * 2^23 rounds to the nearest whole number, ties to even, and leaves it in the low bits.
        const float r = s > 0.f ? __frcp_rn(s) : 0.f;              // no spread: code 0
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = (i & 1) ? __high2float(h[i >> 1]) : __low2float(h[i >> 1]);
            const float d = __fsub_rn(v, lo), q = __fmul_rn(d, r);
            const float c = __fmaf_rn(__fmaf_rn(-q, s, d), r, q);  // at most 15 (1 + 2^-8): the scale is rounded to 8 bits
            codes += __float_as_uint(__fadd_rn(c, 12582912.f)) << (4 * i);
        }
        codes -= 0x3f400000u;                                      // what 0x4b400000, shifted by 0, 4 and 8, adds up to
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = (i & 1) ? __high2float(h[i >> 1]) : __low2float(h[i >> 1]);
        // fmaxf takes the 0 where the quotient is not a number
        const float c = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(v, lo), s)), 0.f), 15.f);
        codes |= static_cast<uint32_t>(s > 0.f ? c : 0.f) << (4 * i);
    }
}

// Writes the row that 16 lanes hold (codes and scale words of kv4_quantise) to token `t` of the tile at `tile`.
// is_v must be the same for the 16 lanes; all 32 lanes must call (`write` false: nothing is stored).
__device__ __forceinline__ void kv4_write_row(unsigned char* tile, int t, bool is_v, int l, uint32_t codes, uint32_t sz, bool write) {
    const int j = l >> 2, c = l & 3;
    // a V row wants the 16-bit halves of lanes (j, c) and (j + 1, c) side by side: the even lane takes the low halves
    // (channels 8 c .. 8 c + 3 of both groups), the odd one the high halves
    const uint32_t other = __shfl_xor_sync(0xffffffffu, codes, 4);
    uint32_t word = codes;
    int at = 16 * c + 4 * j;
    if (is_v) {
        word = (j & 1) ? __byte_perm(other, codes, 0x7632) : __byte_perm(codes, other, 0x5410);
        at = 8 * (2 * c + (j & 1)) + 2 * (j & 2);
    }
    if (!write) return;
    *reinterpret_cast<uint32_t*>(tile + (is_v ? KV4_V_CODES : 0) + t * 64 + at) = word;
    if (c == 0) *reinterpret_cast<uint32_t*>(tile + (is_v ? KV4_V_SCALES : KV4_K_SCALES) + t * 16 + j * 4) = sz;
}

__device__ __forceinline__ float kv4_scale_of(uint32_t sz) { return __uint_as_float(sz << 16); }
__device__ __forceinline__ float kv4_min_of(uint32_t sz) { return __uint_as_float(sz & 0xffff0000u); }
#endif
