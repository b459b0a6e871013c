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
// Codes and scale word of one row; 8 neighbouring lanes (aligned) hold the row, lane l of them channels 16 l .. 16 l + 15
// in `x`.  codes: nibble i of word k = channel 16 l + 8 k + i.  sz: scale | minimum << 16 of the lane's group (lanes 2 j and
// 2 j + 1).  All 32 lanes must call.
__device__ __forceinline__ void kv4_quantise(const uint4 (&x)[2], uint32_t (&codes)[2], uint32_t& sz) {
    const uint32_t xs[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(xs);
    __nv_bfloat162 mn = __hmin2_nan(__hmin2_nan(__hmin2_nan(h[0], h[1]), __hmin2_nan(h[2], h[3])), __hmin2_nan(__hmin2_nan(h[4], h[5]), __hmin2_nan(h[6], h[7])));
    __nv_bfloat162 mx = __hmax2_nan(__hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])), __hmax2_nan(__hmax2_nan(h[4], h[5]), __hmax2_nan(h[6], h[7])));
    mn = __hmin2_nan(mn, __lowhigh2highlow(mn));
    mx = __hmax2_nan(mx, __lowhigh2highlow(mx));
    // {minimum, -maximum} of the lane, then of the group's two lanes: one minimum of pairs
    uint32_t pair = __byte_perm(*reinterpret_cast<uint32_t*>(&mn), *reinterpret_cast<uint32_t*>(&mx), 0x5410) ^ 0x80000000u;
    const uint32_t other = __shfl_xor_sync(0xffffffffu, pair, 1);
    const __nv_bfloat162 m = __hmin2_nan(*reinterpret_cast<const __nv_bfloat162*>(&pair), *reinterpret_cast<const __nv_bfloat162*>(&other));
    pair = *reinterpret_cast<const uint32_t*>(&m);
    const float lo = __uint_as_float(pair << 16);
    const float spread = __fsub_rn(-__uint_as_float(pair & 0xffff0000u), lo);
    codes[0] = codes[1] = 0;
    if (__all_sync(0xffffffffu, spread == 0.f || (spread >= 0x1p-96f && spread <= 0x1p96f))) {
        // Quotients after Markstein (Computation of elementary functions on the IBM RISC System/6000 processor, 1990):
        // q = d r with r about 1 / s, then q + (d - q s) r, the bracket being exact in a fused operation.  A quotient that is
        // representable, as the borders between two codes are, comes out exactly.  The sum with 1.5 * 2^23 rounds to the
        // nearest whole number, ties to even, and leaves it in the low bits.  Seven operations a value; a division of its
        // own takes three times as many.
        const float fifteenth = 0.066666670143604278564f;
        const float q15 = __fmul_rn(spread, fifteenth);
        const __nv_bfloat16 sb = __float2bfloat16_rn(__fmaf_rn(__fmaf_rn(-q15, 15.f, spread), fifteenth, q15));
        const float s = __bfloat162float(sb);
        sz = __byte_perm(__bfloat16_as_ushort(sb), pair, 0x5410);
        const float r = spread > 0.f ? __fdividef(1.f, s) : 0.f;   // no spread: code 0
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float v = __uint_as_float((i & 1) ? xs[i >> 1] & 0xffff0000u : xs[i >> 1] << 16);
            const float d = __fsub_rn(v, lo), q = __fmul_rn(d, r);
            const float c = __fmaf_rn(__fmaf_rn(-q, s, d), r, q);  // at most 15 (1 + 2^-8): the scale is rounded to 8 bits
            codes[i >> 3] += __float_as_uint(__fadd_rn(c, 12582912.f)) << (4 * (i & 7));
        }
        codes[0] -= 0x3f400000u;                                   // what 0x4b400000, shifted by 0, 4 and 8, adds up to
        codes[1] -= 0x3f400000u;
        return;
    }
    const __nv_bfloat16 sb = __float2bfloat16_rn(__fdiv_rn(spread, 15.f));
    const float s = __bfloat162float(sb);
    sz = __byte_perm(__bfloat16_as_ushort(sb), pair, 0x5410);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float v = __uint_as_float((i & 1) ? xs[i >> 1] & 0xffff0000u : xs[i >> 1] << 16);
        // fmaxf takes the 0 where the quotient is not a number
        const float c = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(v, lo), s)), 0.f), 15.f);
        codes[i >> 3] |= static_cast<uint32_t>(s > 0.f ? c : 0.f) << (4 * (i & 7));
    }
}

// Where lane l of a row's eight puts its two words (the second kv4_step further on) and, for even l, its group's scales,
// counted from the row's codes and scales.
__device__ __forceinline__ int kv4_word_at(bool is_v, int l) { return is_v ? 32 * (l & 1) + 8 * (l & 2) + 4 * (l >> 2) : 32 * (l & 1) + 4 * (l >> 1); }
__device__ __forceinline__ int kv4_step(bool is_v) { return is_v ? 8 : 16; }

// Writes the row that eight lanes hold (codes and scale word of kv4_quantise) to token `t` of the tile at `tile`.  is_v
// must be the same for the eight; all 32 lanes must call (`write` false: nothing is stored).
__device__ __forceinline__ void kv4_write_row(unsigned char* tile, int t, bool is_v, int l, const uint32_t (&codes)[2], uint32_t sz, bool write) {
    // a V row wants the 16-bit halves of two neighbouring groups (lanes l and l ^ 2) side by side: the lane of the even
    // group takes the first word's, the other one the second's
    const bool odd = l & 2;
    const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? codes[0] : codes[1], 2);
    uint32_t w0 = codes[0], w1 = codes[1];
    if (is_v) {
        const uint32_t a = odd ? other : codes[0], b = odd ? codes[1] : other;
        w0 = __byte_perm(a, b, 0x5410);
        w1 = __byte_perm(a, b, 0x7632);
    }
    if (!write) return;
    unsigned char* row = tile + (is_v ? KV4_V_CODES : 0) + t * 64 + kv4_word_at(is_v, l);
    *reinterpret_cast<uint32_t*>(row) = w0;
    *reinterpret_cast<uint32_t*>(row + kv4_step(is_v)) = w1;
    if (!(l & 1)) *reinterpret_cast<uint32_t*>(tile + (is_v ? KV4_V_SCALES : KV4_K_SCALES) + t * 16 + 2 * l) = sz;
}

__device__ __forceinline__ float kv4_scale_of(uint32_t sz) { return __uint_as_float(sz << 16); }
__device__ __forceinline__ float kv4_min_of(uint32_t sz) { return __uint_as_float(sz & 0xffff0000u); }
#endif
