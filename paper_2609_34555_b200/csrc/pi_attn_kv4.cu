// Sparse GQA decode attention over a pool of 4-bit blocks:  softmax(q K^T / sqrt(D)) V  over the tokens of the selected
// blocks, K and V = scale * code + minimum (pi_kv4.cuh).
//
// 160 bytes a (token, KV head) for 4 G D operations: the pool's bytes are what the call cannot do without.  On the way
// to them stands the arithmetic of taking the codes apart, so that is kept out of the wide loops:
//   * a code becomes an fp16 number by one logical operation and one fused multiply-add per PAIR (code_pairs), and the
//     format's nibble order makes the pairs what the matrix instruction takes as they are;
//   * scales and minima never meet the codes.  For K they are applied to the products: with the channels of a group
//     contracted by themselves,  q.k = sum over groups  scale * (q . code) + minimum * (sum of q);  the minima's part is
//     one more small product.  For V the scales are applied to the weights, one set per group, and the minima's part is
//     again one product, of the weights and the minima.
// The contractions run on mma.sync (tokens or channels on M, up to 8 query heads on N), whose operands are registers: the codes
// are taken apart there. tcgen05 reads shared memory or TMEM, so every code would be written back first, two to four times as wide;
// with 4 to 16 query heads on N the matrix pipe is a quarter busy as it is.
// Codes are exact in fp16, queries after a power of two per head; weights times scales are rounded to 11 bits, which in the mean
// square adds an eighth of the output's own rounding (2 % to its square); all sums are in 32 bits.
//
// One (sequence, KV head) per cluster of S CTAs of 4 or 8 warps (S = 1, 2, 4 or 8; both by the launcher's rule).  The item's
// 16-token tiles are dealt out to its warps in turn; a warp streams its own tiles through its own ring of shared-memory
// stages with 16-byte asynchronous copies (a tile is 2560 contiguous bytes), so no warp waits for another until the
// end.  Every warp keeps its own running maximum and sum; the states are merged once, through shared memory, and
// across the cluster through distributed shared memory: one launch, no partials in global memory.
//
// Measured on a B200, back to back: 16 sequences x 128 blocks of 16 tokens, 8 KV heads, G = 4 (42 MB) 15.8 us; 64 x 64 blocks
// of 32 tokens (165 MB) 43.9 us, 3.8 TB/s; one sequence x 64 blocks 5.0 us; 64 x 64 blocks of 32 with G = 16 74 us.  The copies alone
// take 10.9 and 27.6 us of the larger ones.  What bounds them is the length of a step's chain (load, unpack, product, vote,
// exponential, transpose, product) with four warps a scheduler to cover it: about 400 instructions a tile and warp fill 62 % of the issue
// slots with 3.1 of 4 warps present; the integer pipe and the packed fp16 operations, which do not overlap, take 65 % of the
// cycles, the matrix pipe 25 %.
// Tried and not taken: codes as 128 + code in bf16, or as 1024 + code with the offset taken off by a product with a constant
// (one operation less a pair, paid back in matrix instructions); fp8 products (mma.sync turns the operands into fp16 first);
// one CTA per item of 8 warps, and 3 CTAs of 168 registers an SM (slower by 5 to 10 %).
#include <cuda_fp16.h>

#include <algorithm>

#include "pi_attn_merge.cuh"
#include "pi_kv4.cuh"

namespace {

using namespace pi_attn;

// Up to 8 query heads a KV head a warp works on two tiles at a time (the checks and the set-up of a step are shared, and the
// second tile's products fill the waits of the first), with one step ahead on its way; 16 warps an SM have 160 KB in
// flight or at work then.  More heads leave registers for one tile, with three ahead.
__host__ __device__ constexpr int a4_tiles(int NT) { return NT == 1 ? 2 : 1; }
__host__ __device__ constexpr int a4_steps(int NT) { return NT == 1 ? 2 : 4; }      // steps in the ring
__host__ __device__ constexpr int a4_warps_per_sm(int NT) { return NT == 1 ? 16 : 8; }  // what the registers allow
// Power of two of a head and group before its first product: a weight (at most 2^8) times it stays a number, so that no weight
// at all stays none, and whatever may be seen in the result (2^-133 and more) is above the smallest fp16 number.
constexpr int A4_NO_UNIT = 246;                    // the exponent's bits: 2^119

struct Attn4Params {
    const __nv_bfloat16* q;
    const unsigned char* pool;
    const int32_t* sel_slots;
    const int32_t* sel_blocks;
    const int32_t* sel_count;
    const int32_t* ctx_len;
    __nv_bfloat16* out;
    float* lse;
    pi_status_ref st;
    long long block_bytes;
    float scale_log2;
    uint32_t raise, raise64;        // 0x64006400, 0x54005400
    int Hq, Hkv, G, B, K, C;
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, unsigned long long policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
// (v & mask) | raise in one operation: it takes one immediate, so `raise` comes in a register (a kernel argument -- seen as a
// constant, it costs every pair a second operation: 218 instead of 159 of them a tile on the pipe that bounds this kernel)
__device__ __forceinline__ uint32_t masked(uint32_t v, uint32_t mask, uint32_t raise) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(v), "r"(mask), "r"(raise));
    return d;
}
// The four pairs of a word, nibbles n (low half) and n + 4 (high half), as fp16 numbers, less 8: -8 .. 7.  0x6400 | nibble is
// 1024 + nibble and 0x6400 | 16 nibble is 1024 + 16 nibble, so two of the four need no shift; bringing them back is exact.
// (Bits placed below a large number's exponent, and the number taken off: Kim, Henry, Fahim and Hassan Awadalla, Who Says
// Elephants Can't Run, 2022.)  Counted from the middle, since what a weight's rounding is worth is multiplied by the code: from 0 on, with
// a mean of 7.5 that the minima have to cancel, it doubles the error (tests/test_kv4_accuracy_cpu.py).
__device__ __forceinline__ void code_pairs(uint32_t w, uint32_t raise, uint32_t (&p)[4]) {
    const __half2 low = __halves2half2(__ushort_as_half(0xe408), __ushort_as_half(0xe408));        // -1032
    const __half2 sixteenth = __halves2half2(__ushort_as_half(0x2c00), __ushort_as_half(0x2c00));  // 1 / 16
    const __half2 high = __halves2half2(__ushort_as_half(0xd480), __ushort_as_half(0xd480));       // -72
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t v = i ? w >> 8 : w, a = masked(v, 0x000f000fu, raise), b = masked(v, 0x00f000f0u, raise);
        const __half2 x = __hadd2(*reinterpret_cast<const __half2*>(&a), low), y = __hfma2(*reinterpret_cast<const __half2*>(&b), sixteenth, high);
        p[2 * i] = *reinterpret_cast<const uint32_t*>(&x);
        p[2 * i + 1] = *reinterpret_cast<const uint32_t*>(&y);
    }
}
// For K: from 0 on, and the second pair as 64 + code (0x5400 | 16 nibble), which is half the operations (2 % of the call's time).
// The offset's part of the products is taken off with the minima's; cut to 32 bits on the way, that leaves scores about 1 off by
// 8e-7 in the mean square and scores about 100 by 8e-5 (measured), some six times what codes from 0 would: 4 % of the output's
// own rounding.
__device__ __forceinline__ void code_pairs_k(uint32_t w, uint32_t raise, uint32_t raise64, uint32_t (&p)[4]) {
    const __half2 low = __halves2half2(__ushort_as_half(0xe400), __ushort_as_half(0xe400));        // -1024
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t v = i ? w >> 8 : w, a = masked(v, 0x000f000fu, raise);
        const __half2 x = __hadd2(*reinterpret_cast<const __half2*>(&a), low);
        p[2 * i] = *reinterpret_cast<const uint32_t*>(&x);
        p[2 * i + 1] = masked(v, 0x00f000f0u, raise64);
    }
}
// d = a b
__device__ __forceinline__ void mma_f16_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_bf16_zero(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// 1 / x of a power of two well inside the range
__device__ __forceinline__ float inverse_power(float x) { return __uint_as_float(0x7f000000u - __float_as_uint(x)); }
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {          // both products in one operation
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t max_f16x2(uint32_t a, uint32_t b) {
    const __half2 v = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
}
// The power of two at or below |x|, at least the smallest normal number.
__device__ __forceinline__ float power_of(float x) { return __uint_as_float(max(__float_as_uint(x) & 0x7f800000u, 0x00800000u)); }
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ void sts128_zero(uint32_t a) { asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(a), "r"(0u) : "memory"); }
__device__ __forceinline__ void ldsm_x2_t(uint32_t addr, uint32_t& a, uint32_t& b) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(a), "=r"(b) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t word_of(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// NT: tiles of 8 query heads; WARPS of a CTA.
template <int NT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, a4_warps_per_sm(NT) / WARPS)
attn_kv4_kernel(Attn4Params p) {
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;
    const int S = static_cast<int>(cluster_nctarank()), rank = static_cast<int>(cluster_ctarank());
    const int item = blockIdx.x / S, seq = item / p.Hkv, h = item - seq * p.Hkv;
    constexpr int TP = a4_tiles(NT), STEPS = a4_steps(NT), STAGES = STEPS * TP;
    const int SUB = p.B >> 4;
    // (the other half of this barrier stands before the first store into another CTA's shared memory: by then it runs)
    if (S > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    pi_grid_dependency_wait();
    pi_launch_dependents();

    // the queries, the entries of the warp's first 32 tiles and the list's length are fetched beside one another
    uint4 query[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int g = nt * 8 + r;
        const __nv_bfloat16* qg = p.q + (static_cast<size_t>(seq) * p.Hq + static_cast<size_t>(h) * p.G + (g < p.G ? g : 0)) * PI_HEAD_DIM;
#pragma unroll
        for (int j = 0; j < 4; ++j) query[nt][j] = g < p.G ? __ldg(reinterpret_cast<const uint4*>(qg + 32 * j + 8 * c)) : make_uint4(0, 0, 0, 0);
    }
    const int first = rank * WARPS + warp, stride = WARPS * S, log_sub = 31 - __clz(SUB);
    const int32_t* slots = p.sel_slots + static_cast<size_t>(seq) * p.K;
    const int32_t* blocks = p.sel_blocks + static_cast<size_t>(seq) * p.K;
    auto entry_of = [&](int n) -> int2 {
        const int j = (first + n * stride) >> log_sub;
        return j < p.K ? make_int2(slots[j], blocks[j]) : make_int2(0, -1);
    };
    const int2 entry = entry_of(lane);
    const int ctx = p.ctx_len[seq];
    int cnt = p.sel_count[seq];
    if (cnt < 0 || cnt > p.K) {
        if (h == 0 && rank == 0 && tid == 0) pi_report(p.st, PI_ERR_CAPACITY, PI_STAGE_ATTN, seq, cnt, p.K);
        cnt = 0;
    }
    const int n_tiles = cnt * SUB;
    const int n_mine = first < n_tiles ? (n_tiles - first + stride - 1) / stride : 0;

    // The warp's n-th tile: byte offset from the head's first one (a sequence's pool is below 2^31 bytes), valid tokens.
    auto meta_of = [&](int n, int2 e) -> uint2 {
        if (n >= n_mine || e.y < 0) return make_uint2(0u, 0u);
        const int t = first + n * stride, sub = t & (SUB - 1);
        if (e.x < 0 || e.x >= p.C) {
            if (h == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_ATTN, seq, t >> log_sub, e.x);
            return make_uint2(0u, 0u);
        }
        const long long left = static_cast<long long>(ctx) - (static_cast<long long>(e.y) * p.B + sub * 16);
        return make_uint2(static_cast<uint32_t>(e.x * p.block_bytes) + sub * KV4_TILE_BYTES, left < 0 ? 0u : left > 16 ? 16u : static_cast<uint32_t>(left));
    };
    uint2 meta = meta_of(lane, entry), meta_next = make_uint2(0u, 0u);     // of tiles 32 i + lane, and of the 32 after those
    unsigned some = __ballot_sync(0xffffffffu, meta.y != 0u), whole = __ballot_sync(0xffffffffu, meta.y == 16u), some_next = 0u;

    const unsigned char* head_base = p.pool + static_cast<long long>(seq) * p.C * p.block_bytes + static_cast<long long>(h) * SUB * KV4_TILE_BYTES + lane * 16;
    const uint32_t ring = smem_u32(smem) + warp * (STAGES * KV4_TILE_BYTES);
    const unsigned long long policy = pi_l2_stream_policy();
    uint32_t fill = 0u;                                  // stage of the next tile
    auto issue = [&](int i, unsigned mask, uint32_t offsets) {      // the step of tiles i .. of a batch of 32 into its stages, one commit
#pragma unroll
        for (int k = 0; k < TP; ++k) {
            const uint32_t offset = __shfl_sync(0xffffffffu, offsets, i + k);
            if ((mask >> (i + k)) & 1u) {
                const unsigned char* src = head_base + offset;
                const uint32_t dst = ring + fill + lane * 16;
#pragma unroll
                for (int x = 0; x < KV4_TILE_BYTES / 512; ++x) copy16(dst + x * 512, src + x * 512, policy);
            }
            fill = fill == (STAGES - 1) * KV4_TILE_BYTES ? 0u : fill + KV4_TILE_BYTES;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int n = 0; n < STEPS - 1; ++n) issue(n * TP, some, meta.x);

    // ---- the queries as B operands, in the channel order of the K codes, as fp16 numbers: every head is scaled by a power of
    // two so that its largest channel lies in [1, 2); what is below 2^-14 of that is rounded at 2^-25 of it, less than the
    // sums below round.  With them, for the minima's own products, lane (r, c)'s {-64 times the sum over every
    // second pair, sum} of head r over the channels of group c, to meet {scale, minimum}, as three bf16 numbers (2^-25
    // together).  One warp prepares a group of channels for all.
    uint4* s_bq = reinterpret_cast<uint4*>(smem + WARPS * STAGES * KV4_TILE_BYTES);       // [NT][4 groups][32 lanes]
    uint32_t* s_bz = reinterpret_cast<uint32_t*>(s_bq + NT * 4 * 32);                            // [NT][3][32]
    float* s_scale = reinterpret_cast<float*>(s_bz + NT * 3 * 32);                               // [NT][8 heads]
    float4* s_in = reinterpret_cast<float4*>(s_scale + NT * 8);                                  // from the cluster: see the end
    static_assert(WARPS >= 4, "one warp a group of channels");
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        if (WARPS > 4 && warp >= 4) break;
        const int mine = warp, part = nt * 4 + warp;
        uint4 own = query[nt][0];
        __nv_bfloat162 top2 = __float2bfloat162_rn(0.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j == mine) own = query[nt][j];
            const __nv_bfloat162* y = reinterpret_cast<const __nv_bfloat162*>(&query[nt][j]);
            top2 = __hmax2(__hmax2(__hmax2(__habs2(y[0]), __habs2(y[1])), __hmax2(__habs2(y[2]), __habs2(y[3]))), top2);
        }
        float top = fmaxf(__low2float(top2), __high2float(top2));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        top = power_of(top);
        const float inv = 1.f / top;
        const uint32_t xs[4] = {own.x, own.y, own.z, own.w};
        float f[8], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(xs[i] << 16) * inv;
            f[2 * i + 1] = __uint_as_float(xs[i] & 0xffff0000u) * inv;
            sum += f[2 * i] + f[2 * i + 1];
        }
        // pair n = channels (n, n + 4) of the eight
        s_bq[part * 32 + lane] = make_uint4(pack_f16(f[0], f[4]), pack_f16(f[1], f[5]), pack_f16(f[2], f[6]), pack_f16(f[3], f[7]));
        float off = 0.f;                           // what 64 at every second pair adds, of the numbers as they are packed
#pragma unroll
        for (int i = 1; i < 8; i += 2) off -= 64.f * __half2float(__float2half_rn(f[i]));
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        off += __shfl_xor_sync(0xffffffffu, off, 1);
        off += __shfl_xor_sync(0xffffffffu, off, 2);
        if (c == mine) {
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const float hi = __bfloat162float(__float2bfloat16_rn(sum));
                const float oh = __bfloat162float(__float2bfloat16_rn(off));
                s_bz[(nt * 3 + i) * 32 + lane] = pack_bf16(oh, hi);
                sum -= hi;
                off -= oh;
            }
            if (mine == 0) s_scale[nt * 8 + r] = p.scale_log2 * top;
        }
    }
    __syncthreads();
    uint32_t bq[NT][4][2][2], bz[NT][3];
    float scale[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 x = s_bq[(nt * 4 + j) * 32 + lane];
            bq[nt][j][0][0] = x.x; bq[nt][j][0][1] = x.y; bq[nt][j][1][0] = x.z; bq[nt][j][1][1] = x.w;
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) bz[nt][i] = s_bz[(nt * 3 + i) * 32 + lane];
        scale[nt][0] = s_scale[nt * 8 + 2 * c];
        scale[nt][1] = s_scale[nt * 8 + 2 * c + 1];
    }

    // ---- running state: o[j][mt] = channels 32 j + 4 r + 2 mt (+ 1 in the upper two) of heads 2 c, 2 c + 1, times the head's unit[j];
    // z = row r of {scale, minimum} of the four groups, weighted, for the same heads; m (exp2 domain) and l as usual
    float o[NT][4][2][4], z[NT][4], m[NT][2], l[NT][2], unit[NT][4][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = A4_NO_MAX;
        l[nt][0] = l[nt][1] = 0.f;
        z[nt][0] = z[nt][1] = z[nt][2] = z[nt][3] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            unit[nt][j][0] = unit[nt][j][1] = __uint_as_float(static_cast<uint32_t>(A4_NO_UNIT) << 23);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][j][0][e] = o[nt][j][1][e] = 0.f;
        }
    }
    // Row r of a tile's products is token pr (row r + 8: pr + 8): then the four tokens that a lane needs of V, rows 2 c,
    // 2 c + 1, 2 c + 8, 2 c + 9, are c, c + 4, c + 8, c + 12, and the lanes of one load read neighbouring rows.
    const int pr = (r >> 1) + 4 * (r & 1);
    const int pl = ((lane & 7) >> 1) + 4 * (lane & 1) + (lane & 8);     // the token whose scales this lane names to ldmatrix

    const uint32_t raise = p.raise, raise64 = p.raise64;
    uint32_t tile = ring;                                // first stage of the step at hand
    bool begun = false;                                  // a step has been added up
    for (int n = 0; n < n_mine; n += TP, tile = tile == ring + (STAGES - TP) * KV4_TILE_BYTES ? ring : tile + TP * KV4_TILE_BYTES) {
        const int i = n & 31;
        if (i == 0) {
            if (n) {
                meta = meta_next;
                some = some_next;
                whole = __ballot_sync(0xffffffffu, meta.y == 16u);
            }
            some_next = 0u;
            if (n + 32 < n_mine) {
                meta_next = meta_of(n + 32 + lane, entry_of(n + 32 + lane));
                some_next = __ballot_sync(0xffffffffu, meta_next.y != 0u);
            }
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(STEPS - 2) : "memory");
        __syncwarp();                                   // the step is filled by all lanes, and the previous one read by all
        if (i + (STEPS - 1) * TP < 32) issue(i + (STEPS - 1) * TP, some, meta.x);
        else issue(i + (STEPS - 1) * TP - 32, some_next, meta_next.x);
        constexpr unsigned all_of = (1u << TP) - 1u;
        if (!((some >> i) & all_of)) continue;
        // ---- S^T = K q^T: the minima's products first, then the codes' group by group
        float s[TP][NT][4];
#pragma unroll
        for (int k = 0; k < TP; ++k) {
            const uint32_t at = tile + k * KV4_TILE_BYTES;
            const uint4 ka = lds128(at + pr * 64 + c * 16), kb = lds128(at + (pr + 8) * 64 + c * 16);
            const uint4 za = lds128(at + KV4_K_SCALES + pr * 16), zb = lds128(at + KV4_K_SCALES + (pr + 8) * 16);
            const uint32_t ya = lds32(at + KV4_K_SCALES + pr * 16 + c * 4), yb = lds32(at + KV4_K_SCALES + (pr + 8) * 16 + c * 4);
            const uint32_t az[4] = {ya, yb, ya, yb};    // {scale, minimum} of group c: places 2 c, 2 c + 1 (and + 8)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                mma_bf16_zero(s[k][nt], az, bz[nt][2], 0u);
                mma_bf16(s[k][nt], az, bz[nt][0], bz[nt][1]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t a[4], b[4];
                code_pairs_k(word_of(ka, j), raise, raise64, a);
                code_pairs_k(word_of(kb, j), raise, raise64, b);
                const float sa = kv4_scale_of(word_of(za, j)), sb = kv4_scale_of(word_of(zb, j));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float x[4];
                    mma_f16_zero(x, a[0], b[0], a[1], b[1], bq[nt][j][0][0], bq[nt][j][0][1]);
                    mma_f16(x, a[2], b[2], a[3], b[3], bq[nt][j][1][0], bq[nt][j][1][1]);
                    s[k][nt][0] = fmaf(sa, x[0], s[k][nt][0]); s[k][nt][1] = fmaf(sa, x[1], s[k][nt][1]);
                    s[k][nt][2] = fmaf(sb, x[2], s[k][nt][2]); s[k][nt][3] = fmaf(sb, x[3], s[k][nt][3]);
                }
            }
        }
        if (((whole >> i) & all_of) != all_of) {        // what lies behind the last token may be anything, NaN among it
#pragma unroll
            for (int k = 0; k < TP; ++k) {
                const int nvalid = static_cast<int>(__shfl_sync(0xffffffffu, meta.y, i + k));
                if (lane < 16 && lane >= nvalid) sts128_zero(tile + k * KV4_TILE_BYTES + KV4_V_SCALES + lane * 16);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (pr >= nvalid) s[k][nt][0] = s[k][nt][1] = -INFINITY;
                    if (pr + 8 >= nvalid) s[k][nt][2] = s[k][nt][3] = -INFINITY;
                }
            }
            __syncwarp();
        }
        // ---- online softmax over the step's tokens.  The reference m moves only when a score exceeds it by 8 (a factor of
        // 256, far from any overflow), so that most steps neither reduce a maximum across lanes nor touch the sums.
        // (The score is rounded before m is taken off: fused, the rounding of m would be left over in every weight, and for
        // scores of 2^28 and more that alone leaves the range.  One operation a score, 1 % of the time.)
        float w[TP][NT][4];
        bool over = false;
#pragma unroll
        for (int k = 0; k < TP; ++k)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[k][nt][e] = __fmul_rn(s[k][nt][e], scale[nt][e & 1]);
                    w[k][nt][e] = s[k][nt][e] - m[nt][e & 1];
                }
                over |= max3(fmaxf(w[k][nt][0], w[k][nt][1]), w[k][nt][2], w[k][nt][3]) > 8.f;
            }
        if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float mx = fmaxf(s[0][nt][e], s[0][nt][2 + e]);
#pragma unroll
                    for (int k = 1; k < TP; ++k) mx = max3(mx, s[k][nt][e], s[k][nt][2 + e]);
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                    const float m_new = fmaxf(m[nt][e], mx), fall = m[nt][e] - m_new, alpha = ex2(fall);
#pragma unroll
                    for (int k = 0; k < TP; ++k) {
                        w[k][nt][e] = s[k][nt][e] - m_new;
                        w[k][nt][2 + e] = s[k][nt][2 + e] - m_new;
                    }
                    m[nt][e] = m_new;
                    if (!begun) continue;                // the warp's first step: nothing has been summed yet
                    l[nt][e] *= alpha;
                    z[nt][e] *= alpha;
                    // What the head has seen so far counts for 2^fall less from here on, and its units rise by the whole part of
                    // that: tokens that have lost their weight take no bits from those that have it.
                    const int rise = static_cast<int>(fminf(-fall, 255.f));
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int have = static_cast<int>(__float_as_uint(unit[nt][j][e]) >> 23), now = min(have + rise, A4_NO_UNIT);
                        const float f = ex2(fall + static_cast<float>(now - have));
                        unit[nt][j][e] = __uint_as_float(static_cast<uint32_t>(now) << 23);
                        o[nt][j][0][e] *= f; o[nt][j][0][2 + e] *= f;
                        o[nt][j][1][e] *= f; o[nt][j][1][2 + e] *= f;
                    }
                }
        }
        begun = true;
        // ---- the weights; with them the minima's share of the result, for all four groups in one product.  Minima and
        // scales are bf16, so the weights take part as a bf16 head (the upper half of the number) and a bf16 remainder.
#pragma unroll
        for (int k = 0; k < TP; ++k) {
            uint32_t az[4];
            ldsm_x2_t(tile + k * KV4_TILE_BYTES + KV4_V_SCALES + pl * 16, az[0], az[2]);
            az[1] = az[3] = 0u;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float rest[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[k][nt][e] = ex2(w[k][nt][e]);
                    rest[e] = w[k][nt][e] - __uint_as_float(__float_as_uint(w[k][nt][e]) & 0xffff0000u);
                }
                l[nt][0] += w[k][nt][0] + w[k][nt][2];
                l[nt][1] += w[k][nt][1] + w[k][nt][3];
                mma_bf16(z[nt], az, movm_t(pack_bf16(rest[0], rest[1])), movm_t(pack_bf16(rest[2], rest[3])));
                mma_bf16(z[nt], az, movm_t(__byte_perm(__float_as_uint(w[k][nt][0]), __float_as_uint(w[k][nt][1]), 0x7632)),
                         movm_t(__byte_perm(__float_as_uint(w[k][nt][2]), __float_as_uint(w[k][nt][3]), 0x7632)));
            }
        }
        // ---- weight times scale, one set per group, in fp16: 11 bits, where bf16 would need two numbers.  Its narrow range is
        // covered by a power of two per head and group (`unit`), set by the first step so that the largest product is about 2^8,
        // lowered when a later one leaves the range and raised when the head's maximum moves.  A product that is 2^-22 of the
        // largest of its head and group, and more, keeps its 11 bits; what a smaller one is off by is 2^-33 of the largest.
        // Per head: weights that are everything for one are nothing for its neighbour, and columns without a head have weights too.
        uint32_t pw[TP][NT][4][2];
        auto products = [&]() {
            uint32_t top = 0u;
#pragma unroll
            for (int k = 0; k < TP; ++k) {
                const uint32_t at = tile + k * KV4_TILE_BYTES + KV4_V_SCALES;
                const uint4 va = lds128(at + pr * 16), vb = lds128(at + (pr + 8) * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float sa = kv4_scale_of(word_of(va, j)), sb = kv4_scale_of(word_of(vb, j));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        // (the weight first: scale times unit may leave 32 bits, and then no weight would be no number)
                        const float2 u = make_float2(unit[nt][j][0], unit[nt][j][1]);
                        const float2 pa = mul2(mul2(make_float2(w[k][nt][0], w[k][nt][1]), u), make_float2(sa, sa));
                        const float2 pb = mul2(mul2(make_float2(w[k][nt][2], w[k][nt][3]), u), make_float2(sb, sb));
                        pw[k][nt][j][0] = pack_f16(pa.x, pa.y);
                        pw[k][nt][j][1] = pack_f16(pb.x, pb.y);
                        top = max_f16x2(top, max_f16x2(pw[k][nt][j][0], pw[k][nt][j][1]));
                    }
                }
            }
            return top;
        };
        // (a loop of two rounds at most, so that the products' code is there once)
#pragma unroll 1
        for (bool again = false;; again = true) {
            const uint32_t top = products();
            const __half2 t = *reinterpret_cast<const __half2*>(&top);
            if (again || !__any_sync(0xffffffffu, __hgt(__hmax(__low2half(t), __high2half(t)), __ushort_as_half(0x7800)))) break;      // 2^15
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float sc[TP][2];                    // scales, 2^-20 of them: a product may leave fp32
#pragma unroll
                for (int k = 0; k < TP; ++k) {
                    const uint32_t at = tile + k * KV4_TILE_BYTES + KV4_V_SCALES + j * 4;
                    sc[k][0] = kv4_scale_of(lds32(at + pr * 16)) * 0x1p-20f;
                    sc[k][1] = kv4_scale_of(lds32(at + (pr + 8) * 16)) * 0x1p-20f;
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    // the two heads' largest products of the group in the step, cut to bf16: the exponent is all that counts.  (One
                    // that leaves fp16 is above 2^-104, since a unit is at most 2^119, so 2^-20 of it is a normal number.)
                    float mx[2] = {0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < TP; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) mx[e] = max3(mx[e], w[k][nt][e] * sc[k][0], w[k][nt][2 + e] * sc[k][1]);
                    uint32_t pair = __byte_perm(__float_as_uint(mx[0]), __float_as_uint(mx[1]), 0x7632);
#pragma unroll
                    for (int d = 4; d <= 16; d <<= 1) {
                        const uint32_t other = __shfl_xor_sync(0xffffffffu, pair, d);
                        const __nv_bfloat162 v = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&pair), *reinterpret_cast<const __nv_bfloat162*>(&other));
                        pair = *reinterpret_cast<const uint32_t*>(&v);
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        // exponents: of 2^8 / (2^20 mx), from which the product of the largest weight and scale is 2^8 and more
                        const int top_exp = min(static_cast<int>(e ? pair >> 23 : (pair >> 7) & 0xffu), 239);
                        const int have = static_cast<int>(__float_as_uint(unit[nt][j][e]) >> 23), now = top_exp > 0 ? min(242 - top_exp, have) : have;
                        const float f = __uint_as_float(static_cast<uint32_t>(max(127 + now - have, 0)) << 23);     // (2^-127 and less: 0)
                        unit[nt][j][e] = __uint_as_float(static_cast<uint32_t>(now) << 23);
                        o[nt][j][0][e] *= f; o[nt][j][0][2 + e] *= f;
                        o[nt][j][1][e] *= f; o[nt][j][1][2 + e] *= f;
                    }
                }
            }
        }
        // ---- O^T += V^T (weight scale), group by group
#pragma unroll
        for (int k = 0; k < TP; ++k) {
            uint2 x[4];
#pragma unroll
            for (int a = 0; a < 4; ++a) x[a] = lds64(tile + k * KV4_TILE_BYTES + KV4_V_CODES + (4 * a + c) * 64 + r * 8);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned sel = (j & 1) ? 0x7632u : 0x5410u;
                uint32_t a[4], b[4];
                code_pairs(__byte_perm(j < 2 ? x[0].x : x[0].y, j < 2 ? x[1].x : x[1].y, sel), raise, a);
                code_pairs(__byte_perm(j < 2 ? x[2].x : x[2].y, j < 2 ? x[3].x : x[3].y, sel), raise, b);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint32_t b0 = movm_t(pw[k][nt][j][0]), b1 = movm_t(pw[k][nt][j][1]);
                    mma_f16(o[nt][j][0], a[0], a[1], b[0], b[1], b0, b1);
                    mma_f16(o[nt][j][1], a[2], a[3], b[2], b[3], b0, b1);
                }
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");

    // ---- the warp's state into shared memory: o [warp][G][128], then m and l [warp][G] (the ring is done with)
    __syncthreads();
    float* s_o = reinterpret_cast<float*>(smem);
    float* s_m = s_o + WARPS * p.G * PI_HEAD_DIM;
    float* s_l = s_m + WARPS * p.G;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float sum = l[nt][e];
#pragma unroll
            for (int d = 4; d <= 16; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            const int g = nt * 8 + 2 * c + e;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // the minima's share is in the lanes that hold row 2 j + 1, the scales', of which the codes lack 8, in those of row 2 j
                const float f = inverse_power(unit[nt][j][e]), zj = fmaf(8.f, __shfl_sync(0xffffffffu, z[nt][e], 8 * j + c), __shfl_sync(0xffffffffu, z[nt][e], 8 * j + 4 + c));
                const float4 v = make_float4(fmaf(o[nt][j][0][e], f, zj), fmaf(o[nt][j][0][2 + e], f, zj), fmaf(o[nt][j][1][e], f, zj), fmaf(o[nt][j][1][2 + e], f, zj));
                if (g < p.G) *reinterpret_cast<float4*>(s_o + (warp * p.G + g) * PI_HEAD_DIM + 32 * j + 4 * r) = v;
            }
            if (g < p.G && r == 0) { s_m[warp * p.G + g] = m[nt][e]; s_l[warp * p.G + g] = sum; }
        }
    __syncthreads();

    conclude<WARPS>(p, seq, h, S, rank, tid, s_o, s_m, s_l, s_in);
}

}  // namespace

int pi_launch_attn_kv4(pi_ctx* c, int batch, const void* q, const void* pool, const int32_t* sel_slots, const int32_t* sel_blocks,
                       const int32_t* sel_count, const int32_t* ctx_len, void* out, float* lse, cudaStream_t stream) {
    const pi_config& cfg = c->cfg;
    Attn4Params p;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.pool = static_cast<const unsigned char*>(pool);
    p.sel_slots = sel_slots; p.sel_blocks = sel_blocks; p.sel_count = sel_count; p.ctx_len = ctx_len;
    p.out = static_cast<__nv_bfloat16*>(out);
    p.lse = lse;
    p.st = pi_status_of(c);
    p.block_bytes = kv4_block_bytes(cfg.n_kv_heads, cfg.block_tokens);
    p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(PI_HEAD_DIM));
    p.raise = 0x64006400u;
    p.raise64 = 0x54005400u;
    p.Hq = cfg.n_q_heads; p.Hkv = cfg.n_kv_heads; p.G = cfg.n_q_heads / cfg.n_kv_heads;
    p.B = cfg.block_tokens; p.K = cfg.budget_blocks; p.C = cfg.pool_slots;
    const int NT = p.G <= 8 ? 1 : 2, tiles = cfg.budget_blocks * (cfg.block_tokens / 16);
    const long long items = static_cast<long long>(batch) * cfg.n_kv_heads, room = static_cast<long long>(a4_warps_per_sm(NT)) * c->n_sms;
    // CTAs per item: what takes least by this estimate (microseconds, less what every call takes).  A cluster costs 1.0 more than
    // a CTA by itself; a step of its warps 1.0, or with k CTAs on the SM 0.12 + 0.59 k, when they fill its pipes (more than 8
    // heads: 0.8, or 0.5 k); the GPU starts 170 CTAs (85) in one, from three an SM on all in 3.0.  Measured, with S = 1 / 2 / 4 /
    // 8: 64 items x 64 tiles 11.7 / 8.5 / 7.3 / 8.1 us, 144 x 16 tiles 5.2 / 5.9 / 10.7 / 16.1, 8 x 48 tiles 9.2 / 7.0 / 6.0 /
    // 5.2, 128 x 128 tiles 20.7 / 16.1 / 16.0 / 20.4.  Clusters that would not all be on the GPU at once lose to smaller ones.
    int split = 1, warps = 4;
    double least = 0.;
    for (int s = 1; s <= A4_MAX_SPLIT; s *= 2) {
        const long long ctas = items * s, per_sm = (ctas + c->n_sms - 1) / c->n_sms, per_step = s * warps * a4_tiles(NT), steps = (tiles + per_step - 1) / per_step;
        if (s > 1 && ctas * warps > room * 7 / 8) break;
        const double step = NT == 1 ? std::max(1., 0.12 + 0.59 * static_cast<double>(per_sm)) : std::max(0.8, 0.5 * static_cast<double>(per_sm));
        const double start = NT == 2 ? static_cast<double>(ctas) / 85. : per_sm > 2 ? 3. : static_cast<double>(ctas) / 170.;
        const double cost = (s > 1 ? 1. : 0.) + static_cast<double>(steps - 1) * step + start;
        if (s == 1 || cost < least) { split = s; least = cost; }
    }
    // Few items with long lists leave SMs with one CTA each, which 8 warps use better (8 items x 256 tiles 7.2 us, 8.4 with 4
    // warps; x 1024 16.1, 21.4; one item x 1024 15.8, 20.7); a shorter list gains little (8 x 128 tiles 5.8, 6.2), more items nothing
    // (16 x 256 9.9 both ways).
    if (NT == 1 && split == A4_MAX_SPLIT && items * split * 8 <= room && tiles >= 32 * std::max(items, 8ll)) warps = 8;
    const size_t ring = static_cast<size_t>(warps) * a4_steps(NT) * a4_tiles(NT) * KV4_TILE_BYTES + NT * (4 * 32 * 16 + 3 * 32 * 4 + 8 * 4);
    // (the merge of a CTA's warps, up to 33 KB for four, takes the ring's place; what the cluster sends lies behind)
    const size_t smem = ring + (split > 1 ? static_cast<size_t>(p.G) * (PI_HEAD_DIM * 4 + split * 8) : 0);
    auto launch = [&](auto kernel) -> int {
        if (smem > 48 * 1024) PI_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3(static_cast<unsigned>(items * split));
        lc.blockDim = dim3(warps * 32);
        lc.dynamicSmemBytes = smem;
        lc.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = split;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        lc.attrs = attr;
        lc.numAttrs = split > 1 ? 2 : 1;
        PI_CUDA_TRY(cudaLaunchKernelEx(&lc, kernel, p));
        return PI_OK;
    };
    if (NT == 1) return warps == 4 ? launch(attn_kv4_kernel<1, 4>) : launch(attn_kv4_kernel<1, 8>);
    return launch(attn_kv4_kernel<2, 4>);
}
