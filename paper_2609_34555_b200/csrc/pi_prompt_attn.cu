// Causal attention over a packed batch of prompts:  out = softmax(q K^T / sqrt(D)) V,  query i of a sequence with n queries and m
// keys seeing the keys j <= i + m - n.
//
// 4 D operations a (query head, visible pair) against 4 D bytes a (key, KV head): for prompts of more than a few hundred tokens
// the matrix pipe is what the call cannot do without, so both products run on tcgen05.  One CTA has the 256 rows of two query
// tiles (A and B): a row is a (token, query head) pair of ONE KV head, G rows a token, so that the G heads share every key and
// value that is fetched, and a chunk of a few tokens still fills its rows.  K and V tiles of 128 tokens come by TMA into a ring of
// five stages; S = Q K^T (128 x 128, fp32) and O (128 x 128, fp32) of both query tiles fill the 512 columns of tensor memory:
//     warps 0-3, 4-7   softmax of tile A, B: a thread has a row, so its maximum and sum need no other lane
//     warp 8           issues the products: ... O_A += P_A V(j), S_A = Q_A K(j+1)^T, O_B += P_B V(j), S_B = Q_B K(j+1)^T ...
//     warp 9           TMA, and the care for values that some row must not see
// While one tile's softmax runs, the tensor pipe works on the other tile's products.  P takes S's place in tensor memory, in 16 bits: a
// weight is rounded to the type of V, which adds to a result in the mean square about what the rounding of the output itself does (the
// tensor core wants both operands of one type; weights in two halves would cost half as much again on the pipe that bounds the
// call).  The sum of the weights, the maxima and all products' sums are in 32 bits.
//
// The maximum that is taken off moves only when a score exceeds it by a factor of 2^8 after the exponential, so that O is seldom
// rescaled; then the softmax warps do it themselves, between their S and their P, when no product of their tile is in flight.
#include <cuda_fp16.h>

#include "pi_attn_core.cuh"

namespace {

using namespace pi_attn;

constexpr int PA_THREADS = 384;                  // three warpgroups: softmax of A, softmax of B, the rest (two of its warps have nothing to do)
// registers of a softmax thread and of the others: 256 x 208 + 128 x 80 of the 384 x 168 that the block is launched with
constexpr int PA_SOFTMAX_REGS = 208, PA_OTHER_REGS = 80;
static_assert(256 * PA_SOFTMAX_REGS + 128 * PA_OTHER_REGS <= PA_THREADS * 168, "more than the block has");
constexpr int PA_ROWS = 128;                        // rows of a query tile, and tokens of a K or V tile
constexpr int PA_STAGES = 5;
constexpr int PA_HALF = PA_ROWS * 128;              // 64 channels of 128 rows
constexpr int PA_TILE = 2 * PA_HALF;
constexpr float PA_NO_MAX = -3.40282347e38f;        // the lowest number, for -infinity in the running maximum: differences are no NaN
constexpr float PA_FAR = 1024.f;
constexpr uint32_t PA_TMEM_S = 0, PA_TMEM_O = 256;  // columns: S (and P) of A and B, O of A and B

struct PromptParams {
    const int32_t* q_start;
    const int32_t* k_start;
    void* out;
    float* lse;
    const void* v;
    pi_status_ref st;
    long long wait_cycles, v_tok, v_head;
    float scale_log2;                               // log2(e) / sqrt(D)
    int n_seqs, Hq, Hkv, G, tq, n_q, n_k;           // tq: tokens of a query tile
};

// ---------------------------------------------------------------- PTX wrappers
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void tma_load_q(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// D[tensor memory] (+)= A[shared memory] B[shared memory]
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u) : "memory");
}
// D[tensor memory] (+)= A[tensor memory] B[shared memory]
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u) : "memory");
}
// 32 columns of this warp's 32 lanes
__device__ __forceinline__ void tc_ld32(uint32_t addr, float* r) {
    uint32_t* u = reinterpret_cast<uint32_t*>(r);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]),
          "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]),
          "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(addr));
}
__device__ __forceinline__ void tc_st32(uint32_t addr, const uint32_t* u) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(addr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]),
          "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]), "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]),
          "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]), "r"(u[30]), "r"(u[31])
        : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float pa_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float pa_max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// a b + c, a pair in one operation
__device__ __forceinline__ float2 pa_fma(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 pa_add(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// Shared-memory matrices of 128-byte rows, 128-byte swizzle (eight rows of 128 bytes repeat).  Q and K: rows are what the result
// has rows or columns of, 64 channels a row; 8 rows further on is 1024 bytes.  V: rows are what is summed over; 64 channels
// further on is the other half of the tile (16384 bytes), eight tokens further on 1024 bytes.
__device__ __forceinline__ uint64_t desc_k_major(uint32_t addr) {
    return static_cast<uint64_t>((addr >> 4) & 0x3fffu) | (1ull << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t desc_mn_major(uint32_t addr) {
    return static_cast<uint64_t>((addr >> 4) & 0x3fffu) | (static_cast<uint64_t>(PA_HALF >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

template <typename T> struct Form;
template <> struct Form<__nv_bfloat16> {
    static constexpr uint32_t code = 1u;            // of the instruction descriptor
    static constexpr uint32_t exponent = 0x7f807f80u, one = 0x00800080u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16(lo, hi); }
    static __device__ __forceinline__ float value(uint32_t half) { return __uint_as_float(half << 16); }
};
template <> struct Form<__half> {
    static constexpr uint32_t code = 0u;
    static constexpr uint32_t exponent = 0x7c007c00u, one = 0x04000400u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ float value(uint32_t half) { return __half2float(__ushort_as_half(static_cast<unsigned short>(half))); }
};
// The halves of a word that are infinite or NaN, as the upper bit of each.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & Form<T>::exponent) + Form<T>::one) & 0x80008000u; }

struct Span { int q0, n, k0, m; };                  // a sequence's queries and keys

// Sequence s, or nothing where its bounds make no sense.
__device__ __forceinline__ Span span_of(const PromptParams& p, int s, bool tell) {
    Span x = {0, 0, 0, 0};
    if (s >= p.n_seqs) return x;
    const int a = p.q_start[s], b = p.q_start[s + 1], c = p.k_start[s], d = p.k_start[s + 1];
    if (a < 0 || b < a || b > p.n_q || c < 0 || d < c || d > p.n_k) {
        const bool q_wrong = a < 0 || b < a || b > p.n_q;
        if (tell) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_PROMPT, s, q_wrong ? a : c, q_wrong ? b : d);
        return x;
    }
    x.q0 = a; x.n = b - a; x.k0 = c; x.m = d - c;
    return x;
}

template <typename T>
__global__ void __launch_bounds__(PA_THREADS, 1)
prompt_attn_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, PromptParams p) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_bar[2 + 3 * PA_STAGES + 6];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_odd;                  // s_odd: values that are no numbers were taken out of a tile
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pi_grid_dependency_wait();
    pi_launch_dependents();

    // ---- the CTA's work: blocks of 2 tq tokens, counted from the last one of the last sequence (the longest come first), heads innermost
    const int h = static_cast<int>(blockIdx.x % static_cast<unsigned>(p.Hkv)), item = static_cast<int>(blockIdx.x / static_cast<unsigned>(p.Hkv));
    const int per_block = 2 * p.tq;
    int total = 0;
    for (int s0 = 0; s0 < p.n_seqs; s0 += 32) total += (span_of(p, s0 + lane, blockIdx.x == 0 && warp == 0).n + per_block - 1) / per_block;
    total = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(total)));
    if (item >= total) return;
    int at = total - 1 - item, block = 0;
    Span me = {0, 0, 0, 0};
    for (int s0 = 0; s0 < p.n_seqs; s0 += 32) {
        const Span x = span_of(p, s0 + lane, false);
        const int nb = (x.n + per_block - 1) / per_block;
        int upto = nb;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += y;
        }
        const unsigned found = __ballot_sync(0xffffffffu, at < upto);
        if (found) {
            const int from = __ffs(static_cast<int>(found)) - 1;
            block = at - __shfl_sync(0xffffffffu, upto - nb, from);
            me.q0 = __shfl_sync(0xffffffffu, x.q0, from); me.n = __shfl_sync(0xffffffffu, x.n, from);
            me.k0 = __shfl_sync(0xffffffffu, x.k0, from); me.m = __shfl_sync(0xffffffffu, x.m, from);
            break;
        }
        at -= __shfl_sync(0xffffffffu, upto, 31);
    }
    const int first = block * per_block;            // the block's first token
    const int off = me.m - me.n;                    // token i sees the keys j < i + off + 1
    const int n_a = min(p.tq, me.n - first), n_b = min(p.tq, max(0, me.n - first - p.tq));
    auto seen_by = [&](int i) { return min(max(i + off + 1, 0), me.m); };
    const int tiles_a = (seen_by(first + n_a - 1) + PA_ROWS - 1) / PA_ROWS, tiles_b = n_b ? (seen_by(first + p.tq + n_b - 1) + PA_ROWS - 1) / PA_ROWS : 0;
    const int n_tiles = max(tiles_a, tiles_b);
    const int odd_from = seen_by(first) / PA_ROWS;  // from this tile on, some row of the block does not see all of a tile

    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = smem + 2 * PA_TILE;
    const uint32_t bars = smem_u32(s_bar);
    const uint32_t q_full = bars, drained = bars + 8, kv_full = bars + 16, kv_empty = kv_full + 8 * PA_STAGES, s_full = kv_empty + 8 * PA_STAGES, p_full = s_full + 16,
                   o_full = p_full + 16, v_good = o_full + 16;
    if (tid == 0) {
        mbar_init(q_full, 1);
        mbar_init(drained, 1);
        for (int i = 0; i < PA_STAGES; ++i) { mbar_init(kv_full + 8 * i, 1); mbar_init(kv_empty + 8 * i, 1); mbar_init(v_good + 8 * i, 1); }
        for (int t = 0; t < 2; ++t) { mbar_init(s_full + 8 * t, 1); mbar_init(p_full + 8 * t, 4); mbar_init(o_full + 8 * t, 1); }
        s_abort = 0;
        s_odd = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    volatile int* abort = &s_abort;

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PA_SOFTMAX_REGS));
        // ---- softmax: thread = row r of tile t, token r / G, head r % G
        const int t = warp >> 2, r = tid & 127, tok = r / p.G, g = r - tok * p.G;
        const int n_tok = t ? n_b : n_a, tiles = t ? tiles_b : tiles_a;
        const bool real = tok < n_tok && tok < p.tq;
        const int i = first + t * p.tq + tok;
        const int seen = real ? seen_by(i) : INT32_MAX;      // (rows of no query may be anything: none is looked at)
        const int all_see = __reduce_min_sync(0xffffffffu, seen);
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;      // the warp's 32 lanes of tensor memory
        const uint32_t at_s = tmem + lanes + PA_TMEM_S + 128 * t, at_o = tmem + lanes + PA_TMEM_O + 128 * t;
        const float c = p.scale_log2;
        float m = PA_NO_MAX, mc = PA_NO_MAX, l = 0.f;      // the reference of the row's weights, as a score and times c; their sum
        bool far = false;
        bool alive = true;
        for (int j = 0; j < tiles; ++j) {
            if (!mbar_wait(s_full + 8 * t, j & 1, abort, p.wait_cycles)) { alive = false; break; }
            tc_fence_after();
            float s[128];
#pragma unroll
            for (int x = 0; x < 4; ++x) tc_ld32(at_s + 32 * x, s + 32 * x);
            tc_wait_ld();
            if ((j + 1) * PA_ROWS > all_see) {
                const int left = seen - j * PA_ROWS;
#pragma unroll
                for (int x = 0; x < 128; ++x) s[x] = x < left ? s[x] : -INFINITY;
            }
            float mx4[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                mx4[x] = fmaxf(s[x], s[x + 4]);
#pragma unroll
                for (int y = 8; y < 128; y += 8) mx4[x] = pa_max3(mx4[x], s[x + y], s[x + y + 4]);
            }
            const float mx = fmaxf(pa_max3(mx4[0], mx4[1], mx4[2]), mx4[3]);
            if (__any_sync(0xffffffffu, mx * c - mc > 8.f)) {
                const float m_new = fmaxf(m, mx), mc_new = m_new * c;
                // (far from 0 the reference's own rounding counts: see below)
                const float alpha = pa_ex2(fabsf(mc_new) > PA_FAR ? (m - m_new) * c : mc - mc_new);
                m = m_new;
                mc = mc_new;
                far = __any_sync(0xffffffffu, fabsf(mc) > PA_FAR);
                l *= alpha;
                if (j > 0) {
#pragma unroll 1
                    for (int x = 0; x < 4; ++x) {
                        float o[32];
                        tc_ld32(at_o + 32 * x, o);
                        tc_wait_ld();
#pragma unroll
                        for (int y = 0; y < 32; ++y) o[y] *= alpha;
                        tc_st32(at_o + 32 * x, reinterpret_cast<const uint32_t*>(o));
                    }
                    tc_wait_st();
                }
            }
            // The weight is 2^(s c - mc), one fused operation and the exponential: mc is what the row's weights are counted from, and its
            // rounding is in all of them alike.  Where it is large that rounding would leave the range of the weights, so there the
            // maximum is taken off before the scale.
            float2 less = make_float2(-mc, -mc);
            if (far) {
#pragma unroll
                for (int x = 0; x < 128; ++x) s[x] -= m;
                less = make_float2(0.f, 0.f);
            }
            const float2 cc = make_float2(c, c);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint32_t w[32];
#pragma unroll
                for (int y = 0; y < 32; ++y) {
                    float2 v = pa_fma(make_float2(s[64 * x + 2 * y], s[64 * x + 2 * y + 1]), cc, less);
                    v.x = pa_ex2(v.x);
                    v.y = pa_ex2(v.y);
                    sum = pa_add(sum, v);
                    w[y] = Form<T>::pack(v.x, v.y);
                }
                tc_st32(at_s + 32 * x, w);
            }
            l += sum.x + sum.y;
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full + 8 * t);
        }
        // ---- the row's result
        if (alive && tiles > 0) alive = mbar_wait(o_full + 8 * t, 0, abort, p.wait_cycles);
        if (alive && n_tok > 0) {
            tc_fence_after();
            const bool none = l == 0.f;             // (a NaN among the sums has to come through)
            const float inv = none ? 0.f : 1.f / l;
            const size_t row = static_cast<size_t>(me.q0 + i) * p.Hq + static_cast<size_t>(h) * p.G + g;
            const bool odd = s_odd != 0;
#pragma unroll 1
            for (int x = 0; x < 4; ++x) {
                float o[32];
                if (tiles > 0) {
                    tc_ld32(at_o + 32 * x, o);
                    tc_wait_ld();
                }
                if (odd && real) {                  // what was taken out of the values: infinities and NaN that the row does see
                    for (int k = odd_from * PA_ROWS; k < seen; ++k) {
                        const uint32_t* v = reinterpret_cast<const uint32_t*>(static_cast<const T*>(p.v) + (me.k0 + k) * p.v_tok + h * p.v_head + 32 * x);
#pragma unroll
                        for (int y = 0; y < 16; ++y) {
                            const uint32_t w = v[y], bad = not_finite<T>(w);
                            if (bad & 0x8000u) o[2 * y] += Form<T>::value(w & 0xffffu);
                            if (bad & 0x80000000u) o[2 * y + 1] += Form<T>::value(w >> 16);
                        }
                    }
                }
                if (!real) continue;
                uint4* to = reinterpret_cast<uint4*>(static_cast<T*>(p.out) + row * PI_HEAD_DIM + 32 * x);
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    uint32_t w[4];
#pragma unroll
                    for (int z = 0; z < 4; ++z) w[z] = none ? 0u : Form<T>::pack(o[8 * y + 2 * z] * inv, o[8 * y + 2 * z + 1] * inv);
                    to[y] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            if (real && p.lse) p.lse[row] = none ? -INFINITY : (mc + log2f(l)) * 0.6931471805599453f;
        }
        tc_fence_before();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PA_OTHER_REGS));
        if (warp == 9) {
            // ---- TMA: K0 V0 K1 V1 ...; the whole warp waits, one lane issues.  Three loads behind, a V tile that some row must not
            // see all of is looked through: rows behind the sequence's end become 0, and so does every value that is no number
            // (its weight would be 0 where it is masked, and 0 times it is none); those are put back at the end, row by row.
            const int loads = 2 * n_tiles;
            auto look = [&](int n) -> bool {            // load n is in the ring: is it such a V tile?
                const int j = n >> 1;
                if (!(n & 1) || j < odd_from) return true;
                if (!mbar_wait(kv_full + 8 * (n % PA_STAGES), (n / PA_STAGES) & 1, abort, p.wait_cycles)) return false;
                const uint32_t tile = ring + (n % PA_STAGES) * PA_TILE;
                const int real = me.m - j * PA_ROWS;    // rows of the sequence
                bool odd = false;
#pragma unroll 4
                for (int i = lane; i < PA_TILE / 16; i += 32) {
                    const int row = (i >> 3) & (PA_ROWS - 1);
                    uint32_t w[4];
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(tile + i * 16));
                    const uint32_t bad = not_finite<T>(w[0]) | not_finite<T>(w[1]) | not_finite<T>(w[2]) | not_finite<T>(w[3]);
                    if (row >= real) w[0] = w[1] = w[2] = w[3] = 0u;
                    else if (bad) {
                        odd = true;
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[k] &= ~((not_finite<T>(w[k]) >> 15) * 0xffffu);
                    }
                    if (row >= real || bad) asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(tile + i * 16), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                }
                if (odd) s_odd = 1;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(v_good + 8 * (n % PA_STAGES));
                return true;
            };
            if (n_tiles > 0 && lane == 0) {
                const uint32_t bytes = static_cast<uint32_t>(p.tq) * p.G * 128u;
                mbar_expect_tx(q_full, bytes * (n_b ? 4u : 2u));
                for (int t = 0; t < (n_b ? 2 : 1); ++t)
                    for (int x = 0; x < 2; ++x) tma_load_q(smem + t * PA_TILE + x * PA_HALF, &map_q, q_full, 64 * x, 0, h, me.q0 + first + t * p.tq);
            }
            int n = 0;
            bool alive = true;
            for (; n < loads && alive; ++n) {
                const int stage = n % PA_STAGES;
                if (n >= PA_STAGES && !mbar_wait(kv_empty + 8 * stage, (n / PA_STAGES - 1) & 1, abort, p.wait_cycles)) break;
                if (lane == 0) {
                    const CUtensorMap* map = (n & 1) ? &map_v : &map_k;
                    mbar_expect_tx(kv_full + 8 * stage, PA_TILE);
                    for (int x = 0; x < 2; ++x) tma_load_3d(ring + stage * PA_TILE + x * PA_HALF, map, kv_full + 8 * stage, 64 * x, h, me.k0 + (n >> 1) * PA_ROWS);
                }
                __syncwarp();
                if (n >= 3) alive = look(n - 3);
            }
            for (int i = max(0, n - 3); i < n && alive; ++i) alive = look(i);
            if (*abort) {                               // copies in flight end before the CTA does
                volatile int none = 0;
                if (n_tiles > 0) mbar_wait(q_full, 0, &none, p.wait_cycles);
                for (int i = max(0, n - PA_STAGES); i < n; ++i) mbar_wait(kv_full + 8 * (i % PA_STAGES), (i / PA_STAGES) & 1, &none, p.wait_cycles);
            }
        } else if (warp == 8) {
            if (lane == 0 && n_tiles > 0) {
                constexpr uint32_t base = (1u << 4) | (Form<T>::code << 7) | (Form<T>::code << 10) | (static_cast<uint32_t>(PA_ROWS >> 3) << 17) | (static_cast<uint32_t>(PA_ROWS >> 4) << 24);
                constexpr uint32_t idesc_s = base, idesc_o = base | (1u << 16);      // V: channels run along its rows
                auto product_s = [&](int t, int n) {
                    const uint64_t a = desc_k_major(smem + t * PA_TILE), b = desc_k_major(ring + (n % PA_STAGES) * PA_TILE);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint64_t step = static_cast<uint64_t>(((k >> 2) * PA_HALF + (k & 3) * 32) >> 4);
                        tc_mma_ss(tmem + PA_TMEM_S + 128 * t, a + step, b + step, idesc_s, k > 0);
                    }
                    tc_commit(s_full + 8 * t);
                };
                auto product_o = [&](int t, int n, bool add) {
                    const uint64_t b = desc_mn_major(ring + (n % PA_STAGES) * PA_TILE);
#pragma unroll
                    for (int k = 0; k < 8; ++k) tc_mma_ts(tmem + PA_TMEM_O + 128 * t, tmem + PA_TMEM_S + 128 * t + 8 * k, b + static_cast<uint64_t>((k * 2048) >> 4), idesc_o, add || k > 0);
                };
                const int tiles[2] = {tiles_a, tiles_b};
                bool alive = mbar_wait(q_full, 0, abort, p.wait_cycles) && mbar_wait(kv_full, 0, abort, p.wait_cycles);
                if (alive) {
                    tc_fence_after();
                    for (int t = 0; t < 2; ++t)
                        if (tiles[t] > 0) product_s(t, 0);
                    tc_commit(kv_empty);
                }
                for (int j = 0; j < n_tiles && alive; ++j) {
                    const int nv = 2 * j + 1, nk = 2 * j + 2;
                    if (j < odd_from) alive = mbar_wait(kv_full + 8 * (nv % PA_STAGES), (nv / PA_STAGES) & 1, abort, p.wait_cycles);
                    else alive = mbar_wait(v_good + 8 * (nv % PA_STAGES), ((j - odd_from) / PA_STAGES) & 1, abort, p.wait_cycles);     // (a V tile meets its stage again five tiles on)
                    if (alive && j + 1 < n_tiles) alive = mbar_wait(kv_full + 8 * (nk % PA_STAGES), (nk / PA_STAGES) & 1, abort, p.wait_cycles);
                    for (int t = 0; t < 2 && alive; ++t) {
                        if (j >= tiles[t]) continue;
                        alive = mbar_wait(p_full + 8 * t, j & 1, abort, p.wait_cycles);
                        if (!alive) break;
                        tc_fence_after();
                        product_o(t, nv, j > 0);
                        if (j + 1 < tiles[t]) product_s(t, nk);
                        else tc_commit(o_full + 8 * t);
                    }
                    if (!alive) break;
                    tc_commit(kv_empty + 8 * (nv % PA_STAGES));
                    if (j + 1 < n_tiles) tc_commit(kv_empty + 8 * (nk % PA_STAGES));
                }
                // products in flight end before the CTA does
                volatile int none = 0;
                tc_commit(drained);
                mbar_wait(drained, 0, &none, p.wait_cycles);
            }
            __syncwarp();
        }
    }
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
    if (tid == 0 && s_abort) pi_report(p.st, PI_ERR_TIMEOUT, PI_STAGE_PROMPT, static_cast<int>(blockIdx.x), block, n_tiles);
}

typedef CUresult (*encode_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int make_map(pi_ctx* c, CUtensorMap* map, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    const cuuint32_t step[4] = {1, 1, 1, 1};
    const CUresult r = reinterpret_cast<encode_fn>(c->encode_tiled_fn)(map, type, rank, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                                                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? PI_OK : PI_ERR_CUDA;
}

}  // namespace

int pi_launch_prompt_attn(pi_ctx* c, int n_seqs, int dtype, int n_q, int n_k, const void* q, int64_t q_tok, int64_t q_head, const void* k, int64_t k_tok, int64_t k_head,
                          const void* v, int64_t v_tok, int64_t v_head, const int32_t* q_start, const int32_t* k_start, void* out, float* lse, cudaStream_t stream) {
    const pi_config& cfg = c->cfg;
    PromptParams p;
    p.q_start = q_start; p.k_start = k_start;
    p.out = out; p.lse = lse; p.v = v; p.v_tok = v_tok; p.v_head = v_head;
    p.st = pi_status_of(c);
    p.wait_cycles = c->wait_limit_cycles;
    p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(PI_HEAD_DIM));
    p.n_seqs = n_seqs; p.Hq = cfg.n_q_heads; p.Hkv = cfg.n_kv_heads; p.G = cfg.n_q_heads / cfg.n_kv_heads; p.n_q = n_q; p.n_k = n_k;
    p.tq = PA_ROWS / p.G;
    const CUtensorMapDataType type = dtype == PI_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    CUtensorMap map_q, map_k, map_v;
    {
        const cuuint64_t dims[4] = {PI_HEAD_DIM, static_cast<cuuint64_t>(p.G), static_cast<cuuint64_t>(p.Hkv), static_cast<cuuint64_t>(n_q)};
        const cuuint64_t strides[3] = {static_cast<cuuint64_t>(q_head) * 2, static_cast<cuuint64_t>(q_head) * 2 * p.G, static_cast<cuuint64_t>(q_tok) * 2};
        const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(p.G), 1, static_cast<cuuint32_t>(p.tq)};
        const int rc = make_map(c, &map_q, type, 4, q, dims, strides, box);
        if (rc != PI_OK) return rc;
    }
    for (int i = 0; i < 2; ++i) {
        // (without a single key nothing is fetched through these, but a map has to stand for something)
        const cuuint64_t dims[3] = {PI_HEAD_DIM, static_cast<cuuint64_t>(n_k ? p.Hkv : 1), static_cast<cuuint64_t>(n_k ? n_k : 1)};
        const cuuint64_t strides[2] = {static_cast<cuuint64_t>(i ? v_head : k_head) * 2, static_cast<cuuint64_t>(i ? v_tok : k_tok) * 2};
        const cuuint32_t box[3] = {64, 1, PA_ROWS};
        const int rc = make_map(c, i ? &map_v : &map_k, type, 3, n_k ? (i ? v : k) : q, dims, strides, box);
        if (rc != PI_OK) return rc;
    }
    const long long blocks = n_q / (2 * p.tq) + static_cast<long long>(n_seqs < n_q ? n_seqs : n_q), grid = blocks * p.Hkv;
    if (grid > INT32_MAX) return PI_ERR_UNSUPPORTED_DIM;
    const size_t smem = 2 * PA_TILE + PA_STAGES * PA_TILE + 1024;
    auto launch = [&](auto kernel) -> int {
        PI_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
        PI_CUDA_TRY(pi_launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(PA_THREADS), smem, stream, map_q, map_k, map_v, p));
        return PI_OK;
    };
    return dtype == PI_DTYPE_BF16 ? launch(prompt_attn_kernel<__nv_bfloat16>) : launch(prompt_attn_kernel<__half>);
}
