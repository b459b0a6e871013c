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
//     warp 9           TMA
//     warp 10          which piece of work comes next
//     warp 11          looks through the V tiles that some row must not see all of
// While one tile's softmax runs, the tensor pipe works on the other tile's products.  P takes S's place in tensor memory, in 16 bits: a
// weight is rounded to the type of V, which adds to a result in the mean square about what the rounding of the output itself does (the
// tensor core wants both operands of one type; weights in two halves would cost half as much again on the pipe that bounds the
// call).  In fp16 they are counted 2^7 times as large, up to 2^15, so that they keep 11 bits down to 2^-21 of the row's reference and are off
// by 2^-32 of it at most below that: a long tail under one large score keeps its share.  The sum of the weights, the maxima and all
// products' sums are in 32 bits.
//
// An item is a block of up to 2 tq tokens (tq = 128 / G; of tq where SMs would be idle) of a sequence and a KV head.  Where a block has one query tile, the two softmax groups
// take every second K/V tile of it and are joined at the end.  CTAs stay and take over the places of CTAs that have not begun, the longest
// sequences first, so that the next item's loads and first product run under the last one's end; few items with many keys are shared by
// clusters of two to eight CTAs (the launcher's rule).
//
// The maximum that is taken off moves only when a score exceeds it by a factor of 2^8 after the exponential, so that O is seldom
// rescaled; then the softmax warps do it themselves, between their S and their P, when no product of their tile is in flight.
//
// Measured on a B200 (32 query heads, 8 KV heads, bf16; 1 643 TFLOP/s is what a library product reaches in a short run, 1 394 for seconds):
// one prompt of 8 192 tokens 434 us, 1 267 TFLOP/s, in a run of a few milliseconds, 496 us for longer, where the power limit takes the
// clock from 1.7 to 1.45 GHz; 23 prompts of 0 to 1 500 tokens 173 us, 214 for longer; 77 tokens 7.0 us; 16 sequences of one token after 16 384
// 171 us, 6.3 TB/s, after 0 to 16 384 87 us (105 before the longest sequences came first); 500 tokens after 65 536 with 64 heads in fp16 920 to 950 us.  An iteration (two query tiles, one K/V tile) takes 3 270 cycles,
// of which the tensor pipe and the exponentials are busy for 2 048 each.
// Tried and not taken: a share of the exponentials as polynomials (3 % fewer cycles, the same time), P handed over in two halves, a
// reference without each tile's maximum, clusters of 16; the next item's first product ahead of this one's last, weights of masked keys left
// out 32 at a time (both cost the steady state more than they gave); a ring of four stages to make room for whole-line stores.
#include <cuda_fp16.h>

#include "pi_attn_core.cuh"

namespace {

using namespace pi_attn;

constexpr int PA_THREADS = 384;                  // three warpgroups: softmax of A, softmax of B, the rest
// registers of a softmax thread and of the others: 256 x 208 + 128 x 88 of the 384 x 168 that the block is launched with
constexpr int PA_SOFTMAX_REGS = 208, PA_OTHER_REGS = 88;
static_assert(256 * PA_SOFTMAX_REGS + 128 * PA_OTHER_REGS <= PA_THREADS * 168, "more than the block has");
constexpr int PA_SOFTMAX = 256;                     // threads of the softmax warps
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
    int per_block;                                  // tokens of an item: 2 tq, or tq
    uint32_t by_block;                              // 2^32 / per_block, rounded up
    int log_hkv;
    bool wide;                                      // out is aligned to 32 bytes
    int hold_last;                                  // test only: an item's last V tile is never fetched
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
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0u;
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
// (nothing that is made of what a load brings may be moved in front of the wait)
template <int N>
__device__ __forceinline__ void tc_wait_ld(float (&r)[N]) {
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+f"(r[i]));
}
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
    static constexpr float lift = 0.f;              // weights are 2^lift times as large: a weight is at most 2^8 before
    static constexpr uint32_t exponent = 0x7f807f80u, one = 0x00800080u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16(lo, hi); }
    // the larger magnitudes of two pairs, NaN where either is NaN (one operation)
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
        return *reinterpret_cast<const uint32_t*>(&m);
    }
    static __device__ __forceinline__ float value(uint32_t half) { return __uint_as_float(half << 16); }
};
template <> struct Form<__half> {
    static constexpr uint32_t code = 0u;
    static constexpr float lift = 7.f;
    static constexpr uint32_t exponent = 0x7c007c00u, one = 0x04000400u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        const __half2 m = __hmax2_nan(*reinterpret_cast<const __half2*>(&a), __habs2(*reinterpret_cast<const __half2*>(&b)));
        return *reinterpret_cast<const uint32_t*>(&m);
    }
    static __device__ __forceinline__ float value(uint32_t half) { return __half2float(__ushort_as_half(static_cast<unsigned short>(half))); }
};
// The halves of a word that are infinite or NaN, as the upper bit of each.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & Form<T>::exponent) + Form<T>::one) & 0x80008000u; }

struct Span { int q0, n, k0, m; };                  // a sequence's queries and keys

__device__ __forceinline__ bool makes_sense(const PromptParams& p, int a, int b, int c, int d) { return a >= 0 && b >= a && b <= p.n_q && c >= 0 && d >= c && d <= p.n_k; }
// Sequence s, or nothing where its bounds make no sense.
__device__ __forceinline__ Span span_of(const PromptParams& p, int s, bool tell) {
    Span x = {0, 0, 0, 0};
    if (s >= p.n_seqs) return x;
    const int a = p.q_start[s], b = p.q_start[s + 1], c = p.k_start[s], d = p.k_start[s + 1];
    if (!makes_sense(p, a, b, c, d)) {
        const bool q_wrong = a < 0 || b < a || b > p.n_q;
        if (tell) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_PROMPT, s, q_wrong ? a : c, q_wrong ? b : d);
        return x;
    }
    x.q0 = a; x.n = b - a; x.k0 = c; x.m = d - c;
    return x;
}

// One piece of work: a block of up to 2 tq tokens of a sequence and a KV head.
struct Item {
    int q0, n, k0, m;                               // the sequence
    int first, h;                                   // the block's first token, its KV head; h < 0: there is no more work
};

// What follows from an item, for every role alike.
struct Plan {
    int off, n_a, n_b, lo, hi, tiles_a, tiles_b, seen_first, odd_from, last_a, last_b;      // last_: keys that the last token of tile A, B sees
    bool pair;
    __device__ __forceinline__ Plan(const PromptParams& p, const Item& w, int rank, int split) {
        off = w.m - w.n;                            // token i sees the keys j < i + off + 1
        n_a = min(p.tq, w.n - w.first);
        n_b = min(p.per_block - p.tq, max(0, w.n - w.first - p.tq));
        last_a = seen(w, w.first + n_a - 1);
        last_b = n_b ? seen(w, w.first + p.tq + n_b - 1) : last_a;
        tiles_a = (last_a + PA_ROWS - 1) / PA_ROWS;
        tiles_b = (last_b + PA_ROWS - 1) / PA_ROWS;
        pair = n_b == 0;                            // one query tile: the softmax groups take every second K/V tile each
        const int all = max(tiles_a, tiles_b);
        lo = static_cast<int>(static_cast<long long>(all) * rank / split);
        hi = static_cast<int>(static_cast<long long>(all) * (rank + 1) / split);
        tiles_a = min(tiles_a, hi);
        tiles_b = min(tiles_b, hi);
        seen_first = seen(w, w.first);
        odd_from = seen_first / PA_ROWS;            // from this tile on, some row of the block does not see all of a tile
    }
    __device__ __forceinline__ int seen(const Item& w, int i) const { return min(max(i + off + 1, 0), w.m); }
    // group t's first K/V tile, and how far it is to the next
    __device__ __forceinline__ int begin(int t) const { return pair ? lo + t : lo; }
    __device__ __forceinline__ int step() const { return pair ? 2 : 1; }
    __device__ __forceinline__ int end(int t) const { return t ? tiles_b : tiles_a; }
};

// The waits and arrivals across a cluster: what was written before the arrival is seen behind the wait.
__device__ __forceinline__ bool mbar_try_cluster(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort, long long limit) {
    const long long t0 = clock64();
    while (!mbar_try_cluster(bar, parity)) {
        if (*abort) return false;
        if (clock64() - t0 > limit) { *abort = 1; return false; }
    }
    return true;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// Barriers, in 8-byte places.
enum : uint32_t {
    B_Q_FULL = 0, B_Q_EMPTY = 1, B_DRAINED = 2, B_MERGED = 3, B_HALF = 4, B_NEXT = 5, B_ITEM_FULL = 6, B_ITEM_EMPTY = 8, B_S_FULL = 10, B_P_FULL = 12, B_O_FULL = 14,
    B_ALL = 16, B_SHARE_FULL = 17, B_SHARE_EMPTY = 18, B_WANTED = 19, B_KV_FULL = 20, B_KV_EMPTY = B_KV_FULL + PA_STAGES, B_V_GOOD = B_KV_EMPTY + PA_STAGES, B_COUNT = B_V_GOOD + PA_STAGES
};

constexpr uint32_t PA_ML_AT = 2 * PA_ROWS * 512;    // a cluster's shares: [256 rows][128] in 32 bits, then every row's reference and sum
constexpr int GROUPS = 4;                           // times 1024 sequences: as many as a context may have
constexpr int PA_FEW = 64;                          // so many rows have their shares in query tile B's place, which such an item leaves free

// A CTA takes one item after the other: it begins with its own place in the grid and then takes over CTAs that have not begun yet, so that loads,
// barriers and tensor memory run on.  SPLIT: a cluster of CTAs does so, and shares every item, each with a run of its K/V tiles.
template <typename T, bool SPLIT>
__global__ void __launch_bounds__(PA_THREADS, 1)
prompt_attn_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, PromptParams p) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(16) uint32_t s_next[4];    // what came of taking over a CTA
    __shared__ __align__(8) uint64_t s_bar[B_COUNT];
    __shared__ Item s_item[2];
    __shared__ float2 s_ml[PA_ROWS];                // tile A alone: reference and sum of group B's rows
    __shared__ float2 s_share[PA_FEW];              // SPLIT, few rows: reference and sum of the CTA's share
    __shared__ unsigned char s_order[32];           // of 32 sequences, by their keys
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_odd[2];               // s_odd: values that are no numbers were taken out of a tile
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int split = SPLIT ? static_cast<int>(cluster_nctarank()) : 1, rank = SPLIT ? static_cast<int>(cluster_ctarank()) : 0;
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = smem + 2 * PA_TILE;
    const uint32_t bars = smem_u32(s_bar);
    auto bar = [&](uint32_t place) { return bars + 8 * place; };
    if (tid == 0) {
        for (uint32_t i = 0; i < B_COUNT; ++i) {
            const bool by_warps = i == B_P_FULL || i == B_P_FULL + 1 || i == B_MERGED || i == B_HALF;
            mbar_init(bar(i), by_warps ? 4 : i == B_ALL ? 8 : i == B_SHARE_FULL || i == B_SHARE_EMPTY ? 8 * split : i == B_ITEM_EMPTY || i == B_ITEM_EMPTY + 1 ? 11 * split : i >= B_KV_EMPTY && i < B_KV_EMPTY + PA_STAGES ? 2 : 1);
        }
        s_abort = 0;
        s_odd[0] = s_odd[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == 9 && lane < 3) asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &map_q : lane == 1 ? &map_k : &map_v));
    pi_grid_dependency_wait();
    pi_launch_dependents();
    tc_fence_before();
    if (SPLIT) cluster_sync_all();                  // (the others' barriers are there too)
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    volatile int* abort = &s_abort;
    // A warp's waits, for what this CTA or (`_cluster`) another has written.  A wait that is given up is given up by all lanes: a warp
    // whose lanes went different ways would stand at its next vote for good.
    auto wait = [&](uint32_t place, uint32_t parity) {
        if (__all_sync(0xffffffffu, mbar_try(bar(place), parity))) return true;
        return __all_sync(0xffffffffu, mbar_wait(bar(place), parity, abort, p.wait_cycles)) != 0;
    };
    auto wait_cluster = [&](uint32_t place, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait_cluster(bar(place), parity, abort, p.wait_cycles)) != 0; };
    auto wait_here = [&](uint32_t place, uint32_t parity) { return SPLIT ? wait_cluster(place, parity) : wait(place, parity); };
    // item number `it` of this CTA, for the roles that are told
    auto item_of = [&](int it, Item& w) -> bool {
        if (!wait_here(B_ITEM_FULL + (it & 1), (it >> 1) & 1)) return false;
        w = s_item[it & 1];
        return w.h >= 0;
    };
    auto done_with = [&](int it) {
        __syncwarp();
        if (lane != 0) return;
        if (SPLIT) mbar_arrive_cluster(map_shared_rank(bar(B_ITEM_EMPTY + (it & 1)), 0));      // rank 0 tells the cluster its items
        else mbar_arrive(bar(B_ITEM_EMPTY + (it & 1)));
    };
    // one arrival of this warp at the same barrier of every CTA of the cluster
    auto arrive_at_all = [&](uint32_t place) {
        __syncwarp();
        if (lane < split) mbar_arrive_cluster(map_shared_rank(bar(place), lane));
    };

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PA_SOFTMAX_REGS));
        // ---- softmax: thread = row r of tile t (of tile A where that is alone), token r / G, head r % G
        const int t = warp >> 2, r = tid & 127, tok = r / p.G, g = r - tok * p.G;
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;      // the warp's 32 lanes of tensor memory
        const uint32_t at_s = tmem + lanes + PA_TMEM_S + 128 * t, at_o = tmem + lanes + PA_TMEM_O + 128 * t;
        const float c = p.scale_log2;
        auto far_off = [](float x) { return fabsf(x) > PA_FAR && x != PA_NO_MAX; };
        uint32_t steps = 0u, results = 0u, merges = 0u;      // so far: S of this tile, O of this tile, items of one query tile
        bool alive = true;
        Item w;
        for (int it = 0; alive && item_of(it, w); ++it) {
            const Plan plan(p, w, rank, split);
            const int n_tok = t && !plan.pair ? plan.n_b : plan.n_a, i = w.first + (t && !plan.pair ? p.tq : 0) + tok;
            const bool real = tok < n_tok;
            const int seen = real ? plan.seen(w, i) : INT32_MAX;     // (rows of no query may be anything: none is looked at)
            const int all_see = __reduce_min_sync(0xffffffffu, seen);
            const int begin = plan.begin(t), end = plan.end(t);
            float m = PA_NO_MAX, mc = PA_NO_MAX, l = 0.f;            // the reference of the row's weights, as a score, and times c less the lift; their sum
            bool far = false;
            for (int j = begin; j < end; j += plan.step(), ++steps) {
                if (!wait(B_S_FULL + t, steps & 1u)) { alive = false; break; }
                tc_fence_after();
                float s[128];
#pragma unroll
                for (int x = 0; x < 4; ++x) tc_ld32(at_s + 32 * x, s + 32 * x);
                tc_wait_ld(s);
                if ((j + 1) * PA_ROWS > all_see) {
                    // (bits of a word for 32 keys: half the operations of 128 comparisons, 37 prompts of 256 tokens 62.6 us instead of 63.9)
                    const int left = seen - j * PA_ROWS;
#pragma unroll
                    for (int x = 0; x < 128; x += 32) {
                        const int here = min(max(left - x, 0), 32);
                        const uint32_t keep = static_cast<uint32_t>((1ull << here) - 1ull);
#pragma unroll
                        for (int y = 0; y < 32; ++y) s[x + y] = (keep >> y) & 1u ? s[x + y] : -INFINITY;
                    }
                }
                float mx4[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    mx4[x] = fmaxf(s[x], s[x + 4]);
#pragma unroll
                    for (int y = 8; y < 128; y += 8) mx4[x] = pa_max3(mx4[x], s[x + y], s[x + y + 4]);
                }
                const float mx = fmaxf(pa_max3(mx4[0], mx4[1], mx4[2]), mx4[3]);
                // (each row by itself: what its neighbours are does not change its bits.  Far from 0 as the weights are counted there: with the reference
                // rounded in both, scores that are far apart might seem equal, and a weight leave its range)
                const bool over = real && (far ? (mx - m) * c > 8.f : mx * c - mc > 8.f + Form<T>::lift);
                if (__any_sync(0xffffffffu, over)) {
                    const float m_new = over ? mx : m, mc_new = over ? mx * c - Form<T>::lift : mc;
                    // (far from 0 the reference's own rounding counts: see below)
                    const float alpha = pa_ex2(far_off(mc_new) ? (m - m_new) * c : mc - mc_new);
                    m = m_new;
                    mc = mc_new;
                    far = far_off(mc);
                    l *= alpha;
                    if (j > begin) {
#pragma unroll 1
                        for (int x = 0; x < 4; ++x) {
                            float o[32];
                            tc_ld32(at_o + 32 * x, o);
                            tc_wait_ld(o);
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
                if (__any_sync(0xffffffffu, far)) {
                    const float off = far ? m : 0.f;             // (a row's bits do not hang on the rows beside it)
#pragma unroll
                    for (int x = 0; x < 128; ++x) s[x] -= off;
                    if (far) less = make_float2(Form<T>::lift, Form<T>::lift);
                }
                const float2 cc = make_float2(c, c);
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    uint32_t u[32];
#pragma unroll
                    for (int y = 0; y < 32; ++y) {
                        float2 v = pa_fma(make_float2(s[64 * x + 2 * y], s[64 * x + 2 * y + 1]), cc, less);
                        v.x = pa_ex2(v.x);
                        v.y = pa_ex2(v.y);
                        sum = pa_add(sum, v);
                        u[y] = Form<T>::pack(v.x, v.y);
                    }
                    tc_st32(at_s + 32 * x, u);
                }
                l += sum.x + sum.y;
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B_P_FULL + t));
            }
            // ---- the row's result
            if (alive && end > begin) alive = wait(B_O_FULL + t, results++ & 1u);
            if (!alive) break;
            tc_fence_after();
            bool some = end > begin;                // there is an O of this group
            bool other_some = false;
            float f = 1.f, f_other = 0.f;
            if (plan.pair) {
                // tile A's rows twice, with every second K/V tile each: group A takes both, out of the same lanes of tensor memory
                if (t == 1) {
                    s_ml[r] = make_float2(mc, l);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(B_HALF));
                } else {
                    if (!wait(B_HALF, merges & 1u)) { alive = false; break; }
                    tc_fence_after();
                    const float2 ml = s_ml[r];
                    other_some = plan.end(1) > plan.begin(1);
                    const float top = fmaxf(mc, ml.x);
                    f = pa_ex2(mc - top);
                    f_other = pa_ex2(ml.x - top);
                    l = l * f + ml.y * f_other;
                    mc = top;
                }
            }
            const bool few = plan.pair && plan.n_a * p.G <= PA_FEW;
            const uint32_t share = smem + (few ? PA_TILE : 0), share_ml = few ? smem_u32(s_share) : smem + PA_ML_AT;
            if (SPLIT) {
                // the last item's shares have been read by all; Q's and the ring's place is free when both groups have their O
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B_ALL));
                if (!wait(B_ALL, it & 1) || (it > 0 && !wait_cluster(B_SHARE_EMPTY, (it - 1) & 1))) { alive = false; break; }
            }
            const bool none = l == 0.f;             // (a NaN among the sums has to come through)
            const float inv = none ? 0.f : 1.f / l;
            const bool odd = s_odd[it & 1] != 0;
            const size_t row = static_cast<size_t>(w.q0 + i) * p.Hq + static_cast<size_t>(w.h) * p.G + g;
            if (!(plan.pair && t == 1)) {
#pragma unroll 1
                for (int x = 0; x < 4; ++x) {
                    float o[32];
                    __syncwarp();                   // (rows of no query, and rows that see different numbers of odd values, come here at different times)
                    if (some) {
                        tc_ld32(at_o + 32 * x, o);
                        tc_wait_ld(o);
                    } else {
#pragma unroll
                        for (int y = 0; y < 32; ++y) o[y] = 0.f;
                    }
                    if (other_some) {
                        float o2[32];
                        tc_ld32(at_o + 128 + 32 * x, o2);
                        tc_wait_ld(o2);
#pragma unroll
                        for (int y = 0; y < 32; ++y) o[y] = o[y] * f + o2[y] * f_other;
                    }
                    if (!real) continue;
                    if (odd) {                      // what was taken out of the values: infinities and NaN that the row does see
                        for (int k = max(plan.seen_first, plan.lo * PA_ROWS); k < min(seen, plan.hi * PA_ROWS); ++k) {
                            const uint32_t* v = reinterpret_cast<const uint32_t*>(static_cast<const T*>(p.v) + (w.k0 + k) * p.v_tok + w.h * p.v_head + 32 * x);
#pragma unroll
                            for (int y = 0; y < 16; ++y) {
                                const uint32_t u = v[y], bad = not_finite<T>(u);
                                if (bad & 0x8000u) o[2 * y] += Form<T>::value(u & 0xffffu);
                                if (bad & 0x80000000u) o[2 * y + 1] += Form<T>::value(u >> 16);
                            }
                        }
                    }
                    if (SPLIT) {                    // the CTA's share of the row, in 32 bits, where the cluster finds it (the ring is done with)
                        const uint32_t at = share + static_cast<uint32_t>(128 * t + r) * 512u;
#pragma unroll
                        for (int y = 0; y < 8; ++y)
                            asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(at + (((8 * x + y) ^ (r & 31)) << 4)), "f"(o[4 * y]), "f"(o[4 * y + 1]), "f"(o[4 * y + 2]), "f"(o[4 * y + 3]) : "memory");
                    } else {
                        // (32 bytes a store where the output allows it, past L1: a lane's stores go to a row of its own, one line each.  23 ragged prompts 188 us,
                        // 196 through L1; with neighbours exchanging halves, for 64 bytes a row, 191)
                        uint4* to = reinterpret_cast<uint4*>(static_cast<T*>(p.out) + row * PI_HEAD_DIM + 32 * x);
                        uint32_t u[16];
#pragma unroll
                        for (int y = 0; y < 16; ++y) u[y] = none ? 0u : Form<T>::pack(o[2 * y] * inv, o[2 * y + 1] * inv);
                        if (p.wide) {
#pragma unroll
                            for (int y = 0; y < 16; y += 8)
                                asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to + y / 4), "r"(u[y]), "r"(u[y + 1]), "r"(u[y + 2]), "r"(u[y + 3]), "r"(u[y + 4]), "r"(u[y + 5]), "r"(u[y + 6]), "r"(u[y + 7]) : "memory");
                        } else {
#pragma unroll
                            for (int y = 0; y < 16; y += 4) to[y / 4] = make_uint4(u[y], u[y + 1], u[y + 2], u[y + 3]);
                        }
                    }
                }
                if (SPLIT) {
                    if (real) asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(share_ml + static_cast<uint32_t>(128 * t + r) * 8u), "f"(mc), "f"(l) : "memory");
                } else if (real && p.lse) p.lse[row] = none ? -INFINITY : (mc + log2f(l)) * 0.6931471805599453f;
            }
            tc_fence_before();
            if (SPLIT) {
                // ---- the cluster's shares of every row into one: rank r concludes every `split`-th row; four channels a thread
                arrive_at_all(B_SHARE_FULL);
                if (!wait_cluster(B_SHARE_FULL, it & 1)) { alive = false; break; }
                const int rows = few ? PA_FEW : plan.pair ? PA_ROWS : 2 * PA_ROWS;
                // (two quads a round, from two CTAs at a time: what comes from them takes about a microsecond)
                constexpr int AT_ONCE = 2;
                for (int x0 = tid; x0 < rows / split * 32; x0 += AT_ONCE * PA_SOFTMAX) {
                    float4 o[AT_ONCE];
                    float top[AT_ONCE], sum_of[AT_ONCE];
                    size_t row_of[AT_ONCE];
                    bool real_of[AT_ONCE];
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) {
                        const int x = x0 + u * PA_SOFTMAX, rr = (x >> 5) * split + rank, of = rr >> 7, in = rr & 127, to = in / p.G;
                        real_of[u] = x < rows / split * 32 && to < (of ? plan.n_b : plan.n_a);
                        row_of[u] = static_cast<size_t>(w.q0 + w.first + of * p.tq + to) * p.Hq + static_cast<size_t>(w.h) * p.G + (in - to * p.G);
                        o[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                        top[u] = PA_NO_MAX;
                        sum_of[u] = 0.f;
                    }
#pragma unroll 2
                    for (int k = 0; k < split; ++k) {
                        float2 ml[AT_ONCE];
                        float4 v[AT_ONCE];
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) {
                            const int x = x0 + u * PA_SOFTMAX, rr = (x >> 5) * split + rank;
                            if (!real_of[u]) continue;
                            ml[u] = ld_cluster2(map_shared_rank(share_ml + static_cast<uint32_t>(rr) * 8u, k));
                            v[u] = ld_cluster4(map_shared_rank(share + static_cast<uint32_t>(rr) * 512u + (((x & 31) ^ (rr & 31)) << 4), k));
                        }
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) {
                            if (!real_of[u]) continue;
                            const float most = fmaxf(top[u], ml[u].x), f = pa_ex2(ml[u].x - most), was = pa_ex2(top[u] - most);
                            sum_of[u] = sum_of[u] * was + ml[u].y * f;
                            o[u].x = o[u].x * was + v[u].x * f; o[u].y = o[u].y * was + v[u].y * f;
                            o[u].z = o[u].z * was + v[u].z * f; o[u].w = o[u].w * was + v[u].w * f;
                            top[u] = most;
                        }
                    }
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) {
                        if (!real_of[u]) continue;
                        const int quad = (x0 + u * PA_SOFTMAX) & 31;
                        const bool nothing = sum_of[u] == 0.f;
                        const float by = nothing ? 0.f : 1.f / sum_of[u];
                        *reinterpret_cast<uint2*>(static_cast<T*>(p.out) + row_of[u] * PI_HEAD_DIM + 4 * quad) =
                            nothing ? make_uint2(0u, 0u) : make_uint2(Form<T>::pack(o[u].x * by, o[u].y * by), Form<T>::pack(o[u].z * by, o[u].w * by));
                        if (p.lse && quad == 0) p.lse[row_of[u]] = nothing ? -INFINITY : (top[u] + log2f(sum_of[u])) * 0.6931471805599453f;
                    }
                }
                arrive_at_all(B_SHARE_EMPTY);
            }
            if (plan.pair) {                        // B's O may be written anew when A has read it
                __syncwarp();
                if (t == 0) {
                    if (lane == 0) mbar_arrive(bar(B_MERGED));
                } else if (!wait(B_MERGED, merges & 1u)) {
                    alive = false;
                    break;
                }
                ++merges;
            }
            done_with(it);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PA_OTHER_REGS));
        if (warp == 9) {
            // ---- TMA: Q, then K0 V0 K1 V1 ...
            uint32_t n = 0u, items = 0u;            // loads, and items with any, so far
            bool alive = true, q_issued = false, shares = false;     // shares: those of an earlier item lie where loads go
            Item w;
            for (int it = 0; alive && item_of(it, w); ++it) {
                const Plan plan(p, w, rank, split);
                done_with(it);
                const bool in_the_way = SPLIT && it > 0 && (shares || plan.n_b), few = plan.pair && plan.n_a * p.G <= PA_FEW;
                shares |= SPLIT && !few;
                if (plan.hi <= plan.lo) {
                    if (rank == 0 && lane == 0) mbar_arrive(bar(B_WANTED));
                    continue;
                }
                if (in_the_way) {
                    // The shares of the last item have to have been read, and with them all before it (an item is told when the cluster is done
                    // with the one before the last).  This phase and no other can be told by its parity: the one before it is over, and the next ends
                    // behind the loads that this warp is about to issue.
                    if (!wait_cluster(B_SHARE_EMPTY, (it - 1) & 1)) { alive = false; break; }
                    asm volatile("fence.proxy.async;" ::: "memory");
                    shares = !few;
                }
                if (items && !wait(B_Q_EMPTY, (items - 1) & 1u)) { alive = false; break; }
                if (lane == 0) {
                    const uint32_t bytes = static_cast<uint32_t>(p.tq) * p.G * 128u;
                    mbar_expect_tx(bar(B_Q_FULL), bytes * (plan.n_b ? 4u : 2u));
                    for (int t = 0; t < (plan.n_b ? 2 : 1); ++t)
                        for (int x = 0; x < 2; ++x) tma_load_q(smem + t * PA_TILE + x * PA_HALF, &map_q, bar(B_Q_FULL), 64 * x, 0, w.h, w.q0 + w.first + t * p.tq);
                }
                q_issued = true;
                ++items;
                for (int i = 2 * plan.lo; i < 2 * plan.hi; ++i, ++n) {
                    const uint32_t stage = n % PA_STAGES;
                    if (n >= PA_STAGES && !wait(B_KV_EMPTY + stage, (n / PA_STAGES - 1) & 1u)) { alive = false; break; }
                    if (p.hold_last && i == 2 * plan.hi - 1) { alive = false; break; }
                    if (lane == 0) {
                        const CUtensorMap* map = (i & 1) ? &map_v : &map_k;
                        mbar_expect_tx(bar(B_KV_FULL + stage), PA_TILE);
                        for (int x = 0; x < 2; ++x) tma_load_3d(ring + stage * PA_TILE + x * PA_HALF, map, bar(B_KV_FULL + stage), 64 * x, w.h, w.k0 + (i >> 1) * PA_ROWS);
                    }
                    __syncwarp();
                }
                // (what comes next is asked for when this item's loads have all been issued, and no sooner: until then others may come to it first)
                if (rank == 0 && lane == 0) mbar_arrive(bar(B_WANTED));
            }
            if (!alive || *abort) {                 // copies in flight end before the CTA does
                volatile int none = 0;
                if (q_issued) mbar_wait(bar(B_Q_FULL), (items - 1) & 1u, &none, p.wait_cycles);
                for (uint32_t i = n < PA_STAGES ? 0u : n - PA_STAGES; i < n; ++i) mbar_wait(bar(B_KV_FULL + i % PA_STAGES), (i / PA_STAGES) & 1u, &none, p.wait_cycles);
            }
        } else if (warp == 8) {
            // ---- the products.  One lane issues them, but everything they are made of is kept the same in all lanes, and plainly so (values from
            // lane 0, votes): their operands are uniform registers, and moving each of them there took longer than the products
            // themselves (8192 tokens 520 us instead of 433).
            constexpr uint32_t base = (1u << 4) | (Form<T>::code << 7) | (Form<T>::code << 10) | (static_cast<uint32_t>(PA_ROWS >> 3) << 17) | (static_cast<uint32_t>(PA_ROWS >> 4) << 24);
            constexpr uint32_t idesc_s = base, idesc_o = base | (1u << 16);      // V: channels run along its rows
            const uint32_t utmem = __shfl_sync(0xffffffffu, tmem, 0), usmem = __shfl_sync(0xffffffffu, smem, 0), uring = usmem + 2 * PA_TILE;
            // The pipe holds about two of them behind the one at work, 100 cycles or so, so whatever this warp does between two products
            // is seen unless it is short: one wait (60 cycles when what it waits for is there) between any two, stages counted and not
            // divided out (23 ragged prompts 180 us instead of 184, of 8192 tokens 2 % fewer cycles).
            const uint64_t desc_q = desc_k_major(usmem), desc_k = desc_k_major(uring), desc_v = desc_mn_major(uring);
            constexpr uint32_t tile_step = PA_TILE >> 4;
            uint32_t stage = 0u, filled = 0u, good = 0u;     // of the next load; bits: which phase of a stage's KV_FULL and V_GOOD comes next
            uint32_t items = 0u, made = 0u;                  // bit t of `made`: which phase of tile t's P_FULL comes next
            bool alive = true;
            Item w;
            auto after = [](uint32_t at) { return at == PA_STAGES - 1 ? 0u : at + 1; };
            auto full = [&](uint32_t at) {
                const uint32_t phase = (filled >> at) & 1u;
                filled ^= 1u << at;
                return wait(B_KV_FULL + at, phase);
            };
            // V of a tile that is looked through first waits for that
            auto full_v = [&](uint32_t at, bool odd) {
                if (!odd) return full(at);
                const uint32_t phase = (good >> at) & 1u;
                good ^= 1u << at;
                filled ^= 1u << at;
                return wait(B_V_GOOD + at, phase);
            };
            auto weights = [&](int t) {
                const uint32_t phase = (made >> t) & 1u;
                made ^= 1u << t;
                return wait(B_P_FULL + t, phase);
            };
            // (`half`: no row sees the upper 64 of a tile's keys, and they are left out of both products; the softmax masks what stands in their scores' place.
            // 16 prompts of 1 024 tokens 159 us instead of 162)
            auto product_s = [&](int t, uint32_t q_step, uint32_t at, bool half) {
                const uint64_t qa = desc_q + q_step, kb = desc_k + at * tile_step;
                const uint32_t idesc = half ? idesc_s - (static_cast<uint32_t>(PA_ROWS >> 4) << 17) : idesc_s;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint64_t step = static_cast<uint64_t>(((k >> 2) * PA_HALF + (k & 3) * 32) >> 4);
                        tc_mma_ss(utmem + PA_TMEM_S + 128 * t, qa + step, kb + step, idesc, k > 0);
                    }
                    tc_commit(bar(B_S_FULL + t));
                }
            };
            auto product_o = [&](int t, uint32_t at, bool add, bool half) {
                const uint64_t vb = desc_v + at * tile_step;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) tc_mma_ts(utmem + PA_TMEM_O + 128 * t, utmem + PA_TMEM_S + 128 * t + 8 * k, vb + static_cast<uint64_t>((k * 2048) >> 4), idesc_o, add || k > 0);
                    if (!half) {
#pragma unroll
                        for (int k = 4; k < 8; ++k) tc_mma_ts(utmem + PA_TMEM_O + 128 * t, utmem + PA_TMEM_S + 128 * t + 8 * k, vb + static_cast<uint64_t>((k * 2048) >> 4), idesc_o, true);
                    }
                }
            };
            auto signal = [&](uint32_t place) {
                if (elect_one()) tc_commit(bar(place));
            };
            for (int it = 0; alive && item_of(it, w); ++it) {
                w.q0 = __shfl_sync(0xffffffffu, w.q0, 0); w.n = __shfl_sync(0xffffffffu, w.n, 0);
                w.k0 = __shfl_sync(0xffffffffu, w.k0, 0); w.m = __shfl_sync(0xffffffffu, w.m, 0);
                w.first = __shfl_sync(0xffffffffu, w.first, 0); w.h = __shfl_sync(0xffffffffu, w.h, 0);
                const Plan plan(p, w, rank, split);
                done_with(it);
                if (plan.hi <= plan.lo) continue;
                if (!wait(B_Q_FULL, items++ & 1u) || !full(stage)) { alive = false; break; }
                tc_fence_after();
                const int count = plan.hi - plan.lo;
                auto half = [&](int t, int j) { return (t ? plan.last_b : plan.last_a) <= j * PA_ROWS + PA_ROWS / 2; };
                if (plan.pair) {
                    // one query tile: S of the first two K tiles, then V after V; a group's next K is two tiles on, and is waited for behind the product
                    // with V, which frees a place for the loads
                    product_s(0, 0u, stage, half(0, plan.lo));
                    signal(B_KV_EMPTY + stage);
                    uint32_t sv = after(stage), sk = after(sv);
                    if (count > 1) {
                        if (!full(sk)) { alive = false; break; }
                        tc_fence_after();
                        product_s(1, 0u, sk, half(1, plan.lo + 1));
                        signal(B_KV_EMPTY + sk);
                    }
                    if (count <= 2) signal(B_Q_EMPTY);
                    for (int x = 0; x < count; ++x) {
                        const int t = x & 1;
                        const bool next = x + 2 < count;
                        sk = after(after(after(sv)));
                        alive = full_v(sv, plan.lo + x >= plan.odd_from) && weights(t);
                        if (!alive) break;
                        tc_fence_after();
                        product_o(t, sv, x >= 2, half(t, plan.lo + x));
                        signal(B_KV_EMPTY + sv);
                        if (next) {
                            alive = full(sk);
                            if (!alive) break;
                            tc_fence_after();
                            product_s(t, 0u, sk, half(t, plan.lo + x + 2));
                            signal(B_KV_EMPTY + sk);
                            if (x + 3 == count) signal(B_Q_EMPTY);
                        } else signal(B_O_FULL + t);
                        if (x + 1 < count) sv = after(after(sv));
                    }
                    stage = after(sv);
                } else {
                    const bool a_some = plan.lo < plan.tiles_a;
                    if (a_some) product_s(0, 0u, stage, half(0, plan.lo));
                    product_s(1, tile_step, stage, half(1, plan.lo));          // (tile B sees as many tiles as the item has)
                    signal(B_KV_EMPTY + stage);
                    if (count == 1) signal(B_Q_EMPTY);
                    uint32_t sv = after(stage);
                    alive = full_v(sv, plan.lo >= plan.odd_from);
                    for (int x = 0; x < count && alive; ++x) {
                        const int j = plan.lo + x;
                        const uint32_t sk = after(sv), sv_next = after(sk);
                        const bool next = x + 1 < count;
                        if (j < plan.tiles_a) {
                            if (!weights(0)) { alive = false; break; }
                            tc_fence_after();
                            product_o(0, sv, x > 0, half(0, j));
                        }
                        if (next && !full(sk)) { alive = false; break; }
                        if (j < plan.tiles_a) {
                            if (j + 1 < plan.tiles_a) {
                                tc_fence_after();
                                product_s(0, 0u, sk, half(0, j + 1));
                            } else signal(B_O_FULL);
                        }
                        if (!weights(1)) { alive = false; break; }
                        tc_fence_after();
                        product_o(1, sv, x > 0, half(1, j));
                        signal(B_KV_EMPTY + sv);
                        if (next) {
                            alive = full_v(sv_next, j + 1 >= plan.odd_from);
                            if (!alive) break;
                            tc_fence_after();
                            product_s(1, tile_step, sk, half(1, j + 1));
                            signal(B_KV_EMPTY + sk);
                            if (x + 2 == count) signal(B_Q_EMPTY);
                        } else signal(B_O_FULL + 1);
                        if (next) sv = sv_next;
                    }
                    stage = after(sv);
                }
            }
            // products in flight end before the CTA does
            volatile int none = 0;
            if (elect_one()) tc_commit(bar(B_DRAINED));
            mbar_wait(bar(B_DRAINED), 0, &none, p.wait_cycles);
            __syncwarp();
        } else if (warp == 11) {
            // ---- a V tile that some row must not see all of is looked through: rows behind the sequence's end become 0, and so does every
            // value that is no number (its weight would be 0 where it is masked, and 0 times it is none); those are put back at the
            // end, row by row.  A stage is given back by this warp as well as by the products, whether it is looked through or not: the phases
            // of its loads are told by parity, and none may go by meanwhile.
            uint32_t n = 0u;
            bool alive = true;
            Item w;
            for (int it = 0; alive && item_of(it, w); ++it) {
                const Plan plan(p, w, rank, split);
                bool odd = false;
                for (int i = 2 * plan.lo; i < 2 * plan.hi; ++i, ++n) {
                    const uint32_t stage = n % PA_STAGES, tile = ring + stage * PA_TILE;
                    if (!wait(B_KV_FULL + stage, (n / PA_STAGES) & 1u)) { alive = false; break; }
                    const int j = i >> 1;
                    if (!(i & 1) || j < plan.odd_from) {
                        if (lane == 0) mbar_arrive(bar(B_KV_EMPTY + stage));
                        continue;
                    }
                    const int rows = min(w.m - j * PA_ROWS, PA_ROWS), from = max(plan.seen_first - j * PA_ROWS, 0);      // of the sequence; not seen by all
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t at = tile + half * PA_HALF + lane * 16;
#pragma unroll 4
                        for (int x = rows * 128; x < PA_HALF; x += 512)
                            if (x + lane * 16 < PA_HALF) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(at + x), "r"(0u) : "memory");
                        for (int x0 = from * 128; x0 < rows * 128; x0 += 8 * 512) {
                            uint32_t u[8][4], most = 0u;     // the largest magnitudes
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const int x = x0 + 512 * k;
                                if (x + lane * 16 < rows * 128) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u[k][0]), "=r"(u[k][1]), "=r"(u[k][2]), "=r"(u[k][3]) : "r"(at + x));
                                else u[k][0] = u[k][1] = u[k][2] = u[k][3] = 0u;
                            }
#pragma unroll
                            for (int k = 0; k < 8; ++k)
#pragma unroll
                                for (int y = 0; y < 4; ++y) most = Form<T>::larger(most, u[k][y]);
                            if (!not_finite<T>(most)) continue;
                            odd = true;
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                if (x0 + 512 * k + lane * 16 >= rows * 128) continue;
#pragma unroll
                                for (int y = 0; y < 4; ++y) u[k][y] &= ~((not_finite<T>(u[k][y]) >> 15) * 0xffffu);
                                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at + x0 + 512 * k), "r"(u[k][0]), "r"(u[k][1]), "r"(u[k][2]), "r"(u[k][3]) : "memory");
                            }
                        }
                    }
                    if (odd) s_odd[it & 1] = 1;
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(bar(B_V_GOOD + stage));
                        mbar_arrive(bar(B_KV_EMPTY + stage));
                    }
                }
                done_with(it);
            }
        } else if (rank == 0) {
            // ---- warp 10: which items are this CTA's, or its cluster's.  Blocks are counted from the last one of the last sequence, so that the longest of a
            // sequence come first; KV heads innermost.  32 sequences at a time are put in the order of their keys, so that the longest of them come first
            // too, and what is short fills the end.
            const int per_block = p.per_block;
            // (quotients by multiplication: a lone warp takes 200 cycles for a division, and the first item waits for five of them)
            auto blocks_of = [&](int n) {
                const unsigned x = static_cast<unsigned>(n + per_block - 1), q = __umulhi(x, p.by_block);
                return static_cast<int>(q - (q * per_block > x));
            };
            auto spans_from = [&](int s0, bool tell) {
                Span x = span_of(p, s0 + lane, tell);
                const int count = min(p.n_seqs - s0, 32);
                if (count > 1) {
                    const int key = x.n > 0 ? x.m : -1;
                    int before = 0;
#pragma unroll 8
                    for (int k = 0; k < count; ++k) {
                        const int other = __shfl_sync(0xffffffffu, key, k);
                        before += other < key || (other == key && k < lane);
                    }
                    if (lane < count) s_order[before] = static_cast<unsigned char>(lane);
                    __syncwarp();
                    const int from = lane < count ? s_order[lane] : lane;
                    __syncwarp();
                    x.q0 = __shfl_sync(0xffffffffu, x.q0, from); x.n = __shfl_sync(0xffffffffu, x.n, from);
                    x.k0 = __shfl_sync(0xffffffffu, x.k0, from); x.m = __shfl_sync(0xffffffffu, x.m, from);
                }
                return x;
            };
            // `group`: 32 sequences, from number group_at on.  Where there are more, every group's blocks are counted once (lane l: groups l, 32 + l, ...), and
            // an item finds its group among the sums: looking through all sequences for every item, 32 single tokens after 8 000 keys took 753 us behind
            // 2 016 empty sequences, now 189 (alone 180), 4 096 tokens over 64 keys each 28.8 ms, now 1.01.
            const bool tell = blockIdx.x == 0;
            int group_at = 0, upto_group[GROUPS], total = 0;
            Span group = {0, 0, 0, 0};
            if (p.n_seqs <= 32) {
                group = spans_from(0, tell);
                total = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(blocks_of(group.n))));
            } else {
                group_at = -1;
                // (eight groups' bounds on their way at a time)
#pragma unroll 1
                for (int s0 = 0; s0 < p.n_seqs; s0 += 256) {
                    Span x[8];
#pragma unroll
                    for (int g = 0; g < 8; ++g) x[g] = span_of(p, s0 + 32 * g + lane, false);
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const int at = s0 + 32 * g;
                        total += static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(blocks_of(x[g].n))));
#pragma unroll
                        for (int i = 0; i < GROUPS; ++i)
                            if (at >> 5 == 32 * i + lane) upto_group[i] = total;
                    }
                }
                for (int s = lane; tell && s < p.n_seqs; s += 32) (void)span_of(p, s, true);
                __syncwarp();
                // (lanes behind the last group: more than any place)
#pragma unroll
                for (int i = 0; i < GROUPS; ++i)
                    if (32 * (32 * i + lane) >= p.n_seqs) upto_group[i] = total;
            }
            unsigned place = blockIdx.x / static_cast<unsigned>(split);      // (of a cluster: its first CTA's)
            uint32_t asked = 0u;
            bool more = true;
            // This warp's waits last as long as an item does, so their limit grows with the longest item told so far: 2^15 cycles a K/V tile, ten times what one takes.
            long long patience = p.wait_cycles;
            auto wait_item = [&](uint32_t place, uint32_t parity) {
                return __all_sync(0xffffffffu, SPLIT ? mbar_wait_cluster(bar(place), parity, abort, patience) : mbar_wait(bar(place), parity, abort, patience)) != 0;
            };
            for (int it = 0;; ++it) {
                Item w = {0, 0, 0, 0, 0, -1};
                const int item = static_cast<int>(place >> p.log_hkv);
                const bool has = more && item < total;
                if (has) {
                    int at = total - 1 - item;
                    if (p.n_seqs > 32) {
                        int s0 = 0, before = 0;
#pragma unroll
                        for (int i = GROUPS - 1; i >= 0; --i) {
                            if (1024 * i >= p.n_seqs) continue;
                            const unsigned found = __ballot_sync(0xffffffffu, at < upto_group[i]);
                            if (!found) break;
                            const int from = __ffs(static_cast<int>(found)) - 1;
                            s0 = 1024 * i + 32 * from;
                            before = from ? __shfl_sync(0xffffffffu, upto_group[i], from - 1) : i ? __shfl_sync(0xffffffffu, upto_group[i - 1], 31) : 0;
                        }
                        at -= before;
                        if (s0 != group_at) group = spans_from(s0, false);
                        group_at = s0;
                    }
                    const int nb = blocks_of(group.n);
                    int upto = nb;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        const int y = __shfl_up_sync(0xffffffffu, upto, d);
                        if (lane >= d) upto += y;
                    }
                    const unsigned found = __ballot_sync(0xffffffffu, at < upto);
                    if (found) {
                        const int from = __ffs(static_cast<int>(found)) - 1;
                        w.first = (at - __shfl_sync(0xffffffffu, upto - nb, from)) * per_block;
                        w.q0 = __shfl_sync(0xffffffffu, group.q0, from); w.n = __shfl_sync(0xffffffffu, group.n, from);
                        w.k0 = __shfl_sync(0xffffffffu, group.k0, from); w.m = __shfl_sync(0xffffffffu, group.m, from);
                        w.h = static_cast<int>(place) & (p.Hkv - 1);
                    }
                }
                if (it >= 2 && !wait_item(B_ITEM_EMPTY + (it & 1), ((it >> 1) - 1) & 1)) break;
                patience = max(patience, p.wait_cycles + (static_cast<long long>(w.m / PA_ROWS + 1) << 15));
                if (SPLIT) {                        // lane k tells rank k
                    if (lane < split) {
                        const uint32_t at = map_shared_rank(smem_u32(&s_item[it & 1]), lane), odd = map_shared_rank(smem_u32(&s_odd[it & 1]), lane);
                        const int v[6] = {w.q0, w.n, w.k0, w.m, w.first, w.h};
#pragma unroll
                        for (int k = 0; k < 6; ++k) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at + 4 * k), "r"(v[k]) : "memory");
                        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(odd), "r"(0) : "memory");
                        mbar_arrive_cluster(map_shared_rank(bar(B_ITEM_FULL + (it & 1)), lane));
                    }
                } else if (lane == 0) {
                    s_item[it & 1] = w;
                    s_odd[it & 1] = 0;
                    mbar_arrive(bar(B_ITEM_FULL + (it & 1)));
                }
                __syncwarp();
                if (!has) break;
                if (!wait_item(B_WANTED, it & 1)) break;
                // a CTA that has not begun gives its place up, if there is one (a place behind the last item too, and then the next)
                uint32_t got = 0u;
                do {
                    if (lane == 0) {
                        mbar_expect_tx(bar(B_NEXT), 16);
                        asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(s_next)), "r"(bar(B_NEXT)) : "memory");
                    }
                    __syncwarp();
                    volatile int none = 0;          // (the answer is written into this CTA's memory, so it is waited for in any case)
                    if (!__all_sync(0xffffffffu, mbar_wait(bar(B_NEXT), asked++ & 1u, &none, p.wait_cycles))) { *abort = 1; got = 0u; break; }
                    asm volatile(
                        "{\n .reg .b128 r;\n .reg .pred c;\n ld.shared.b128 r, [%2];\n clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 c, r;\n selp.u32 %0, 1, 0, c;\n mov.u32 %1, 0;\n"
                        " @c clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n}"
                        : "=r"(got), "=r"(place) : "r"(smem_u32(s_next)) : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (read before the next answer is written)
                    __syncwarp();
                    place /= static_cast<unsigned>(split);
                } while (got && static_cast<int>(place >> p.log_hkv) >= total);
                more = got != 0u;
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (SPLIT) cluster_sync_all();                  // no CTA ends while another reads its share or arrives at its barriers
    if (warp == 8) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
    if (tid == 0 && s_abort) pi_report(p.st, PI_ERR_TIMEOUT, PI_STAGE_PROMPT, static_cast<int>(blockIdx.x), s_item[0].first, s_item[0].h);
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
    PromptParams p = {};
    p.q_start = q_start; p.k_start = k_start;
    p.out = out; p.lse = lse; p.v = v; p.v_tok = v_tok; p.v_head = v_head;
    p.st = pi_status_of(c);
    p.wait_cycles = c->wait_limit_cycles;
    p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(PI_HEAD_DIM));
    p.n_seqs = n_seqs; p.Hq = cfg.n_q_heads; p.Hkv = cfg.n_kv_heads; p.G = cfg.n_q_heads / cfg.n_kv_heads; p.n_q = n_q; p.n_k = n_k;
    p.tq = PA_ROWS / p.G;
    while ((1 << p.log_hkv) < p.Hkv) ++p.log_hkv;  // (a power of two: pi_create)
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
    p.hold_last = cfg.test_hold_producer;
    p.wide = (reinterpret_cast<uintptr_t>(out) & 31u) == 0;
    const long long seqs = n_seqs < n_q ? n_seqs : n_q;
    auto items_of = [&](int block) { return (n_q + seqs * (block - 1)) / block * p.Hkv; };
    // Items of one query tile where each has an SM to itself: the two groups then share its K/V tiles.  77 tokens 7.2 us instead of 8.1, 512 11.1
    // instead of 13.6, 100 after 4 000 20.7 instead of 29.7, 6 of 1 to 90 after 0 to 1 000 15.6 instead of 22.3.
    p.per_block = items_of(p.tq) <= c->n_sms ? p.tq : 2 * p.tq;
    p.by_block = 0xffffffffu / static_cast<uint32_t>(p.per_block) + 1;
    const long long items = items_of(p.per_block);
    const size_t smem = 2 * PA_TILE + PA_STAGES * PA_TILE + 1024;
    cudaLaunchConfig_t lc = {};
    lc.blockDim = dim3(PA_THREADS);
    lc.dynamicSmemBytes = smem;
    lc.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    // how many clusters of 2^power CTAs are resident at a time, asked once
    auto resident = [&](int power) {
        int& n = c->pa_resident_clusters[power];
        if (n < 0) {
            auto kernel = prompt_attn_kernel<__nv_bfloat16, true>;
            cudaLaunchConfig_t one = lc;
            attr[0].val.clusterDim.x = 1 << power;
            one.gridDim = dim3(1 << power);
            one.stream = nullptr;
            one.attrs = attr;
            one.numAttrs = 1;
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess ||
                cudaOccupancyMaxActiveClusters(&n, kernel, &one) != cudaSuccess) {
                (void)cudaGetLastError();
                n = 0;
            }
        }
        return n;
    };
    // CTAs that share an item: where the items leave SMs without work and the keys are many, a cluster for each, of a power of two of CTAs up to
    // eight, as long as all clusters are resident at once (16 of eight are not: 2 of 20 tokens after 8 000 37.9 us instead of 28.1 with four; of clusters
    // of 16 fewer than eight are).  A cluster costs 2 to 4 us more than a CTA, and a K/V tile 1 us: 8 items of one token and 4 / 8 / 32 / 128 tiles take
    // 10.2 / 13.4 / 33 / 120 us with 1 CTA each, 12.5 / 14.1 / 24 / 68 with 2, 11.4 / 12.4 / 18 / 40 with 4, 12.6 / 12.6 / 16 / 28 with 8.
    const long long tiles = (n_k / seqs + PA_ROWS - 1) / PA_ROWS;
    int split = 1;
    for (int power = 1; power <= 3 && tiles >= 4 * split && tiles >= 8 && items <= resident(power); ++power) split *= 2;
    // How long each sequence is, only the kernel sees; the rule goes by the mean.  Where several of them make up to two items an SM and keep it busy
    // for a while, one that is longer than the others would be what the call waits for, so there two CTAs share each item.  Sequences of
    // like length lose less by it than the others gain: 16 of one token after 16 384 take 175 us instead of 166, after 0 to 16 384
    // 89 instead of 132; 12 of 4 after 16 000 159 instead of 142, after 0 to 16 000 81 instead of 127; 8 of 200 after 8 000 262 instead of 266, of 1 to 200
    // after 0 to 8 000 87 instead of 143; of the others only 32 of one token after 0 to 8 192 loses, 107 instead of 95.  With fewer keys it does
    // not pay: 16 of one token after 4 096 57 instead of 46, 6 of 100 after 3 000 75 instead of 53 (of 1 to 100 after 0 to 3 000 41 instead of 50).
    if (split == 1 && seqs > 1 && items <= 2 * c->n_sms && tiles > 32) split = 2;
    const long long grid = items * split;
    if (grid > INT32_MAX) return PI_ERR_UNSUPPORTED_DIM;
    lc.gridDim = dim3(static_cast<unsigned>(grid));
    attr[0].val.clusterDim.x = split;
    lc.attrs = split > 1 ? attr : attr + 1;
    lc.numAttrs = split > 1 ? 2 : 1;
    auto launch = [&](auto kernel) -> int {
        PI_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
        PI_CUDA_TRY(cudaLaunchKernelEx(&lc, kernel, map_q, map_k, map_v, p));
        return PI_OK;
    };
    if (dtype == PI_DTYPE_BF16) return split > 1 ? launch(prompt_attn_kernel<__nv_bfloat16, true>) : launch(prompt_attn_kernel<__nv_bfloat16, false>);
    return split > 1 ? launch(prompt_attn_kernel<__half, true>) : launch(prompt_attn_kernel<__half, false>);
}
