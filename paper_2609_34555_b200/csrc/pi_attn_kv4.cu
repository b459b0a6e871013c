// Sparse GQA decode attention over a pool of 4-bit blocks:  softmax(q K^T / sqrt(D)) V  over the tokens of the selected
// blocks, K and V = scale * code + minimum (pi_kv4.cuh).
//
// 160 bytes a (token, KV head) for 4 G D operations: the pool's bytes are what the call cannot do without.  On the way
// to them stands the arithmetic of taking the codes apart, so that is kept out of the wide loops:
//   * a code becomes a bf16 number by two logical operations per PAIR: 0x4300 | code is 128 + code exactly, and the
//     format's nibble order makes (word >> 4 n) & 0x000f000f a pair that the matrix instruction takes as it is;
//   * scales and minima never meet the codes.  For K they are applied to the products: with the channels of a group
//     contracted by themselves,  q.k = sum over groups  scale * (q . code) + minimum * (sum of q),  two fused
//     multiply-adds per (token, head, group) instead of one per channel.  For V they are applied to the weights:
//     the contraction over tokens takes p * scale, one set per group, and the minima's part is a separate sum of
//     p * minimum per (head, group).
// The contractions run on mma.sync (tokens or channels on M, up to 8 query heads on N): with G <= 16 query heads per
// KV head a 128-row tcgen05 tile would be nearly empty, and the codes have to pass through registers anyway.
// q and the codes are exact in bf16; p * scale is split into a bf16 head and a bf16 remainder (2^-17 together), so
// that the weights add nothing to the one rounding of the output.  With G <= 4 the two halves of N carry the head and
// the remainder, and the split costs no second instruction.
//
// One (sequence, KV head) per cluster of S CTAs of 8 warps (S = 1, 2, 4 or 8 by the launcher's rule).  The item's
// 16-token tiles are dealt out to its warps in turn; a warp streams its own tiles through its own ring of shared-memory
// stages with 16-byte asynchronous copies (a tile is 2560 contiguous bytes), so no warp waits for another until the
// end.  Every warp keeps its own running maximum and sum; the states are merged once, through shared memory, and
// across the cluster through distributed shared memory: one launch, no partials in global memory.
#include "pi_attn_core.cuh"
#include "pi_kv4.cuh"

namespace {

using namespace pi_attn;

constexpr int A4_WARPS = 8;
constexpr int A4_THREADS = A4_WARPS * 32;
constexpr int A4_STAGES = 4;

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
// Pair n of a word: nibbles n (low half) and n + 4 (high half), each as the bf16 number 128 + nibble.
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int n) { return ((w >> (4 * n)) & 0x000f000fu) | 0x43004300u; }
// 128 + code -> code - 8, exactly.
__device__ __forceinline__ uint32_t less_136(uint32_t x) {
    const __nv_bfloat162 c = __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308));
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), c);
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t word_of(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// NT: tiles of 8 query heads; DUP (G <= 4): columns 4..7 repeat heads 0..3 and carry the weights' remainders.
template <int NT, bool DUP>
__global__ void __launch_bounds__(A4_THREADS, NT == 1 ? 2 : 1)
attn_kv4_kernel(Attn4Params p) {
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;
    const int S = static_cast<int>(cluster_nctarank()), rank = static_cast<int>(cluster_ctarank());
    const int item = blockIdx.x / S, seq = item / p.Hkv, h = item - seq * p.Hkv;
    const int SUB = p.B >> 4;
    pi_grid_dependency_wait();
    pi_launch_dependents();

    const int ctx = p.ctx_len[seq];
    int cnt = p.sel_count[seq];
    if (cnt < 0 || cnt > p.K) {
        if (h == 0 && rank == 0 && tid == 0) pi_report(p.st, PI_ERR_CAPACITY, PI_STAGE_ATTN, seq, cnt, p.K);
        cnt = 0;
    }
    const int n_tiles = cnt * SUB;
    const int first = rank * A4_WARPS + warp, stride = A4_WARPS * S;
    const int n_mine = first < n_tiles ? (n_tiles - first + stride - 1) / stride : 0;

    // {slot, sub-tile << 16, valid tokens << 20} of the warp's n-th tile (one per lane, 32 at a time)
    auto meta_of = [&](int n) -> uint32_t {
        if (n >= n_mine) return 0u;
        const int t = first + n * stride, j = t / SUB, sub = t - j * SUB;
        const int slot = p.sel_slots[static_cast<size_t>(seq) * p.K + j], blk = p.sel_blocks[static_cast<size_t>(seq) * p.K + j];
        if (blk < 0) return 0u;
        if (slot < 0 || slot >= p.C) {
            if (h == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_ATTN, seq, j, slot);
            return 0u;
        }
        const long long left = static_cast<long long>(ctx) - (static_cast<long long>(blk) * p.B + sub * 16);
        const int nvalid = left < 0 ? 0 : left > 16 ? 16 : static_cast<int>(left);
        return static_cast<uint32_t>(slot) | (static_cast<uint32_t>(sub) << 16) | (static_cast<uint32_t>(nvalid) << 20);
    };
    uint32_t meta = meta_of(lane), meta_next = 0u;

    const unsigned char* head_base = p.pool + static_cast<long long>(seq) * p.C * p.block_bytes + static_cast<long long>(h) * SUB * KV4_TILE_BYTES;
    const uint32_t ring = smem_u32(smem) + warp * (A4_STAGES * KV4_TILE_BYTES);
    const unsigned long long policy = pi_l2_stream_policy();
    auto issue = [&](int n, uint32_t md) {             // tile n into its stage; one commit per tile, also for what is skipped
        if (n < n_mine && (md >> 20)) {
            const unsigned char* src = head_base + static_cast<long long>(md & 0xffffu) * p.block_bytes + ((md >> 16) & 15u) * KV4_TILE_BYTES + lane * 16;
            const uint32_t dst = ring + (n % A4_STAGES) * KV4_TILE_BYTES + lane * 16;
#pragma unroll
            for (int i = 0; i < KV4_TILE_BYTES / 512; ++i) copy16(dst + i * 512, src + i * 512, policy);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int n = 0; n < A4_STAGES - 1; ++n) issue(n, __shfl_sync(0xffffffffu, meta, n));

    // ---- the queries as B operands, in the channel order of the K codes, and their sums over each group of channels
    uint32_t bq[NT][4][2][2];
    float qs[NT][4][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int g = DUP ? (r & 3) : nt * 8 + r;
        const bool real = g < p.G;
        const __nv_bfloat16* qg = p.q + (static_cast<size_t>(seq) * p.Hq + static_cast<size_t>(h) * p.G + (real ? g : 0)) * PI_HEAD_DIM;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 x = real ? __ldg(reinterpret_cast<const uint4*>(qg + 32 * j + 8 * c)) : make_uint4(0, 0, 0, 0);
            // pair n = channels (n, n + 4) of the eight
            bq[nt][j][0][0] = __byte_perm(x.x, x.z, 0x5410);
            bq[nt][j][0][1] = __byte_perm(x.x, x.z, 0x7632);
            bq[nt][j][1][0] = __byte_perm(x.y, x.w, 0x5410);
            bq[nt][j][1][1] = __byte_perm(x.y, x.w, 0x7632);
            float s[4] = {0.f, 0.f, 0.f, 0.f};
            const uint32_t ones[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
            mma_bf16(s, ones, bq[nt][j][0][0], bq[nt][j][0][1]);
            mma_bf16(s, ones, bq[nt][j][1][0], bq[nt][j][1][1]);
            qs[nt][j][0] = s[0];
            qs[nt][j][1] = s[1];
        }
    }

    // ---- running state: o[j][mt] = channels 32 j + 4 r + 2 mt (+ 1 in the upper two) of heads 2 c, 2 c + 1; zo: the
    // minima's share of group j for this lane's tokens; m, l as usual (exp2 domain)
    float o[NT][4][2][4], zo[NT][4][2], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = -INFINITY;
        l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            zo[nt][j][0] = zo[nt][j][1] = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][j][0][e] = o[nt][j][1][e] = 0.f;
        }
    }
    // Row r of a tile's products is token pr (row r + 8: pr + 8): then the four tokens that a lane needs of V, rows 2 c,
    // 2 c + 1, 2 c + 8, 2 c + 9, are c, c + 4, c + 8, c + 12, and the lanes of one load read neighbouring rows.
    const int pr = (r >> 1) + 4 * (r & 1);

    for (int n = 0; n < n_mine; ++n) {
        if ((n & 31) == 0) {
            if (n) meta = meta_next;
            meta_next = meta_of(n + 32 + lane);
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(A4_STAGES - 2) : "memory");
        __syncwarp();                                   // the stage is filled by all lanes, and the previous one read by all
        {
            const int nn = n + A4_STAGES - 1;
            // (meta_next is not touched before it is needed: its loads have 29 tiles' time to arrive)
            issue(nn, (nn >> 5) == (n >> 5) ? __shfl_sync(0xffffffffu, meta, nn & 31) : __shfl_sync(0xffffffffu, meta_next, nn & 31));
        }
        const int nvalid = static_cast<int>(__shfl_sync(0xffffffffu, meta, n & 31) >> 20);
        if (nvalid == 0) continue;
        const uint32_t tile = ring + (n % A4_STAGES) * KV4_TILE_BYTES;
        // ---- S^T = K q^T, group by group
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
        {
            const uint4 ka = lds128(tile + pr * 64 + c * 16), kb = lds128(tile + (pr + 8) * 64 + c * 16);
            const uint4 za = lds128(tile + KV4_K_SCALES + pr * 16), zb = lds128(tile + KV4_K_SCALES + (pr + 8) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t wa = word_of(ka, j), wb = word_of(kb, j);
                const uint32_t a0[4] = {code_pair(wa, 0), code_pair(wb, 0), code_pair(wa, 1), code_pair(wb, 1)};
                const uint32_t a1[4] = {code_pair(wa, 2), code_pair(wb, 2), code_pair(wa, 3), code_pair(wb, 3)};
                const float sa = kv4_scale_of(word_of(za, j)), sb = kv4_scale_of(word_of(zb, j));
                // the products hold 128 q beside code q: taken off with the minimum
                const float ma = fmaf(-128.f, sa, kv4_min_of(word_of(za, j))), mb = fmaf(-128.f, sb, kv4_min_of(word_of(zb, j)));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float x[4] = {0.f, 0.f, 0.f, 0.f};
                    mma_bf16(x, a0, bq[nt][j][0][0], bq[nt][j][0][1]);
                    mma_bf16(x, a1, bq[nt][j][1][0], bq[nt][j][1][1]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        s[nt][e] = fmaf(sa, x[e], fmaf(ma, qs[nt][j][e], s[nt][e]));
                        s[nt][2 + e] = fmaf(sb, x[2 + e], fmaf(mb, qs[nt][j][e], s[nt][2 + e]));
                    }
                }
            }
        }
        // ---- online softmax over the tile's tokens
        float w[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float s0 = pr < nvalid ? s[nt][e] * p.scale_log2 : -INFINITY;
                const float s1 = pr + 8 < nvalid ? s[nt][2 + e] * p.scale_log2 : -INFINITY;
                float mx = fmaxf(s0, s1);
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                const float m_new = fmaxf(m[nt][e], mx);
                float alpha = 1.f, p0 = 0.f, p1 = 0.f;
                if (m_new != -INFINITY) {
                    alpha = exp2f(m[nt][e] - m_new);
                    p0 = exp2f(s0 - m_new);
                    p1 = exp2f(s1 - m_new);
                }
                m[nt][e] = m_new;
                l[nt][e] = l[nt][e] * alpha + p0 + p1;
                w[nt][e] = p0; w[nt][2 + e] = p1;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    zo[nt][j][e] *= alpha;
                    o[nt][j][0][e] *= alpha; o[nt][j][0][2 + e] *= alpha;
                    o[nt][j][1][e] *= alpha; o[nt][j][1][2 + e] *= alpha;
                }
            }
        // ---- O^T += V^T (p scale), group by group
        uint4 va = lds128(tile + KV4_V_SCALES + pr * 16), vb = lds128(tile + KV4_V_SCALES + (pr + 8) * 16);
        if (nvalid < 16) {                              // what lies behind the last token may be anything, NaN among it
            if (pr >= nvalid) va = make_uint4(0, 0, 0, 0);
            if (pr + 8 >= nvalid) vb = make_uint4(0, 0, 0, 0);
        }
        uint2 x[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) x[a] = lds64(tile + KV4_V_CODES + (4 * a + c) * 64 + r * 8);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned sel = (j & 1) ? 0x7632u : 0x5410u;
            const uint32_t y01 = __byte_perm(j < 2 ? x[0].x : x[0].y, j < 2 ? x[1].x : x[1].y, sel);
            const uint32_t y23 = __byte_perm(j < 2 ? x[2].x : x[2].y, j < 2 ? x[3].x : x[3].y, sel);
            const uint32_t a0[4] = {less_136(code_pair(y01, 0)), less_136(code_pair(y01, 1)), less_136(code_pair(y23, 0)), less_136(code_pair(y23, 1))};
            const uint32_t a1[4] = {less_136(code_pair(y01, 2)), less_136(code_pair(y01, 3)), less_136(code_pair(y23, 2)), less_136(code_pair(y23, 3))};
            const float sa = kv4_scale_of(word_of(va, j)), sb = kv4_scale_of(word_of(vb, j));
            const float ma = fmaf(8.f, sa, kv4_min_of(word_of(va, j))), mb = fmaf(8.f, sb, kv4_min_of(word_of(vb, j)));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                zo[nt][j][0] = fmaf(w[nt][0], ma, fmaf(w[nt][2], mb, zo[nt][j][0]));
                zo[nt][j][1] = fmaf(w[nt][1], ma, fmaf(w[nt][3], mb, zo[nt][j][1]));
                const float p0 = w[nt][0] * sa, p1 = w[nt][1] * sa, p2 = w[nt][2] * sb, p3 = w[nt][3] * sb;
                uint32_t h01 = pack_bf16(p0, p1), h23 = pack_bf16(p2, p3);
                const float2 f01 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&h01));
                const float2 f23 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&h23));
                const uint32_t r01 = pack_bf16(p0 - f01.x, p1 - f01.y), r23 = pack_bf16(p2 - f23.x, p3 - f23.y);
                if (DUP) {
                    if (c >= 2) { h01 = r01; h23 = r23; }
                    const uint32_t b0 = movm_t(h01), b1 = movm_t(h23);
                    mma_bf16(o[nt][j][0], a0, b0, b1);
                    mma_bf16(o[nt][j][1], a1, b0, b1);
                } else {
                    const uint32_t b0 = movm_t(h01), b1 = movm_t(h23), d0 = movm_t(r01), d1 = movm_t(r23);
                    mma_bf16(o[nt][j][0], a0, b0, b1);
                    mma_bf16(o[nt][j][1], a1, b0, b1);
                    mma_bf16(o[nt][j][0], a0, d0, d1);
                    mma_bf16(o[nt][j][1], a1, d0, d1);
                }
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");

    // ---- the warp's state into shared memory: o [warp][G][128], then m and l [warp][G] (the ring is done with)
    __syncthreads();
    float* s_o = reinterpret_cast<float*>(smem);
    float* s_m = s_o + A4_WARPS * p.G * PI_HEAD_DIM;
    float* s_l = s_m + A4_WARPS * p.G;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float sum = l[nt][e];
#pragma unroll
            for (int d = 4; d <= 16; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            float z[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                z[j] = zo[nt][j][e];
#pragma unroll
                for (int d = 4; d <= 16; d <<= 1) z[j] += __shfl_xor_sync(0xffffffffu, z[j], d);
            }
            const int g = nt * 8 + 2 * c + e;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float4 v = make_float4(o[nt][j][0][e], o[nt][j][0][2 + e], o[nt][j][1][e], o[nt][j][1][2 + e]);
                if (DUP) {                              // the remainders' columns belong to the head four columns before
                    v.x += __shfl_xor_sync(0xffffffffu, v.x, 2); v.y += __shfl_xor_sync(0xffffffffu, v.y, 2);
                    v.z += __shfl_xor_sync(0xffffffffu, v.z, 2); v.w += __shfl_xor_sync(0xffffffffu, v.w, 2);
                }
                v.x += z[j]; v.y += z[j]; v.z += z[j]; v.w += z[j];
                if (g < p.G && (!DUP || c < 2)) *reinterpret_cast<float4*>(s_o + (warp * p.G + g) * PI_HEAD_DIM + 32 * j + 4 * r) = v;
            }
            if (g < p.G && (!DUP || c < 2) && r == 0) { s_m[warp * p.G + g] = m[nt][e]; s_l[warp * p.G + g] = sum; }
        }
    __syncthreads();

    // ---- the eight warps' states into one: s_o [0][G][128] of this CTA, s_m / s_l [0][G]
    const int n_out = p.G * PI_HEAD_DIM;
    auto write_out = [&](int i, float M, float L, float v) {
        const int g = i >> 7, d = i & 127;
        const size_t row = static_cast<size_t>(seq) * p.Hq + static_cast<size_t>(h) * p.G + g;
        p.out[row * PI_HEAD_DIM + d] = __float2bfloat16_rn(L > 0.f ? v / L : 0.f);
        if (p.lse && d == 0) p.lse[row] = L > 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
    };
    for (int i = tid; i < n_out; i += A4_THREADS) {
        const int g = i >> 7;
        float M = -INFINITY, L = 0.f, v = 0.f;
#pragma unroll
        for (int k = 0; k < A4_WARPS; ++k) M = fmaxf(M, s_m[k * p.G + g]);
#pragma unroll
        for (int k = 0; k < A4_WARPS; ++k) {
            const float a = M == -INFINITY ? 0.f : exp2f(s_m[k * p.G + g] - M);
            L = fmaf(s_l[k * p.G + g], a, L);
            v = fmaf(s_o[k * n_out + i], a, v);
        }
        if (S == 1) write_out(i, M, L, v);
        else {
            // one thread's own places of warp 0's part, which only it reads; M and L behind all parts
            s_o[i] = v;
            if ((i & 127) == 0) { s_l[A4_WARPS * p.G + g] = M; s_l[A4_WARPS * p.G + p.G + g] = L; }
        }
    }
    if (S == 1) return;
    __syncwarp();
    // ---- and the cluster's: every CTA concludes its share of the outputs, reading the others' shared memory
    cluster_sync_all();
    const uint32_t at_o = smem_u32(s_o), at_m = smem_u32(s_l + A4_WARPS * p.G), at_l = at_m + 4 * p.G;
    for (int i = rank * A4_THREADS + tid; i < n_out; i += S * A4_THREADS) {
        const int g = i >> 7;
        float M = -INFINITY, L = 0.f, v = 0.f;
        for (int k = 0; k < S; ++k) M = fmaxf(M, ld_shared_cluster_f32(map_shared_rank(at_m + 4 * g, k)));
        for (int k = 0; k < S; ++k) {
            const float mk = ld_shared_cluster_f32(map_shared_rank(at_m + 4 * g, k));
            const float a = M == -INFINITY ? 0.f : exp2f(mk - M);
            L = fmaf(ld_shared_cluster_f32(map_shared_rank(at_l + 4 * g, k)), a, L);
            v = fmaf(ld_shared_cluster_f32(map_shared_rank(at_o + 4 * i, k)), a, v);
        }
        write_out(i, M, L, v);
    }
    __syncwarp();
    cluster_sync_all();                                 // nobody leaves while its state may still be read
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
    p.Hq = cfg.n_q_heads; p.Hkv = cfg.n_kv_heads; p.G = cfg.n_q_heads / cfg.n_kv_heads;
    p.B = cfg.block_tokens; p.K = cfg.budget_blocks; p.C = cfg.pool_slots;
    // CTAs per item: as many as fill the GPU with two CTAs per SM, as long as every warp still has a tile
    const long long items = static_cast<long long>(batch) * cfg.n_kv_heads, slots = 2ll * c->n_sms;
    const int tiles = cfg.budget_blocks * (cfg.block_tokens / 16);
    int split = 1;
    while (split < 8 && items * split * 2 <= slots && tiles >= split * 2 * A4_WARPS) split *= 2;
    const size_t ring = static_cast<size_t>(A4_WARPS) * A4_STAGES * KV4_TILE_BYTES;
    const size_t merge = (static_cast<size_t>(A4_WARPS) * p.G * (PI_HEAD_DIM + 2) + 2 * p.G) * sizeof(float);
    const size_t smem = ring > merge ? ring : merge;
    auto launch = [&](auto kernel) -> int {
        PI_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3(static_cast<unsigned>(items * split));
        lc.blockDim = dim3(A4_THREADS);
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
    if (p.G <= 4) return launch(attn_kv4_kernel<1, true>);
    if (p.G <= 8) return launch(attn_kv4_kernel<1, false>);
    return launch(attn_kv4_kernel<2, false>);
}
