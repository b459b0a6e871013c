// Sparse GQA decode attention over a pool of 8-bit blocks:  softmax(q K^T / sqrt(D)) V  over the tokens of the selected
// blocks, K and V = scale of (block, head) * e4m3 number (pi_kv8.cuh).
//
// 256 bytes a (token, KV head) for 4 G D operations: the pool's bytes are what the call cannot do without.  The numbers become fp16 by one
// conversion a pair, exactly, and the scales never meet them: K's multiplies the products, V's the weights.  The contractions run on
// mma.sync (tokens or channels on M, up to 8 query heads on N), whose operands are registers, where the numbers are converted; with 4
// to 16 query heads on N the matrix pipe is far from busy.  Queries are exact in fp16 after a power of two per head.  A weight times V's scale
// is rounded to 11 bits (an eighth of the output's own rounding in the mean square), below 2^-21 of its reference to a multiple of 2^-31
// of it; all sums are in 32 bits.
//
// Weights are counted from two references a head: the sum from the largest score, the products with V from the largest score times
// scale (of V).  So a block whose values are small next to another's, and whose weights are not, keeps its bits, and no weight leaves fp16.
// Both move only when they are exceeded by 2^8; the products' weights are 2^7 times as large, up to 2^15, so that a long tail under one large
// score keeps its bits too.
//
// One (sequence, KV head) per cluster of S CTAs of 4, 8 or 16 warps (S = 1, 2, 4 or 8; both by the launcher's rule).  The item's
// 16-token tiles are dealt out to its warps in turn; a warp streams its own tiles through its own ring of shared-memory
// stages with 16-byte asynchronous copies (a tile is 2048 contiguous bytes of K and as many of V), so no warp waits for another until the
// end (pi_attn_merge.cuh).
//
// Measured on a B200, back to back: 64 sequences x 64 blocks of 32 tokens, 8 KV heads, G = 4 (263 MB) 44 us, 6.0 TB/s, 91 % of what a copy
// reaches; 16 x 128 blocks of 16 (67 MB) 14.6 us; one sequence x 64 blocks 4.3 us; 64 x 64 blocks of 32 with G = 16 55 us.  HBM bounds the large
// ones; the others carry about 5 us of launch, two dependent loads before the first tile, and the merge.
#include <cuda_fp16.h>

#include <algorithm>

#include "pi_attn_merge.cuh"
#include "pi_kv8.cuh"

namespace {

using namespace pi_attn;

constexpr int A8_TILE_BYTES = 4096;                // 16 tokens: K, then V
constexpr float A8_LIFT = 7.f;                     // log2 of the factor of the products' weights
__host__ __device__ constexpr int a8_stages(int NT) { return NT == 1 ? 3 : 6; }          // tiles in the ring
__host__ __device__ constexpr int a8_warps_per_sm(int NT) { return NT == 1 ? 16 : 8; }   // what the registers allow

struct Attn8Params {
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
__device__ __forceinline__ void lds128(uint32_t a, uint32_t (&v)[4]) {
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(a));
}
// Two matrices of 16 rows of 16 bytes, transposed: lane (r, c) gets the bytes r (then r + 8) of rows 4 c .. 4 c + 3 of either.
__device__ __forceinline__ void ldsm_bytes_t(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
// The four numbers of a word as fp16 pairs.
__device__ __forceinline__ void numbers(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// NT: tiles of 8 query heads; WARPS of a CTA.
template <int NT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, a8_warps_per_sm(NT) / WARPS)
attn_kv8_kernel(Attn8Params p) {
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;
    const int S = static_cast<int>(cluster_nctarank()), rank = static_cast<int>(cluster_ctarank());
    const int item = blockIdx.x / S, seq = item / p.Hkv, h = item - seq * p.Hkv;
    constexpr int STAGES = a8_stages(NT);
    const int SUB = p.B >> 4;
    // (the other half of this barrier stands before the first store into another CTA's shared memory: by then it runs)
    if (S > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    pi_grid_dependency_wait();
    pi_launch_dependents();
    // the entries of the warp's first 32 tiles, the queries and the list's length are fetched beside one another
    const int first = rank * WARPS + warp, stride = WARPS * S, log_sub = 31 - __clz(SUB);
    const int32_t* slots = p.sel_slots + static_cast<size_t>(seq) * p.K;
    const int32_t* blocks = p.sel_blocks + static_cast<size_t>(seq) * p.K;
    auto entry_of = [&](int n) -> int2 {
        const int j = (first + n * stride) >> log_sub;
        return j < p.K ? make_int2(slots[j], blocks[j]) : make_int2(0, -1);
    };
    const int2 entry = entry_of(lane);
    // channels 64 i + 16 c + 0 .. 15 of head r: what lane (r, c) contracts with
    uint4 query[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int g = nt * 8 + r;
        const uint4* qg = reinterpret_cast<const uint4*>(p.q + (static_cast<size_t>(seq) * p.Hq + static_cast<size_t>(h) * p.G + (g < p.G ? g : 0)) * PI_HEAD_DIM + 16 * c);
#pragma unroll
        for (int j = 0; j < 4; ++j) query[nt][j] = g < p.G ? __ldg(qg + 8 * (j >> 1) + (j & 1)) : make_uint4(0, 0, 0, 0);
    }
    const int ctx = p.ctx_len[seq];
    int cnt = p.sel_count[seq];
    if (cnt < 0 || cnt > p.K) {
        if (h == 0 && rank == 0 && tid == 0) pi_report(p.st, PI_ERR_CAPACITY, PI_STAGE_ATTN, seq, cnt, p.K);
        cnt = 0;
    }
    const int n_tiles = cnt * SUB;
    const int n_mine = first < n_tiles ? (n_tiles - first + stride - 1) / stride : 0;

    const unsigned char* seq_base = p.pool + static_cast<long long>(seq) * p.C * p.block_bytes;
    const unsigned char* scales = seq_base + static_cast<long long>(p.Hkv) * p.B * 256 + h * 8;
    // The warp's n-th tile: byte offset of its K from the head's first one (a sequence's pool is below 2^32 bytes), valid tokens, and
    // the block's two scales.
    struct Meta { uint32_t offset, valid; float2 scale; };
    auto meta_of = [&](int n, int2 e) -> Meta {
        Meta m = {0u, 0u, make_float2(0.f, 0.f)};
        if (n >= n_mine || e.y < 0) return m;
        const int t = first + n * stride, sub = t & (SUB - 1);
        if (e.x < 0 || e.x >= p.C) {
            if (h == 0) pi_report(p.st, PI_ERR_INDEX_RANGE, PI_STAGE_ATTN, seq, t >> log_sub, e.x);
            return m;
        }
        const long long left = static_cast<long long>(ctx) - (static_cast<long long>(e.y) * p.B + sub * 16);
        if (left <= 0) return m;
        m.offset = static_cast<uint32_t>(e.x * p.block_bytes) + sub * 2048;
        m.valid = left > 16 ? 16u : static_cast<uint32_t>(left);
        m.scale = *reinterpret_cast<const float2*>(scales + e.x * p.block_bytes);
        return m;
    };
    Meta meta = meta_of(lane, entry), meta_next = {0u, 0u, make_float2(0.f, 0.f)};    // of tiles 32 i + lane, and of the 32 after those
    unsigned some = __ballot_sync(0xffffffffu, meta.valid != 0u), some_next = 0u;

    const unsigned char* head_base = seq_base + static_cast<long long>(h) * p.B * 256 + lane * 16;
    const uint32_t v_off = static_cast<uint32_t>(p.B) * 128u;
    const uint32_t ring = smem_u32(smem) + warp * (STAGES * A8_TILE_BYTES);
    const unsigned long long policy = pi_l2_stream_policy();
    // Where a lane's 16 bytes go: row lane / 8 (and every fourth on), chunk lane % 8.  K rows are read 16 bytes a lane, two rows of four chunks at
    // a time, and take the other half of the banks in turn; V's chunks are read from eight rows at a time, each from banks of its own.
    const int ck = lane & 7, rk = lane >> 3;
    const uint32_t to_k = rk * 128 + ((ck ^ ((rk & 1) << 2)) << 4), to_v0 = 2048 + rk * 128 + ((ck ^ rk) << 4), to_v1 = 2048 + (rk + 4) * 128 + ((ck ^ (rk + 4)) << 4);
    uint32_t fill = 0u;                                  // stage of the next tile
    auto issue = [&](int i, unsigned mask, uint32_t offsets) {      // tile i of a batch of 32 into its stage, one commit
        const uint32_t offset = __shfl_sync(0xffffffffu, offsets, i);
        if ((mask >> i) & 1u) {
            const unsigned char* src = head_base + offset;
            const uint32_t dst = ring + fill;
#pragma unroll
            for (int x = 0; x < 4; ++x) copy16(dst + to_k + x * 512, src + x * 512, policy);
#pragma unroll
            for (int x = 0; x < 4; ++x) copy16(dst + ((x & 1) ? to_v1 : to_v0) + (x >> 1) * 1024, src + v_off + x * 512, policy);
        }
        fill = fill == (STAGES - 1) * A8_TILE_BYTES ? 0u : fill + A8_TILE_BYTES;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int n = 0; n < STAGES - 1; ++n) issue(n, some, meta.offset);

    // ---- the queries as B operands, as fp16 numbers: every head is scaled by a power of two so that its largest channel lies in
    // [1, 2); what is below 2^-14 of that is rounded at 2^-25 of it, less than the sums below round.
    uint32_t bq[NT][8][2];
    float scale[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        uint32_t top2 = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            top2 = __vmaxu2(top2, __vmaxu2(__vmaxu2(query[nt][j].x & 0x7fff7fffu, query[nt][j].y & 0x7fff7fffu), __vmaxu2(query[nt][j].z & 0x7fff7fffu, query[nt][j].w & 0x7fff7fffu)));
        top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 1));
        top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 2));
        // the power of two at or below the largest magnitude; at least the smallest normal number, at most 2^126
        const uint32_t field = min(max(max(top2 & 0xffffu, top2 >> 16) >> 7, 1u), 253u);
        const float inv = __uint_as_float((254u - field) << 23);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x[4] = {query[nt][j].x, query[nt][j].y, query[nt][j].z, query[nt][j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                bq[nt][2 * j + (i >> 1)][i & 1] = pack_f16(__uint_as_float(x[i] << 16) * inv, __uint_as_float(x[i] & 0xffff0000u) * inv);
        }
        const float mine = p.scale_log2 * __uint_as_float(field << 23);      // of head r
        scale[nt][0] = __shfl_sync(0xffffffffu, mine, 8 * c);
        scale[nt][1] = __shfl_sync(0xffffffffu, mine, 8 * c + 4);
    }

    // ---- running state of heads 2 c, 2 c + 1: l counted from m (exp2 domain); o[i] = channels 16 i + r (+ 8 in the upper two), V's scale in it, counted
    // from m + d (two numbers: in one, a large score would leave no bits for the scale)
    float o[NT][8][4], m[NT][2], d[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = d[nt][0] = d[nt][1] = A4_NO_MAX;
        l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
    }
    // Row r of a tile's products is token tr (row r + 8: tr + 2): then rows 2 c, 2 c + 1, 2 c + 8, 2 c + 9, which a lane contracts V with, are
    // the four neighbouring tokens 4 c .. 4 c + 3, as the transposed load brings them.
    const int tr = 4 * (r >> 1) + (r & 1);
    const uint32_t from_k0 = tr * 128 + ((c ^ ((tr & 1) << 2)) << 4), from_k1 = tr * 128 + (((c + 4) ^ ((tr & 1) << 2)) << 4);
    const int vrow = lane & 15;
    const uint32_t from_v = 2048 + vrow * 128, vchunk = lane >> 4, vturn = vrow & 7;

    uint32_t tile = ring;                                // the stage at hand
    for (int n = 0; n < n_mine; ++n, tile = tile == ring + (STAGES - 1) * A8_TILE_BYTES ? ring : tile + A8_TILE_BYTES) {
        const int i = n & 31;
        if (i == 0) {
            if (n) { meta = meta_next; some = some_next; }
            some_next = 0u;
            if (n + 32 < n_mine) {
                meta_next = meta_of(n + 32 + lane, entry_of(n + 32 + lane));
                some_next = __ballot_sync(0xffffffffu, meta_next.valid != 0u);
            }
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
        __syncwarp();                                   // the tile is filled by all lanes, and the previous one read by all
        if (i + STAGES - 1 < 32) issue(i + STAGES - 1, some, meta.offset);
        else issue(i + STAGES - 1 - 32, some_next, meta_next.offset);
        if (!((some >> i) & 1u)) continue;
        const int nvalid = static_cast<int>(__shfl_sync(0xffffffffu, meta.valid, i));
        const float k_scale = __shfl_sync(0xffffffffu, meta.scale.x, i), v_scale = __shfl_sync(0xffffffffu, meta.scale.y, i);
        // ---- S^T = K q^T
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            uint32_t ka[4], kb[4];
            lds128(tile + (x ? from_k1 : from_k0), ka);
            lds128(tile + (x ? from_k1 : from_k0) + 256, kb);       // (two tokens on: the same turn)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                uint32_t a0, a1, a2, a3;
                numbers(ka[y], a0, a2);
                numbers(kb[y], a1, a3);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(s[nt], a0, a1, a2, a3, bq[nt][4 * x + y][0], bq[nt][4 * x + y][1]);
            }
        }
        bool over = false;
        // log2 of V's scale: what a weight times it is counted by
        const float v_log = static_cast<float>(static_cast<int>((__float_as_uint(v_scale) >> 23) & 0xffu) - 127);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            // (the scores are rounded before the references are taken off: scores of any size keep their differences)
            const float f0 = scale[nt][0] * k_scale, f1 = scale[nt][1] * k_scale;
            s[nt][0] = __fmul_rn(s[nt][0], f0); s[nt][1] = __fmul_rn(s[nt][1], f1);
            s[nt][2] = __fmul_rn(s[nt][2], f0); s[nt][3] = __fmul_rn(s[nt][3], f1);
        }
        if (nvalid < 16) {                              // what lies behind the last token may be anything, NaN among it
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (tr >= nvalid) s[nt][0] = s[nt][1] = -INFINITY;
                if (tr + 2 >= nvalid) s[nt][2] = s[nt][3] = -INFINITY;
            }
            for (int y = nvalid + rk; y < 16; y += 4) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(tile + 2048 + y * 128 + ck * 16), "r"(0u) : "memory");
            __syncwarp();
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float mx = fmaxf(s[nt][e], s[nt][2 + e]) - m[nt][e];
                over |= fmaxf(mx, mx + (v_log - d[nt][e])) > 8.f;
            }
        if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float mx = fmaxf(s[nt][e], s[nt][2 + e]);
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                    const float m_new = fmaxf(m[nt][e], mx), fall = m[nt][e] - m_new, d_new = fmaxf(d[nt][e] + fall, (mx - m_new) + v_log);
                    l[nt][e] *= ex2(fall);
                    const float alpha = ex2(fall + (d[nt][e] - d_new));
                    m[nt][e] = m_new;
                    d[nt][e] = d_new;
#pragma unroll
                    for (int x = 0; x < 8; ++x) { o[nt][x][e] *= alpha; o[nt][x][2 + e] *= alpha; }
                }
        }
        // ---- the weights, and O^T += V^T (weight scale)
        uint32_t b0[NT], b1[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float w[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float t0 = s[nt][e] - m[nt][e], t1 = s[nt][2 + e] - m[nt][e], by = v_log - d[nt][e] + A8_LIFT;
                l[nt][e] += ex2(t0) + ex2(t1);
                w[e] = ex2(t0 + by);
                w[2 + e] = ex2(t1 + by);
            }
            b0[nt] = movm_t(pack_f16(w[0], w[1]));
            b1[nt] = movm_t(pack_f16(w[2], w[3]));
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            uint32_t v[4];
            ldsm_bytes_t(tile + from_v + (((2 * x + vchunk) ^ vturn) << 4), v);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                uint32_t a0, a1, a2, a3;
                numbers(v[2 * y], a0, a2);
                numbers(v[2 * y + 1], a1, a3);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][2 * x + y], a0, a1, a2, a3, b0[nt], b1[nt]);
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");

    // ---- the warp's state into shared memory: o [warp][G][128] counted from m, then m and l [warp][G] (the ring is done with)
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
            for (int x = 4; x <= 16; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
            const int g = nt * 8 + 2 * c + e;
            // 2^d without the factor, in two steps: scales reach from 2^-117 to 2^120
            const float f = m[nt][e] == A4_NO_MAX ? 0.f : ex2(0.5f * (d[nt][e] - A8_LIFT));
            if (g >= p.G) continue;
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                s_o[(warp * p.G + g) * PI_HEAD_DIM + 16 * x + r] = o[nt][x][e] * f * f;
                s_o[(warp * p.G + g) * PI_HEAD_DIM + 16 * x + 8 + r] = o[nt][x][2 + e] * f * f;
            }
            if (r == 0) { s_m[warp * p.G + g] = m[nt][e]; s_l[warp * p.G + g] = sum; }
        }
    __syncthreads();
    conclude<WARPS>(p, seq, h, S, rank, tid, s_o, s_m, s_l, reinterpret_cast<float4*>(smem + WARPS * STAGES * A8_TILE_BYTES));
}

}  // namespace

int pi_launch_attn_kv8(pi_ctx* c, int batch, const void* q, const void* pool, const int32_t* sel_slots, const int32_t* sel_blocks,
                       const int32_t* sel_count, const int32_t* ctx_len, void* out, float* lse, cudaStream_t stream) {
    const pi_config& cfg = c->cfg;
    Attn8Params p;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.pool = static_cast<const unsigned char*>(pool);
    p.sel_slots = sel_slots; p.sel_blocks = sel_blocks; p.sel_count = sel_count; p.ctx_len = ctx_len;
    p.out = static_cast<__nv_bfloat16*>(out);
    p.lse = lse;
    p.st = pi_status_of(c);
    p.block_bytes = kv8_block_bytes(cfg.n_kv_heads, cfg.block_tokens);
    p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(PI_HEAD_DIM));
    p.Hq = cfg.n_q_heads; p.Hkv = cfg.n_kv_heads; p.G = cfg.n_q_heads / cfg.n_kv_heads;
    p.B = cfg.block_tokens; p.K = cfg.budget_blocks; p.C = cfg.pool_slots;
    const int NT = p.G <= 8 ? 1 : 2, tiles = cfg.budget_blocks * (cfg.block_tokens / 16);
    const long long items = static_cast<long long>(batch) * cfg.n_kv_heads, room = static_cast<long long>(a8_warps_per_sm(NT)) * c->n_sms;
    int split = 1, warps = 4;
    if (NT == 1 && items * 8 >= 5 * c->n_sms) {
        // Items enough for most of the SMs: a CTA each, of as many warps as fill seven tenths of the room at most, with four tiles a warp.  4 / 8 / 16 warps:
        // 96 items x 128 tiles 19.5 / 13.6 / 12.7 us, 128 x 128 19.9 / 14.6 / 14.9 (two CTAs of 4 warps 15.2), 192 x 128 23.0 / 19.8 / 25.8,
        // 256 x 128 24.6 / 24.8 / 27.6, 384 x 64 19.3 / 24.4 / 26.8.
        while (warps < 16 && items * warps * 2 * 10 <= room * 7 && tiles >= 4 * warps) warps *= 2;
    } else {
        // CTAs per item: twice as many while they fill half of the warps there is room for, at most, and every warp has two tiles.  Measured with
        // S = 1 / 2 / 4 / 8: 8 items x 64 tiles 10.4 / 7.3 / 5.3 / 4.3 us, 32 x 128 19.1 / 11.9 / 8.3 / 6.8, 64 x 256 36.7 / 20.8 / 15.1 / 15.6.
        while (split < A4_MAX_SPLIT && items * split * 2 * warps <= room / 2 && tiles >= 2 * warps * split * 2) split *= 2;
        // Few items with long lists leave SMs with one CTA each, which more warps use better, two tiles a warp or four: 8 items x 256 tiles
        // 6.4 us with 8, 6.6 with 16; x 512 8.6 and 7.8; x 1024 20.1 with 4, 13.7 with 8, 12.0 with 16; x 2048 23.3 and 19.1.
        if (NT == 1 && split == A4_MAX_SPLIT)
            while (warps < 16 && items * split * warps * 2 <= room / 2 && tiles >= warps * warps * split) warps *= 2;
    }
    const size_t ring = static_cast<size_t>(warps) * a8_stages(NT) * A8_TILE_BYTES;
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
    if (NT == 1) return warps == 4 ? launch(attn_kv8_kernel<1, 4>) : warps == 8 ? launch(attn_kv8_kernel<1, 8>) : launch(attn_kv8_kernel<1, 16>);
    return launch(attn_kv8_kernel<2, 4>);
}
