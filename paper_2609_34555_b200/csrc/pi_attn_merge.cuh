// The end of the attention kernels that give a (sequence, KV head) to a cluster of S CTAs and its tiles to their warps: the warps' softmax
// states, in shared memory, into one, and the result to global memory.
#pragma once

#include <type_traits>

#include "pi_attn_core.cuh"

namespace pi_attn {

constexpr int A4_MAX_SPLIT = 8;                    // CTAs of a cluster that share an item
constexpr float A4_NO_MAX = -3.40282347e38f;       // the lowest number, for -infinity in the running maximum: differences are no NaN

__device__ __forceinline__ void st_cluster_f32x4(uint32_t addr, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster_f32x2(uint32_t addr, float a, float b) {
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1,%2};" ::"r"(addr), "f"(a), "f"(b) : "memory");
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// s_o [WARPS][G][128], s_m and s_l [WARPS][G] (maxima in the exponent's domain, sums under them), written by all of the CTA's warps
// and a __syncthreads() ago; s_in: room for what the cluster sends, G (512 + 8 S) bytes, in use by nothing else.  Where S > 1, every thread
// has arrived at the cluster's barrier once (barrier.cluster.arrive), long ago.
template <int WARPS, typename P>
__device__ __forceinline__ void conclude(const P& p, int seq, int h, int S, int rank, int tid, const float* s_o, const float* s_m, const float* s_l, float4* s_in) {
    // ---- the warps' states into one, four channels (a quad) a thread.  The result goes out, or, where a cluster shares the
    // item, to the CTA that concludes these channels: every head's 32 quads are cut into S runs, run d goes into rank d's
    // s_in [from][head][quad of the run], with the {maximum, sum} of the head in s_ml [from][head].
    const int n_quads = p.G * (PI_HEAD_DIM / 4), log_run = 5 - (31 - __clz(S)), run = 1 << log_run, share = p.G << log_run;
    float2* s_ml = reinterpret_cast<float2*>(s_in + S * share);
    auto write_out = [&](int g, int quad, float M, float L, float4 v) {
        const size_t row = static_cast<size_t>(seq) * p.Hq + static_cast<size_t>(h) * p.G + g;
        const float f = L > 0.f ? 1.f / L : 0.f;
        // (a NaN among the sums has to come through: 0 only where nothing was summed)
        const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x * f, v.y * f), hi = __floats2bfloat162_rn(v.z * f, v.w * f);
        *reinterpret_cast<uint2*>(p.out + row * PI_HEAD_DIM + 4 * quad) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        if (p.lse && quad == 0) p.lse[row] = L > 0.f ? (M + log2f(L)) * 0.6931471805599453f : L == 0.f ? -INFINITY : L;
    };
    // N states {maximum, sum, quad} into one
    auto join = [&](auto number, const float* m_of, const float* l_of, int ml_step, const float4* v_of, int v_step, int n, float& M, float& L, float4& v) {
        constexpr int N = decltype(number)::value;
        float mk[N], lk[N];
        float4 x[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const bool has = k < n;
            mk[k] = has ? m_of[k * ml_step] : A4_NO_MAX;
            lk[k] = has ? l_of[k * ml_step] : 0.f;
            x[k] = has ? v_of[k * v_step] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        M = A4_NO_MAX; L = 0.f;
        v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < N; ++k) M = fmaxf(M, mk[k]);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float f = ex2(mk[k] - M);
            L = fmaf(lk[k], f, L);
            v.x = fmaf(x[k].x, f, v.x); v.y = fmaf(x[k].y, f, v.y); v.z = fmaf(x[k].z, f, v.z); v.w = fmaf(x[k].w, f, v.w);
        }
    };
    if (S > 1) asm volatile("barrier.cluster.wait;" ::: "memory");        // every CTA of the cluster has begun
    for (int i = tid; i < n_quads; i += WARPS * 32) {
        const int g = i >> 5, quad = i & 31;
        float M, L;
        float4 v;
        join(std::integral_constant<int, WARPS>(), s_m + g, s_l + g, p.G, reinterpret_cast<const float4*>(s_o) + i, n_quads, WARPS, M, L, v);
        if (S == 1) { write_out(g, quad, M, L, v); continue; }
        const int to = quad >> log_run, at = quad & (run - 1);
        st_cluster_f32x4(map_shared_rank(smem_u32(s_in + rank * share + (g << log_run) + at), to), v);
        if (at == 0) st_cluster_f32x2(map_shared_rank(smem_u32(s_ml + rank * p.G + g), to), M, L);
    }
    if (S == 1) return;
    asm volatile("barrier.cluster.arrive;\n\tbarrier.cluster.wait;" ::: "memory");      // (not .aligned: lanes leave the loop at different times)
    // ---- this CTA's share of the outputs, out of its own shared memory
    for (int t = tid; t < share; t += WARPS * 32) {
        const int g = t >> log_run;
        const float* ml = reinterpret_cast<const float*>(s_ml + g);
        float M, L;
        float4 v;
        join(std::integral_constant<int, A4_MAX_SPLIT>(), ml, ml + 1, 2 * p.G, s_in + t, share, S, M, L, v);
        write_out(g, (rank << log_run) + (t & (run - 1)), M, L, v);
    }
}

}  // namespace pi_attn
