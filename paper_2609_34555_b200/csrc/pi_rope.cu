// Norm of every query and key head and the position rotation, from the projections to the tensors the path takes.
//
//   y = x * rsqrt(mean(x^2) + eps) * w          (no weights given: y = x)
//   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin)   for the pairs of the first rot_dim channels, at the angle
//   position * inv_freq[pair]; one rounding, to bf16, at the end.
//
// Streams each row once; bound by HBM from a few thousand tokens on, by latency below (B200, back to back: 32768 tokens of
// 32 + 8 bf16 heads, 671 MB, 120 us, 5.6 TB/s; 2049 tokens of 64 + 8 fp16 heads 17.5 us; 16 tokens 1.9 us;
// 8192 tokens of 32 + 8 heads 34 us in 16 bits, 44 us in 32).  A warp works on one token, four
// rows at a time: eight lanes a row, 16 channels a lane: two runs of 8, chosen so that both members of a pair are
// in one lane for neighbouring pairs and for pairs any multiple of 8 channels apart; other distances go through shared memory.  The token's angles are
// taken once per warp, two per lane, and shared through shared memory: the product position * inv_freq in 64 bits
// (32 lose a far position's angle: at 131072 radians their spacing is 2^-7), reduced to a fraction of a turn there,
// the sine and cosine of the rest in 32.
#include <cuda_fp16.h>

#include "pi_common.cuh"

namespace {

constexpr int ROPE_THREADS = 64;
constexpr int ROPE_WARPS = ROPE_THREADS / 32;

struct RopeParams {
    const void* q;
    const void* k;
    long long q_stride, k_stride;                  // elements between tokens
    const int32_t* pos;
    const float* wq;
    const float* wk;
    const float* inv_freq;
    __nv_bfloat16* q_out;
    __nv_bfloat16* k_out;
    float eps;
    int n_tokens, Hq, Hkv, half, parts;            // half = rot_dim / 2; parts = warps a token is cut into
};

template <typename T> struct Raw;                  // eight values as they are loaded
template <> struct Raw<__nv_bfloat16> { uint4 a; };
template <> struct Raw<__half> { uint4 a; };
template <> struct Raw<float> { uint4 a, b; };

__device__ __forceinline__ uint4 load_once(const uint4* p) {         // (L1 is left to the weights)
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, Raw<T>& r) {
    r.a = load_once(reinterpret_cast<const uint4*>(p));
    if constexpr (sizeof(T) == 4) r.b = load_once(reinterpret_cast<const uint4*>(p) + 1);
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw<T>& r, float* f) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            const uint32_t w2[4] = {r.b.x, r.b.y, r.b.z, r.b.w};
            f[i] = __uint_as_float(w[i]);
            f[4 + i] = __uint_as_float(w2[i]);
        } else if constexpr (std::is_same<T, __half>::value) {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = v.x; f[2 * i + 1] = v.y;
        } else {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
__device__ __forceinline__ uint4 narrow8(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// How a pair's members lie: 64 channels apart, side by side, a multiple of 8 apart, any other distance.
enum { PAIR_HALVES_FULL = 0, PAIR_NEIGHBOURS = 1, PAIR_HALVES_RUNS = 2, PAIR_HALVES_ANY = 3 };

// What the registers are cut to.  16-bit inputs, pairs at a fixed distance: 64 registers, 32 warps an SM with 1 KB of loads each on
// their way.  Other distances want 72 (8192 tokens of 40 heads, 64 channels turned: 34.8 us, 41.2 with 64); 32-bit inputs,
// with twice the bytes a load, 96 (43.7 us; 45 with 80 and 74 with 64, where they no longer fit).
constexpr int rope_ctas_per_sm(int bytes, int pair) { return bytes == 4 ? 10 : pair == PAIR_HALVES_FULL || pair == PAIR_NEIGHBOURS ? 16 : 14; }

template <typename T, int PAIR>
__global__ void __launch_bounds__(ROPE_THREADS, rope_ctas_per_sm(sizeof(T), PAIR))
qk_norm_rope_kernel(RopeParams p) {
    __shared__ float2 s_cs[ROPE_WARPS][64];                                    // cos, sin of the token's angles
    __shared__ float s_row[PAIR == PAIR_HALVES_ANY ? ROPE_WARPS : 1][4][8 * 16 + 8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane >> 3, l = lane & 7;
    const long long unit = static_cast<long long>(blockIdx.x) * ROPE_WARPS + warp;
    pi_grid_dependency_wait();
    pi_launch_dependents();
    if (unit >= static_cast<long long>(p.n_tokens) * p.parts) return;
    const int t = static_cast<int>(unit / p.parts), part = static_cast<int>(unit - static_cast<long long>(t) * p.parts);
    const int H = p.Hq + p.Hkv, n_quads = (H + 3) >> 2;
    const T* q = static_cast<const T*>(p.q) + t * p.q_stride;
    const T* k = static_cast<const T*>(p.k) + t * p.k_stride;

    // The lane's two runs of 8 channels.  Pairs a multiple of 8 apart: run i and run i + half / 8, and of the channels that are not
    // turned the rest, in order.
    const int gap = p.half >> 3;
    const bool turned = PAIR != PAIR_HALVES_RUNS || l < gap;
    const int run_a = turned ? l : l + gap, run_b = PAIR == PAIR_HALVES_RUNS && turned ? l + gap : l + 8;
    auto src = [&](int row) { return row < p.Hq ? q + row * PI_HEAD_DIM : k + (row - p.Hq) * PI_HEAD_DIM; };
    Raw<T> a = {}, b = {};
    int quad = part;
    int row = quad * 4 + sub;
    if (row < H) { load8(src(row) + 8 * run_a, a); load8(src(row) + 8 * run_b, b); }
    const float freq[2] = {lane < p.half ? __ldg(p.inv_freq + lane) : 0.f, lane + 32 < p.half ? __ldg(p.inv_freq + lane + 32) : 0.f};
    const int pos = p.pos[t];
    if (pos < 0) return;                                                       // a padding token: its rows stay as they were
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int f = lane + 32 * i;
        float2 cs = make_float2(1.f, 0.f);                                     // channels beyond rot_dim are not turned
        if (f < p.half) {
            double turns = static_cast<double>(pos) * static_cast<double>(freq[i]) * 0.15915494309189533577;   // 1 / (2 pi)
            turns -= rint(turns);
            sincospif(2.f * static_cast<float>(turns), &cs.y, &cs.x);
        }
        s_cs[warp][PAIR == PAIR_HALVES_ANY ? (f & 7) * 8 + (f >> 3) : f] = cs;
    }
    __syncwarp();
    float2 cs[8];                                                              // this lane's eight angles
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (PAIR == PAIR_HALVES_ANY) {                                        // of the lane's first run; the sine with its sign
            const int d = 8 * l + e, f = d < p.half ? d : d - p.half;          // (f < 64)
            cs[e] = s_cs[warp][(f & 7) * 8 + (f >> 3)];
            if (d < p.half) cs[e].y = -cs[e].y;
        } else {
            cs[e] = s_cs[warp][PAIR == PAIR_NEIGHBOURS ? (e < 4 ? 4 * l + e : 32 + 4 * l + e - 4) : 8 * l + e];
        }
    }

    for (; quad < n_quads; quad += p.parts) {
        row = quad * 4 + sub;
        float x[16];
        widen8(a, x);
        widen8(b, x + 8);
        const int next = row + 4 * p.parts;
        if (next < H) { load8(src(next) + 8 * run_a, a); load8(src(next) + 8 * run_b, b); }
        if (p.wq) {
            // (the weights come out of L1 every time: kept in registers they would cost a quarter of the resident warps)
            const float4* g = reinterpret_cast<const float4*>(row >= p.Hq ? p.wk : p.wq);
            float4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __ldg(g + 2 * (i < 2 ? run_a : run_b) + (i & 1));
            auto squares = [&]() {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
                ss += __shfl_xor_sync(0xffffffffu, ss, 1);
                ss += __shfl_xor_sync(0xffffffffu, ss, 2);
                return ss + __shfl_xor_sync(0xffffffffu, ss, 4);
            };
            float ss = squares(), eps = p.eps;
            if (!std::is_same<T, __half>::value) {
                // Rows whose squares leave 32 bits (2^60 and more, or 2^-50 and less where eps does not cover them) are taken 2^80 times
                // smaller or larger, which the quotient does not show.
                const bool large = ss > 0x1p126f, small = ss < 0x1p-100f && p.eps < 0x1p-70f;
                if (__any_sync(0xffffffffu, large || small)) {
                    const float f = large ? 0x1p-80f : small ? 0x1p80f : 1.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] *= f;
                    ss = squares();
                    eps = p.eps * f * f;
                }
            }
            const float r = rsqrtf(ss * (1.f / PI_HEAD_DIM) + eps);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[4 * i] *= r * w[i].x; x[4 * i + 1] *= r * w[i].y; x[4 * i + 2] *= r * w[i].z; x[4 * i + 3] *= r * w[i].w;
            }
        }
        if (PAIR == PAIR_HALVES_FULL || PAIR == PAIR_HALVES_RUNS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!turned) continue;
                const float u = x[e], v = x[8 + e];
                x[e] = u * cs[e].x - v * cs[e].y;
                x[8 + e] = v * cs[e].x + u * cs[e].y;
            }
        } else if (PAIR == PAIR_NEIGHBOURS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if ((e < 4 ? 4 * l + e : 32 + 4 * l + e - 4) >= p.half) continue;
                const float u = x[2 * e], v = x[2 * e + 1];
                x[2 * e] = u * cs[e].x - v * cs[e].y;
                x[2 * e + 1] = v * cs[e].x + u * cs[e].y;
            }
        } else {
            // The members of a pair are rot_dim / 2 channels apart, in whichever lanes: through shared memory, channel d at
            // place 16 (d % 8) + d / 8, so that for any distance the lanes' places lie side by side.
            float* sr = s_row[warp][sub];
            const bool both = p.half > 32;                                     // the second run is turned too
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sr[16 * e + l] = x[e];
                if (both) sr[16 * e + 8 + l] = x[8 + e];
            }
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int d = 8 * l + e, o = d < p.half ? d + p.half : d - p.half;
                if (d < 2 * p.half) x[e] = fmaf(x[e], cs[e].x, sr[16 * (o & 7) + (o >> 3)] * cs[e].y);
                const int f = d + 64 - p.half;                                // (of the second run: always the second member of its pair)
                if (both && f < p.half) {
                    const float2 z = s_cs[warp][(f & 7) * 8 + (f >> 3)];
                    x[8 + e] = fmaf(x[8 + e], z.x, sr[16 * (f & 7) + (f >> 3)] * z.y);
                }
            }
        }
        if (row < H) {
            uint4* dst = reinterpret_cast<uint4*>(row < p.Hq ? p.q_out + (static_cast<size_t>(t) * p.Hq + row) * PI_HEAD_DIM
                                                             : p.k_out + (static_cast<size_t>(t) * p.Hkv + row - p.Hq) * PI_HEAD_DIM);
            dst[run_a] = narrow8(x);
            dst[run_b] = narrow8(x + 8);
        }
    }
}

template <typename T>
int launch(const RopeParams& p, int interleaved, cudaStream_t stream) {
    const long long units = static_cast<long long>(p.n_tokens) * p.parts;
    const dim3 grid(static_cast<unsigned>((units + ROPE_WARPS - 1) / ROPE_WARPS)), block(ROPE_THREADS);
    if (interleaved || p.half == 0) PI_CUDA_TRY(pi_launch_pdl(qk_norm_rope_kernel<T, PAIR_NEIGHBOURS>, grid, block, 0, stream, p));
    else if (p.half == 64) PI_CUDA_TRY(pi_launch_pdl(qk_norm_rope_kernel<T, PAIR_HALVES_FULL>, grid, block, 0, stream, p));
    else if (p.half % 8 == 0) PI_CUDA_TRY(pi_launch_pdl(qk_norm_rope_kernel<T, PAIR_HALVES_RUNS>, grid, block, 0, stream, p));
    else PI_CUDA_TRY(pi_launch_pdl(qk_norm_rope_kernel<T, PAIR_HALVES_ANY>, grid, block, 0, stream, p));
    return PI_OK;
}

}  // namespace

int pi_launch_qk_norm_rope(pi_ctx* c, int n_tokens, int dtype, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                           const int32_t* pos, const float* wq, const float* wk, float eps, const float* inv_freq, int rot_dim,
                           int interleaved, void* q_out, void* k_out, cudaStream_t stream) {
    RopeParams p;
    p.q = q; p.k = k; p.q_stride = q_stride; p.k_stride = k_stride;
    p.pos = pos; p.wq = wq; p.wk = wk; p.inv_freq = inv_freq;
    p.q_out = static_cast<__nv_bfloat16*>(q_out); p.k_out = static_cast<__nv_bfloat16*>(k_out);
    p.eps = eps; p.n_tokens = n_tokens; p.Hq = c->cfg.n_q_heads; p.Hkv = c->cfg.n_kv_heads; p.half = rot_dim / 2;
    // few tokens: a token's rows are spread over several warps, down to four rows each
    const long long want = static_cast<long long>(c->n_sms) * 16;
    const int quads = (p.Hq + p.Hkv + 3) / 4;
    long long parts = (want + n_tokens - 1) / n_tokens;
    p.parts = static_cast<int>(parts < 1 ? 1 : parts > quads ? quads : parts);
    if (dtype == PI_DTYPE_BF16) return launch<__nv_bfloat16>(p, interleaved, stream);
    if (dtype == PI_DTYPE_FP16) return launch<__half>(p, interleaved, stream);
    return launch<float>(p, interleaved, stream);
}
