// The 8-bit form of a KV block and the arithmetic of its numbers, shared by the kernels that write and read it.
//
// A block is [Hkv][K, V][B tokens][128] e4m3 numbers (a sign, four bits of exponent, three of fraction), as the bf16 block is laid
// out, and behind them [Hkv][K, V] scales in fp32; the whole is rounded up to a multiple of 128 bytes.  The tokens of a block
// share the scale of their head and of K or V: a power of two, 2^-7 of the one at or below the largest magnitude among
// them, and at least 2^-117.  The largest number is then below or at 256, so none leaves the format's range, and a value is off by at most half
// a step of its own size, 2^-4, down to 2^-13 of the largest; what is smaller is off by 2^-17 of the largest at most.
//
// A power of two, because scales change: a token joins a block that others are in, and where it is larger than their scale allows they
// are rounded again.  Under a scale 2^k times as large a number keeps its fraction (unless it falls among the smallest), so
// rounding twice is rounding once.  Any other factor would cost every old token half a step each time.
#pragma once

#include "pi_common.cuh"

static inline int64_t kv8_block_bytes(int n_kv_heads, int block_tokens) {
    return static_cast<int64_t>(n_kv_heads) * block_tokens * 256 + (static_cast<int64_t>(n_kv_heads) * 8 + 127) / 128 * 128;
}

#ifdef __CUDACC__
constexpr int KV8_LEAST = 17;                       // exponent field of the smallest magnitude that counts: 2^-110

// The larger of two pairs of magnitudes (bf16, signs cleared), of which infinities and NaN do not count.
__device__ __forceinline__ uint32_t kv8_finite(uint32_t w) {
    w &= 0x7fff7fffu;
    const uint32_t odd = ((w + 0x00800080u) >> 15) & 0x00010001u;        // 1 where the exponent is all ones
    return w & ~(odd * 0xffffu);
}
// Exponent field of the power of two at or below the larger half of w, bounded below; a scale is 2^-7 of that.
__device__ __forceinline__ int kv8_field(uint32_t w) { return max(static_cast<int>(max(w & 0xffffu, w >> 16) >> 7), KV8_LEAST); }
__device__ __forceinline__ float kv8_scale_of(int field) { return __uint_as_float(static_cast<uint32_t>(field - 7) << 23); }
__device__ __forceinline__ float kv8_inverse_of(int field) { return __uint_as_float(static_cast<uint32_t>(261 - field) << 23); }
// The field of a scale out of a block, whatever is in a block that nothing has been stored in yet.
__device__ __forceinline__ int kv8_field_of(uint32_t scale_bits) { return min(max(static_cast<int>((scale_bits >> 23) & 0xffu) + 7, KV8_LEAST), 254); }

__device__ __forceinline__ uint32_t kv8_pair(float lo, float hi) {
    unsigned short d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
    return d;
}
// Four numbers of a row, rounded: x two words of bf16 pairs.  What is no number, or infinite, becomes NaN.
__device__ __forceinline__ uint32_t kv8_round4(uint32_t x0, uint32_t x1, float inverse) {
    const uint32_t x[2] = {x0, x1};
    uint32_t got[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float lo = __uint_as_float(x[i] << 16), hi = __uint_as_float(x[i] & 0xffff0000u);
        got[i] = kv8_pair(lo * inverse, hi * inverse);
        const uint32_t odd = (((x[i] & 0x7fff7fffu) + 0x00800080u) >> 15) & 0x00010001u;
        if (odd) got[i] = (odd & 1u ? 0x7fu : got[i] & 0xffu) | (odd >> 16 ? 0x7f00u : got[i] & 0xff00u);
    }
    return got[0] | got[1] << 16;
}
// The same where everything is known to be a finite number, in a third of the operations.
__device__ __forceinline__ uint32_t kv8_round4_finite(uint32_t x0, uint32_t x1, float inverse) {
    const uint32_t a = kv8_pair(__uint_as_float(x0 << 16) * inverse, __uint_as_float(x0 & 0xffff0000u) * inverse);
    const uint32_t b = kv8_pair(__uint_as_float(x1 << 16) * inverse, __uint_as_float(x1 & 0xffff0000u) * inverse);
    return a | b << 16;
}
// The larger magnitudes of two pairs; NaN where either is NaN.  (One operation with the absolute value in it.)
__device__ __forceinline__ uint32_t kv8_larger(uint32_t a, uint32_t b) {
    const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&m);
}
__device__ __forceinline__ bool kv8_odd(uint32_t w) { return ((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u; }      // infinite or NaN, either half
__device__ __forceinline__ float2 kv8_values(uint32_t pair) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<unsigned short>(pair)));
    float2 f;
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}" : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}
// Four numbers under another scale: times 2^-by, rounded once more.
__device__ __forceinline__ uint32_t kv8_again4(uint32_t codes, float factor) {
    const float2 a = kv8_values(codes & 0xffffu), b = kv8_values(codes >> 16);
    return kv8_pair(a.x * factor, a.y * factor) | kv8_pair(b.x * factor, b.y * factor) << 16;
}
// 2^-(raise of the field), 0 where it is out of range
__device__ __forceinline__ float kv8_factor(int from, int to) { return to - from > 126 ? 0.f : __uint_as_float(static_cast<uint32_t>(127 - (to - from)) << 23); }
#endif
