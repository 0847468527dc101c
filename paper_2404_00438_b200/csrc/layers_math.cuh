// Element-wise arithmetic shared by the layer kernels (binary32): activations, their slopes, the
// 8-bit block form.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>
#include <type_traits>

#include "dlion_layers.h"

namespace dlion {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {       // 2 ulp; results below 2^-126 become 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float recip_fast(float x) {      // 1 ulp
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 1 / (1 + 2^t)
__device__ __forceinline__ float logistic2(float t) { return recip_fast(1.0f + exp2_fast(t)); }

// Beyond 64 the gelu argument only saturates the logistic; held there, its square cannot overflow.  (A NaN is lost here and
// comes back with the factor z.)
__device__ __forceinline__ float held(float z, float most) { return fminf(fmaxf(z, -most), most); }

// half of 1 + tanh(u) is the logistic function of 2u = kGelu2c z (1 + 0.044715 z^2), so every activation costs one ex2 and
// one rcp; -log2(e) is folded into the polynomial.
constexpr float kGelu2c = 1.5957691216057308f;              // 2 sqrt(2/pi)
constexpr float kGeluA = -kGelu2c * kLog2e, kGeluB = kGeluA * 0.044715f;

// The kind is a template parameter: chosen element by element it would keep the elements of a thread from
// overlapping, and a product's epilogue is bound by that latency (the 8192 x 2048 x 8192 product with gelu and
// 8-bit z: 335 us so, 236 us with the choice made once for 32 elements).
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if (ACT == DLION_ACT_RELU) return z < 0.0f ? 0.0f : z;  // NaN stays
    if (ACT == DLION_ACT_SILU) return z * logistic2(-kLog2e * z);
    if (ACT == DLION_ACT_GELU) {
        const float c = held(z, 64.0f);
        return z * logistic2(c * __fmaf_rn(kGeluB, c * c, kGeluA));
    }
    return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if (ACT == DLION_ACT_RELU) return z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
    if (ACT == DLION_ACT_SILU) {
        const float p = logistic2(-kLog2e * z);
        return __fmaf_rn(z * p, 1.0f - p, p);
    }
    if (ACT == DLION_ACT_GELU) {
        const float c = held(z, 64.0f), c2 = c * c;
        const float p = logistic2(c * __fmaf_rn(kGeluB, c2, kGeluA));
        // the factor z last: p (1 - p) is 0 where z times the polynomial would overflow
        return __fmaf_rn(z, __fmaf_rn(0.134145f * kGelu2c, c2, kGelu2c) * __fmaf_rn(-p, p, p), p);
    }
    return 1.0f;
}

// f(std::integral_constant<int, act>) for a kind known at run time
template <class F>
__device__ __forceinline__ void with_act(int act, F f) {
    if (act == DLION_ACT_GELU) {
        f(std::integral_constant<int, DLION_ACT_GELU>{});
    } else if (act == DLION_ACT_SILU) {
        f(std::integral_constant<int, DLION_ACT_SILU>{});
    } else if (act == DLION_ACT_RELU) {
        f(std::integral_constant<int, DLION_ACT_RELU>{});
    } else {
        f(std::integral_constant<int, DLION_ACT_NONE>{});
    }
}

// ---- the 8-bit form: 32 values share 2^(e-127)
// The exponent stops at 248: a step more and what lies above 63.5 steps, bf16's largest value too, would be restored as
// infinity.  There, and only there, a value can lie above 127 steps; it is held as 127 (within8).
constexpr uint32_t kTop8 = 248;
constexpr float kMost8 = 127.0f * 0x1p121f;

// amax_bits: largest |v| of the block as its bit pattern (so that NaN and infinity order last).
__device__ __forceinline__ uint32_t block_exponent(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return 255u;
    // 127 = 1.984375 * 2^6: the power of two is 2^(E-6), or 2^(E-5) when the fraction is above that
    const int e = static_cast<int>(amax_bits >> 23) - 6 + ((amax_bits & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    return e < 1 ? 1u : min(static_cast<uint32_t>(e), kTop8);
}

__device__ __forceinline__ float within8(float v) { return fminf(fmaxf(v, -kMost8), kMost8); }

__device__ __forceinline__ float block_scale(uint32_t e) { return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23); }

// 1 / 2^(e-127), exact (e is in [1, 248] or marks a non-finite block, whose q says nothing)
__device__ __forceinline__ float block_inverse(uint32_t e) { return e == 255u ? 0.0f : __uint_as_float((254u - e) << 23); }

// Conversions between integers and floats run at an eighth of the rate of additions, so the integer is read off, or put
// into, the low bits of 1.5 * 2^23 (or 2^23) plus itself.

// v / 2^(e-127) to the nearest integer, in the low 8 bits
__device__ __forceinline__ uint32_t quantise8(float v, float inverse) { return __float_as_uint(__fmaf_rn(v, inverse, 12582912.0f)); }

// bytes 0 of four words
__device__ __forceinline__ uint32_t bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// The signed bytes of a word, times 2^(e-127).
__device__ __forceinline__ void restore4(uint32_t w, float scale, float (&v)[4]) {
    w ^= 0x80808080u;                                       // q + 128
    v[0] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440)) - 8388736.0f) * scale;
    v[1] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7441)) - 8388736.0f) * scale;
    v[2] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7442)) - 8388736.0f) * scale;
    v[3] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7443)) - 8388736.0f) * scale;
}

// the larger size, NaN if either is
__device__ __forceinline__ float larger(float top, float v) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(top), "f"(fabsf(v)));
    return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ void widen(const uint4& w, float (&v)[8]) {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(x[i]);
        v[2 * i + 1] = bf16_hi(x[i]);
    }
}

// ---- pairs of binary32 values: one instruction for two (in the time of two: it saves issue slots)
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\n"
        "fma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }

__device__ __forceinline__ void widen(const uint4& w, float2 (&v)[4]) {
    v[0] = make_float2(bf16_lo(w.x), bf16_hi(w.x));
    v[1] = make_float2(bf16_lo(w.y), bf16_hi(w.y));
    v[2] = make_float2(bf16_lo(w.z), bf16_hi(w.z));
    v[3] = make_float2(bf16_lo(w.w), bf16_hi(w.w));
}

}  // namespace dlion
