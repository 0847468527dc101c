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

__device__ __forceinline__ float logistic(float t) { return recip_fast(1.0f + exp2_fast(-kLog2e * t)); }

// Beyond 64 the gelu argument only saturates the logistic; held there, its square cannot overflow.
__device__ __forceinline__ float gelu_arg(float z) { return fabsf(z) > 64.0f ? copysignf(64.0f, z) : z; }

constexpr float kGelu2c = 1.5957691216057308f;              // 2 sqrt(2/pi)

// half of 1 + tanh(u) is the logistic function of 2u, so every activation costs one ex2 and one rcp.
// The kind is a template parameter: chosen element by element it would keep the elements of a thread from
// overlapping, and a product's epilogue is bound by that latency (the 8192 x 2048 x 8192 product with gelu and
// 8-bit z: 335 us so, 236 us with the choice made once for 32 elements).
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if (ACT == DLION_ACT_RELU) return z < 0.0f ? 0.0f : z;  // NaN stays
    if (ACT == DLION_ACT_SILU) return z * logistic(z);
    if (ACT == DLION_ACT_GELU) {
        const float c = gelu_arg(z);
        return z * logistic(kGelu2c * c * __fmaf_rn(0.044715f * c, c, 1.0f));
    }
    return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if (ACT == DLION_ACT_RELU) return z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
    if (ACT == DLION_ACT_SILU) {
        const float p = logistic(z);
        const float c = fabsf(z) > 128.0f ? copysignf(128.0f, z) : z;   // p (1 - p) is 0 there
        return __fmaf_rn(c * p, 1.0f - p, p);
    }
    if (ACT == DLION_ACT_GELU) {
        const float c = gelu_arg(z), c2 = c * c;
        const float p = logistic(kGelu2c * c * __fmaf_rn(0.044715f, c2, 1.0f));
        return __fmaf_rn(c * kGelu2c * __fmaf_rn(0.134145f, c2, 1.0f), p * (1.0f - p), p);
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
// amax_bits: largest |v| of the block as its bit pattern (so that NaN and infinity order last).
__device__ __forceinline__ uint32_t block_exponent(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return 255u;
    // 127 = 1.984375 * 2^6: the power of two is 2^(E-6), or 2^(E-5) when the fraction is above that
    const int e = static_cast<int>(amax_bits >> 23) - 6 + ((amax_bits & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    return static_cast<uint32_t>(e < 1 ? 1 : e);
}

__device__ __forceinline__ float block_scale(uint32_t e) { return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23); }

// 1 / 2^(e-127), exact (e is in [1, 249] or marks a non-finite block, whose q is 0)
__device__ __forceinline__ float block_inverse(uint32_t e) { return e == 255u ? 0.0f : __uint_as_float((254u - e) << 23); }

__device__ __forceinline__ int quantise8(float v, float inverse) {
    return __float2int_rn(v * inverse);                     // a non-finite v gives NaN * 0 -> 0, or inf * 0 -> 0
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

}  // namespace dlion
