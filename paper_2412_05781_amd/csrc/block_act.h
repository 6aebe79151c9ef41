// Activations of the transformer-block operators and their derivatives, in fp32; the rounding of pairs.
#pragma once
#include "block_internal.h"

namespace wino {

// Normal distribution function P(z) = (1 + erf(z / sqrt 2)) / 2 and density p(z).  Two-byte storage: erf by formula 7.1.26 of Abramowitz and Stegun,
// Handbook of Mathematical Functions (absolute error 1.5e-7, a 2600th of fp16's half step at 1), whose exponential is the density's as well: one
// exponential and one reciprocal for both.  fp32 storage: the library's erff.
template <typename E> __device__ __forceinline__ void normal_cdf(float z, float& cdf, float& pdf) {
    if constexpr (sizeof(E) == 4) {
        cdf = 0.5f * (1.f + erff(z * 0.70710678f));
        pdf = 0.39894228f * expf(-0.5f * z * z);
    } else {
        const float a = fabsf(z) * 0.70710678f;
        const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, a, 1.f));
        const float ex = __builtin_amdgcn_exp2f(-0.72134752f * z * z);              // exp(-z^2 / 2)
        const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
        const float tail = 0.5f * poly * ex;                                       // P(-|z|)
        cdf = z < 0.f ? tail : 1.f - tail;
        pdf = 0.39894228f * ex;
    }
}

// 1 / (1 + exp(-z))
template <typename E> __device__ __forceinline__ float logistic(float z) {
    if constexpr (sizeof(E) == 4) return 1.f / (1.f + expf(-z));
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z));
}

// Every activation here is z * c(z) with a distribution function c; its derivative is c + z c'.  An infinite z gives 0 at one end and z at
// the other, as the limit says, where the product would be NaN.
template <typename E, int ACT> __device__ __forceinline__ void act_both(float z, float& a, float& slope) {
    if constexpr (ACT == ACT_NONE) { a = z; slope = 1.f; return; }
    float c, d;
    if constexpr (ACT == ACT_SILU) {
        c = logistic<E>(z);
        d = c * (1.f - c);
    } else if constexpr (ACT == ACT_GELU) {
        normal_cdf<E>(z, c, d);
    } else {                                                        // (1 + tanh t) / 2 = logistic(2t), t = sqrt(2/pi) (z + 0.044715 z^3)
        const float zz = z * z;
        c = logistic<E>(1.5957691216f * z * fmaf(0.044715f, zz, 1.f));
        d = c * (1.f - c) * (1.5957691216f * fmaf(0.134145f, zz, 1.f));
    }
    a = c == 0.f ? 0.f : z * c;
    slope = fabsf(z) < 1000.f ? fmaf(z, d, c) : c;
}
template <typename E, int ACT> __device__ __forceinline__ float act_only(float z) { float a, s; act_both<E, ACT>(z, a, s); return a; }

// Two neighbouring elements in one word, rounded to nearest even (one instruction, where two conversions and a merge take four)
template <typename E> __device__ __forceinline__ uint32_t pack_pair(float a, float b) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 v = {a, b};
    if constexpr (std::is_same_v<E, bf16_t>) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    } else {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    }
}

}  // namespace wino
