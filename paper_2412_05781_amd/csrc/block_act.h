// Activations of the transformer-block operators and their derivatives, in fp32; the rounding of pairs.
#pragma once
#include "block_internal.h"

namespace wino {

// Normal distribution function P(z) = (1 + erf(z / sqrt 2)) / 2 and density p(z).  Two-byte storage: P(-|z|) exp(z^2 / 2) as t q(t) with t = 1 / (1 + 0.295 |z|) and q
// of degree five, fitted (linear program over z in 0 .. 20) for the larger of its error relative to P(-|z|), 8.3e-5, and its absolute error, 1e-7: a sixth of fp16's half
// step at any z, where a formula for erf with an absolute error alone is 3 % off at z = -8.  The exponential is the density's as well: one exponential and one reciprocal
// for both.  fp32 storage: the library's erfcf, whose small values are right relative to themselves, as erff's distance from -1 is not.
__device__ __forceinline__ float normal_tail(float z, float& ex) {                       // P(-|z|), and exp(-z^2 / 2)
    const float t = __builtin_amdgcn_rcpf(fmaf(0.295f, fabsf(z), 1.f));
    ex = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    const float poly = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.08242679f, 0.24603293f), -0.04652035f), 0.15518175f), 0.10953041f), 0.11820197f);
    return t * poly * ex;
}
template <typename E> __device__ __forceinline__ void normal_cdf(float z, float& cdf, float& pdf) {
    if constexpr (sizeof(E) == 4) {
        cdf = 0.5f * erfcf(z * -0.70710678f);
        pdf = 0.39894228f * expf(-0.5f * z * z);
    } else {
        float ex;
        const float tail = normal_tail(z, ex);
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
// the other, as the limit says, where the product would be NaN: c and c' have reached their limits long before 1000.
template <typename E, int ACT> __device__ __forceinline__ void act_both(float z, float& a, float& slope) {
    if constexpr (ACT == ACT_NONE) { a = z; slope = 1.f; return; }
    const float zc = __builtin_amdgcn_fmed3f(z, -1000.f, 1000.f);
    float c, d;
    if constexpr (ACT == ACT_SILU) {
        c = logistic<E>(z);
        d = c * (1.f - c);
    } else if constexpr (ACT == ACT_GELU) {
        normal_cdf<E>(z, c, d);
    } else {                                                        // (1 + tanh t) / 2 = logistic(2t), t = sqrt(2/pi) (z + 0.044715 z^3)
        const float zz = zc * zc;
        c = logistic<E>(1.5957691216f * z * fmaf(0.044715f, zz, 1.f));
        d = c * (1.f - c) * (1.5957691216f * fmaf(0.134145f, zz, 1.f));
    }
    a = fmaxf(z, -1000.f) * c;                                      // (a NaN is one in c)
    slope = fmaf(zc, d, c);
}
template <typename E, int ACT> __device__ __forceinline__ float act_only(float z) {
    float a, s;
    if constexpr (ACT == ACT_GELU && sizeof(E) == 2) {              // z P(z) = max(z, 0) - |z| P(-|z|)
        const float tail = normal_tail(z, s);
        return fmaf(-fminf(fabsf(z), 1000.f), tail, fmaxf(z, 0.f));
    }
    act_both<E, ACT>(z, a, s);
    return a;
}

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
