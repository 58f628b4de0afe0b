// Activations and element types of the layers that offer more than ReLU (matmul.hip, group_norm.hip).
// Device code; include from .hip files only.
#ifndef GPULET_ACT_DEVICE_H
#define GPULET_ACT_DEVICE_H

#include <hip/hip_runtime.h>

#include "gpulet.h"

namespace gpulet {

constexpr float kLog2e = 1.44269504f;

// v / (1 + exp(-s)).  exp overflows to infinity below s = -88, where the quotient is zero.
__device__ __forceinline__ float gate(float v, float s) {
    return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * s));
}

// v * Phi(v), Phi the normal distribution function.  Phi(-a) = exp(-a^2 / 2) g(1 / (1 + 0.3 a)) for a >= 0 with g a
// polynomial without constant term, fitted for the smallest relative error over 0 <= a <= 14.5 (1.7e-7): both tails keep
// their relative accuracy (1.6e-6 of the result at most for |v| < 5, 2.5e-7 |v| anywhere), unlike 1 + erf, and a value costs
// one exponential and one reciprocal.
__device__ __forceinline__ float gelu(float v) {
    const float a = __builtin_fabsf(v);
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3f * a);
    float g = 0.0354237035f;
    g = g * t - 0.156158313f;
    g = g * t + 0.204556569f;
    g = g * t - 0.052033823f;
    g = g * t + 0.127691671f;
    g = g * t + 0.100175977f;
    g = g * t + 0.120712131f;
    g = g * t + 0.119632006f;
    const float q = g * t * __builtin_amdgcn_exp2f(-0.5f * kLog2e * (a * a));
    return v * (v > 0.f ? 1.f - q : q);
}

// The activations are three pieces of code.  Kernels take the piece as a template argument: one that holds all three starts
// later, since every line of its code comes from memory once.
//   LINEAR  none, relu: v below 0 becomes 0 (NaN stays), or nothing does
//   GATE    silu, gelu_tanh: v / (1 + exp(-s)) with s = v, or, as (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)),
//           s = 2 sqrt(2 / pi) (v + 0.044715 v^3)
//   NORMAL  gelu
//   SILU    silu alone, four operations shorter than GATE, for kernels that the vector units bound
enum class ActCode { LINEAR, GATE, NORMAL, SILU };
inline ActCode act_code(int act) {
    return act == GPULET_ACT_GELU ? ActCode::NORMAL : act >= GPULET_ACT_SILU ? ActCode::GATE : ActCode::LINEAR;
}

// In place, on N values; `act` is one of the piece's and the same for the whole wavefront.
template <ActCode A, int N>
__device__ __forceinline__ void activate(float (&v)[N], int act) {
    if constexpr (A == ActCode::NORMAL) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = gelu(v[i]);
    } else if constexpr (A == ActCode::SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = gate(v[i], v[i]);
    } else if constexpr (A == ActCode::GATE) {
        const float k1 = act == GPULET_ACT_SILU ? 1.f : 1.59576912f, k3 = act == GPULET_ACT_SILU ? 0.f : 1.59576912f * 0.044715f;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = gate(v[i], v[i] * (k1 + k3 * __builtin_fminf(v[i] * v[i], 1e30f)));   // 0 * inf is no number
    } else {
        const float lo = act == GPULET_ACT_RELU ? 0.f : -__builtin_inff();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < lo ? 0.f : v[i];
    }
}

}  // namespace gpulet
#endif  // GPULET_ACT_DEVICE_H
