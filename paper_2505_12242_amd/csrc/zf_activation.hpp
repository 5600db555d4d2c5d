// The activations of zf_layer.h and their slopes, in fp32.
#pragma once

#include "zf_device.hpp"
#include "zf_layer.h"

namespace zf {

__device__ __forceinline__ float exp_neg(float x) {  // exp(-x)
  return __builtin_amdgcn_exp2f(x * -1.4426950408889634f);
}

// E = exp(-z^2 / 2) and Phi(z), the normal distribution's integral.  With x = |z|,
// Phi(-x) = E R(x), R(x) = erfcx(x / sqrt 2) / 2 a smooth function: a polynomial
// of degree 7 in t = 1 / (1 + 0.3 x), times t, fitted to least relative error over
// [0, 14] (5e-7 with fp32 coefficients, where E is already 0).  So Phi keeps its
// relative precision in the lower tail, which 1 + erf loses, and the slope's
// exponential is shared.
__device__ __forceinline__ void normal(float z, float& e, float& phi) {
  const float x = fabsf(z);
  e = __builtin_amdgcn_exp2f((z * z) * -0.72134752044448170f);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, x, 1.0f));
  constexpr float c[8] = {0.1196293f, 0.120753966f, 0.09991341f, 0.12856193f,
                            -0.053684246f, 0.2063542f, -0.1572035f, 0.035674877f};
  float p = c[7];
#pragma unroll
  for (int i = 6; i >= 0; --i) p = fmaf(p, t, c[i]);
  const float low = e * (p * t);
  phi = z > 0.0f ? 1.0f - low : low;
}

constexpr float kTanhScale = 0.7978845608028654f;  // sqrt(2 / pi)

// Half of 1 + tanh(u), u = sqrt(2 / pi) (z + 0.044715 z^3).
__device__ __forceinline__ float tanh_phi(float z) {
  const float u = kTanhScale * fmaf(0.044715f * z, z * z, z);
  return __builtin_amdgcn_rcpf(1.0f + exp_neg(2.0f * u));
}

template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == ZF_RELU) return z < 0.0f ? 0.0f : z;  // (a NaN stays one)
  if constexpr (ACT == ZF_GELU) {
    float e, phi;
    normal(z, e, phi);
    return z * phi;
  }
  if constexpr (ACT == ZF_GELU_TANH) return z * tanh_phi(z);
  if constexpr (ACT == ZF_SILU) return z * __builtin_amdgcn_rcpf(1.0f + exp_neg(z));
  return z;
}

template <int ACT>
__device__ __forceinline__ float slope(float z) {
  if constexpr (ACT == ZF_RELU) return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
  if constexpr (ACT == ZF_GELU) {
    float e, phi;
    normal(z, e, phi);
    return fmaf(z * 0.3989422804014327f, e, phi);  // 1 / sqrt(2 pi)
  }
  if constexpr (ACT == ZF_GELU_TANH) {
    const float p = tanh_phi(z), w = p * (1.0f - p);
    // (where w is 0 the other factor may be infinite)
    return w == 0.0f ? p : fmaf(z * w, 2.0f * kTanhScale * fmaf(0.134145f * z, z, 1.0f), p);
  }
  if constexpr (ACT == ZF_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.0f + exp_neg(z));
    return p * fmaf(z, 1.0f - p, 1.0f);
  }
  return 1.0f;
}

// f(integral_constant<activation>).
template <typename F>
auto with_activation(int32_t act, F&& f) {
  switch (act) {
    case ZF_RELU: return f(std::integral_constant<int, ZF_RELU>());
    case ZF_GELU: return f(std::integral_constant<int, ZF_GELU>());
    case ZF_GELU_TANH: return f(std::integral_constant<int, ZF_GELU_TANH>());
    case ZF_SILU: return f(std::integral_constant<int, ZF_SILU>());
    default: return f(std::integral_constant<int, ZF_NONE>());
  }
}

}  // namespace zf
