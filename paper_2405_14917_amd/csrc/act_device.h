// The activations of the 8-bit linear layer and their derivatives, in fp32, to a few units of the last place of their own value (the tail of the
// normal distribution as well: it is a factor, not a difference from one).
#pragma once

#include <type_traits>

#include "slim.h"
#include "slim_device.h"

namespace slimact {

constexpr float LOG2E_HI = 1.44269502f, LOG2E_LO = 1.92596299e-8f, LN2 = 0.693147181f;

// exp(x) for |x| up to some 126: the product with log2(e) in two parts, the second one to first order (v_exp_f32 alone would lose |x| / 2 units)
__device__ __forceinline__ float exp_of(float x) {
  const float h = x * LOG2E_HI, l = fmaf(x, LOG2E_LO, fmaf(x, LOG2E_HI, -h));
  return __builtin_amdgcn_exp2f(h) * fmaf(l, LN2, 1.f);
}
// 1 / (1 + exp(-v)); at the ends 0 and 1.  rest: what is missing to 1 (in the upper half not as a difference: it is multiplied by numbers like v)
__device__ __forceinline__ float sigmoid(float v, float& rest) {
  const float e = exp_of(fminf(fmaxf(-v, -126.f), 126.f)), s = __builtin_amdgcn_rcpf(1.f + e);
  rest = v > 0.f ? e * s : 1.f - s;
  return s;
}
__device__ __forceinline__ float sigmoid(float v) {
  float rest;
  return sigmoid(v, rest);
}

// Phi(-|z|) = exp(-z^2 / 2) P(u) u / 2 with u = 1 / (1 + 0.45 |z| / sqrt 2): P of degree 9 is fitted to exp(x^2) erfc(x) / u by least squares, the
// weights raised where the error was large (relative error 3.2e-8); e: exp(-z^2 / 2), its exponent in two parts
__device__ __forceinline__ float normal_tail(float z, float& e) {
  const float a = fminf(fabsf(z), 40.f), u = __builtin_amdgcn_rcpf(fmaf(a, 0.318198052f, 1.f));
  const float t = a * a, r = fmaf(a, a, -t);
  constexpr float C = -0.721347510f, C_LO = -9.62981495e-9f;             // -log2(e) / 2
  const float h = t * C, l = fmaf(r, C, fmaf(t, C_LO, fmaf(t, C, -h)));
  e = __builtin_amdgcn_exp2f(h) * fmaf(l, LN2, 1.f);
  float p = fmaf(u, -0.0414814778f, 0.191080921f);
  p = fmaf(u, p, -0.30129687f);
  p = fmaf(u, p, 0.143105143f);
  p = fmaf(u, p, -0.0227665345f);
  p = fmaf(u, p, 0.120092193f);
  p = fmaf(u, p, 0.175223584f);
  p = fmaf(u, p, 0.228274714f);
  p = fmaf(u, p, 0.253883015f);
  p = fmaf(u, p, 0.253885323f);
  return 0.5f * u * p * e;
}

// tanh form of gelu: z sigmoid(v(z)), v = 2 sqrt(2 / pi) (z + 0.044715 z^3)
constexpr float TANH_A = 1.59576912f, TANH_B = 0.0713548163f;

__device__ __forceinline__ float activated(float z, int act) {
  switch (act) {
    case SLIM_ACT_RELU: return z < 0.f ? 0.f : z;                        // (NaN stays)
    case SLIM_ACT_GELU: {
      float e;
      const float q = normal_tail(z, e);
      return z * (z > 0.f ? 1.f - q : q);
    }
    case SLIM_ACT_GELU_TANH: return z * sigmoid(z * fmaf(TANH_B, z * z, TANH_A));
    case SLIM_ACT_SILU: return z * sigmoid(z);
    default: return z;
  }
}
__device__ __forceinline__ float slope(float z, int act) {
  switch (act) {
    case SLIM_ACT_RELU: return z > 0.f ? 1.f : z == z ? 0.f : z;
    case SLIM_ACT_GELU: {
      float e;
      const float q = normal_tail(z, e);
      return fmaf(z * 0.398942280f, e, z > 0.f ? 1.f - q : q);
    }
    case SLIM_ACT_GELU_TANH: {
      const float c = fminf(fmaxf(z, -1e4f), 1e4f);
      float rest;
      const float s = sigmoid(c * fmaf(TANH_B, c * c, TANH_A), rest);
      return z == z ? fmaf(c * s * rest, fmaf(3.f * TANH_B, c * c, TANH_A), s) : z;
    }
    case SLIM_ACT_SILU: {
      float rest;
      const float s = sigmoid(z, rest);
      return s * fmaf(z, rest, 1.f);
    }
    default: return 1.f;
  }
}

// f with the activation as a constant: one branch for many values
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  switch (act) {
    case SLIM_ACT_RELU: return f(std::integral_constant<int, SLIM_ACT_RELU>());
    case SLIM_ACT_GELU: return f(std::integral_constant<int, SLIM_ACT_GELU>());
    case SLIM_ACT_GELU_TANH: return f(std::integral_constant<int, SLIM_ACT_GELU_TANH>());
    case SLIM_ACT_SILU: return f(std::integral_constant<int, SLIM_ACT_SILU>());
    default: return f(std::integral_constant<int, SLIM_ACT_NONE>());
  }
}
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int act) {
  if (act == SLIM_ACT_NONE) return;
  with_act(act, [&](auto a) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = activated(v[i], decltype(a)::value);
  });
}

}  // namespace slimact
