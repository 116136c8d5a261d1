// Activation functions on float32 and their slopes.
#pragma once
#include "niti_float.cuh"

// 2^s for a sum of exponents (clamped to the float range; the callers report sums outside [-128, 127])
__device__ __forceinline__ float linear_scale(int s) {
  return s >= -126 && s <= 127 ? niti_pow2(s) : s > 127 ? niti_pow2(127) : ldexpf(1.0f, s < -149 ? -149 : s);
}

// (one instruction each, within two steps of 2^-23; 2^x of -inf is 0, 1 / inf is 0)
__device__ __forceinline__ float fast_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float fast_reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Phi of two values, and exp(-z^2 / 2).  For a = |z|: 1 - Phi(a) = t (a1 + t (a2 + ...)) exp(-a^2 / 2) / 2 with t = 1 / (1 + p a /
// sqrt 2), Abramowitz and Stegun 7.1.26 (error of erf at most 1.5e-7, of Phi half of that).  Phi(z) = 1/2 + sign(z) (1/2 - that).
__device__ __forceinline__ F2 normal_cdf2(float z0, float z1, F2 z, F2 &g) {
  float d0, d1, x0, x1;
  fma2(F2(fabsf(z0), fabsf(z1)), F2(0.3275911f * 0.70710678f), F2(1.0f)).get(d0, d1);
  mul2(mul2(z, F2(-0.72134752f)), z).get(x0, x1);
  const F2 t(fast_reciprocal(d0), fast_reciprocal(d1));
  g = F2(fast_exp2(x0), fast_exp2(x1));
  F2 q = fma2(t, F2(-0.5f * 1.061405429f), F2(0.5f * 1.453152027f));
  q = fma2(t, q, F2(-0.5f * 1.421413741f));
  q = fma2(t, q, F2(0.5f * 0.284496736f));
  q = fma2(t, q, F2(-0.5f * 0.254829592f));
  float h0, h1;                                    // 1/2 - tail
  fma2(mul2(q, t), g, F2(0.5f)).get(h0, h1);
  return add2(F2(copysignf(h0, z0), copysignf(h1, z1)), F2(0.5f));
}
__device__ __forceinline__ F2 gelu2(float z0, float z1) {
  const F2 z(z0, z1);
  F2 g(0.0f);
  return mul2(z, normal_cdf2(z0, z1, z, g));
}
__device__ __forceinline__ F2 gelu_slope2(float z0, float z1) {
  const F2 z(z0, z1);
  F2 g(0.0f);
  const F2 cdf = normal_cdf2(z0, z1, z, g);
  return fma2(mul2(z, F2(0.3989422804f)), g, cdf);
}
__device__ __forceinline__ float gelu(float z) {
  float a, b;
  gelu2(z, z).get(a, b);
  return a;
}
__device__ __forceinline__ float gelu_slope(float z) {
  float a, b;
  gelu_slope2(z, z).get(a, b);
  return a;
}
__device__ __forceinline__ float sigmoid(float z) { return fast_reciprocal(1.0f + fast_exp2(z * -1.44269504f)); }
__device__ __forceinline__ float silu(float z) { return z * sigmoid(z); }
__device__ __forceinline__ float silu_slope(float z) {
  const float s = sigmoid(z);
  return s * fmaf(z, 1.0f - s, 1.0f);
}
__device__ __forceinline__ float act_one(float z, int act) {
  switch (act) {
    case NITI_ACT_RELU: return z < 0.0f ? 0.0f : z;
    case NITI_ACT_GELU: return gelu(z);
    case NITI_ACT_SILU: return silu(z);
    default: return z;
  }
}
__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case NITI_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case NITI_ACT_GELU: return gelu_slope(z);
    case NITI_ACT_SILU: return silu_slope(z);
    default: return 1.0f;
  }
}
// e = d act'(z) for a vector
template <int ACT, int N>
__device__ __forceinline__ void act_backward(const float (&d)[N], const float (&z)[N], float (&e)[N]) {
  if constexpr (ACT == NITI_ACT_GELU && N % 2 == 0) {
#pragma unroll
    for (int j = 0; j < N; j += 2) mul2(F2(d[j], d[j + 1]), gelu_slope2(z[j], z[j + 1])).get(e[j], e[j + 1]);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) e[j] = d[j] * act_slope(z[j], ACT);
  }
}
// (N even)
template <int N>
__device__ __forceinline__ void act_all(float (&x)[N], int act) {
  switch (act) {
    case NITI_ACT_RELU:
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = x[j] < 0.0f ? 0.0f : x[j];
      break;
    case NITI_ACT_GELU:
#pragma unroll
      for (int j = 0; j + 1 < N; j += 2) gelu2(x[j], x[j + 1]).get(x[j], x[j + 1]);
      break;
    case NITI_ACT_SILU:
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = silu(x[j]);
      break;
    default: break;
  }
}
