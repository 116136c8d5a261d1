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
// The normal distribution's tail for a = |z|: 1 - Phi(a) = t (a1 + t (a2 + ...)) exp(-a^2 / 2) / 2 with t = 1 / (1 + p a / sqrt 2),
// Abramowitz and Stegun 7.1.26 (error of erf at most 1.5e-7, of Phi half of that).  g receives exp(-a^2 / 2).
__device__ __forceinline__ float normal_tail(float z, float &g) {
  const float t = fast_reciprocal(fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.0f));
  g = fast_exp2(z * -0.72134752f * z);
  float q = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  q = fmaf(t, q, 0.5f * 1.421413741f);
  q = fmaf(t, q, 0.5f * -0.284496736f);
  q = fmaf(t, q, 0.5f * 0.254829592f);
  return q * t * g;
}
__device__ __forceinline__ float gelu(float z) {
  float g;
  const float tail = normal_tail(z, g);
  return z * (z < 0.0f ? tail : 1.0f - tail);
}
__device__ __forceinline__ float gelu_slope(float z) {
  float g;
  const float tail = normal_tail(z, g);
  return fmaf(z * 0.3989422804f, g, z < 0.0f ? tail : 1.0f - tail);
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
template <int N>
__device__ __forceinline__ void act_all(float (&x)[N], int act) {
  switch (act) {
    case NITI_ACT_RELU:
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = x[j] < 0.0f ? 0.0f : x[j];
      break;
    case NITI_ACT_GELU:
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = gelu(x[j]);
      break;
    case NITI_ACT_SILU:
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = silu(x[j]);
      break;
    default: break;
  }
}
