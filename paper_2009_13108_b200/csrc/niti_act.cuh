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
// b = -|z|, not below -40 (there the tail is 0: no product with an infinity), NaN for NaN
__device__ __forceinline__ float minus_magnitude(float z) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(-fabsf(z)), "f"(-40.0f));
  return r;
}
// The normal distribution's tail of two values -b >= 0: Q = 1 - Phi(-b) as q g with g = exp(-b^2 / 2).  q = Q exp(b^2 / 2) falls
// slowly: with t = 1 / (1 - c b), q / t is a polynomial in b t, fitted on [0, 14] for the least relative error of Q (degree 8,
// 1.3e-8), or, for the slope, where q stands beside |b| / sqrt(2 pi), of their sum (degree 6, 7e-8); its value at 0 is 1/2.
// Relative to Q the first leaves what reciprocal, exponential and roundings cost, at most 5 2^-22, and the rounding of the
// exponent, b^2 2^-23.7 (measured 2.4e-7 up to 1, 5.4e-7 up to 3, 1.6e-6 up to 6).  Phi of a negative argument is Q itself:
// 1 - (1 - Q) would leave no digits of a small tail.  (A polynomial of degree 5 that only keeps Q's absolute error below 1e-7 took
// 3 us less of the two error passes of 4096 x 4096, degree 8 there 2 us more.)
template <bool SLOPE>
__device__ __forceinline__ F2 normal_tail2(F2 b, F2 &g) {
  float d0, d1, x0, x1;
  fma2(b, F2(SLOPE ? -0.255f : -0.265f), F2(1.0f)).get(d0, d1);
  mul2(mul2(b, F2(-0.72134752f)), b).get(x0, x1);
  const F2 t(fast_reciprocal(d0), fast_reciprocal(d1)), s = mul2(b, t);
  g = F2(fast_exp2(x0), fast_exp2(x1));
  F2 q(0.0f);
  if (SLOPE) {
    q = fma2(s, F2(-2.25122367e-05f), F2(-0.00022684499f));
    q = fma2(s, q, F2(-4.17664523e-06f));
    q = fma2(s, q, F2(0.0112321274f));
    q = fma2(s, q, F2(0.0790442675f));
    q = fma2(s, q, F2(0.271441787f));
  } else {
    q = fma2(s, F2(7.47861634e-07f), F2(9.37091863e-06f));
    q = fma2(s, q, F2(2.45498723e-05f));
    q = fma2(s, q, F2(-0.000147059225f));
    q = fma2(s, q, F2(-0.000331738207f));
    q = fma2(s, q, F2(0.00898367632f));
    q = fma2(s, q, F2(0.0736756772f));
    q = fma2(s, q, F2(0.266442508f));
  }
  q = fma2(s, q, F2(0.5f));
  return mul2(q, t);
}
// z Phi(z) = max(z, 0) - |z| Q(|z|)
__device__ __forceinline__ F2 gelu2(float z0, float z1) {
  const F2 b(minus_magnitude(z0), minus_magnitude(z1));
  F2 g(0.0f);
  const F2 q = normal_tail2<false>(b, g);
  return fma2(b, mul2(q, g), F2(fmaxf(z0, 0.0f), fmaxf(z1, 0.0f)));
}
// Phi(z) + z phi(z): for negative z u = Q(|z|) - |z| phi(z), for others 1 - u
__device__ __forceinline__ F2 gelu_slope2(float z0, float z1) {
  const F2 b(minus_magnitude(z0), minus_magnitude(z1));
  F2 g(0.0f);
  const F2 q = normal_tail2<true>(b, g);
  float u0, u1;
  mul2(fma2(b, F2(0.3989422804f), q), g).get(u0, u1);
  return F2(z0 < 0.0f ? u0 : 1.0f - u0, z1 < 0.0f ? u1 : 1.0f - u1);
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
constexpr float LOG2E_REST = 1.92596299e-08f;              // log2 e less its float32
// Beyond +-150 the sigmoid is 0 or 1; NaN for NaN
__device__ __forceinline__ float at_least_m150(float z) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(z), "f"(-150.0f));
  return r;
}
__device__ __forceinline__ float at_most_150(float z) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(z), "f"(150.0f));
  return r;
}
// Sigmoids of two values between these: 1 / (1 + 2^x) for x = -z log2 e rounded, corrected for what x misses by, of which a multiply-add
// has all but the error of log2 e: s' = -s (1 - s), against a relative error of |z| 2^-24.  Within 2^-21 of themselves.
__device__ __forceinline__ F2 sigmoid2(F2 z) {
  const F2 n = mul2(z, F2(1.44269504f)), miss = fma2(z, F2(-1.44269504f), n);       // -x, and by how much x is too small
  float n0, n1, d0, d1;
  n.get(n0, n1);
  add2(F2(fast_exp2(-n0), fast_exp2(-n1)), F2(1.0f)).get(d0, d1);
  const F2 s(fast_reciprocal(d0), fast_reciprocal(d1));
  return fma2(mul2(s, add2(s, F2(-1.0f))), fma2(z, F2(-LOG2E_REST * 0.69314718f), mul2(miss, F2(0.69314718f))), s);
}
__device__ __forceinline__ F2 silu2(float z0, float z1) {
  const float a0 = at_least_m150(z0), a1 = at_least_m150(z1);
  return mul2(F2(a0, a1), sigmoid2(F2(at_most_150(a0), at_most_150(a1))));
}
// s (1 + z (1 - s))
__device__ __forceinline__ F2 silu_slope2(float z0, float z1) {
  const F2 z(at_most_150(at_least_m150(z0)), at_most_150(at_least_m150(z1))), s = sigmoid2(z);
  return mul2(s, fma2(z, fma2(s, F2(-1.0f), F2(1.0f)), F2(1.0f)));
}
__device__ __forceinline__ float silu(float z) {
  float a, b;
  silu2(z, z).get(a, b);
  return a;
}
__device__ __forceinline__ float silu_slope(float z) {
  float a, b;
  silu_slope2(z, z).get(a, b);
  return a;
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
  } else if constexpr (ACT == NITI_ACT_SILU && N % 2 == 0) {
#pragma unroll
    for (int j = 0; j < N; j += 2) mul2(F2(d[j], d[j + 1]), silu_slope2(z[j], z[j + 1])).get(e[j], e[j + 1]);
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
      for (int j = 0; j + 1 < N; j += 2) silu2(x[j], x[j + 1]).get(x[j], x[j + 1]);
      break;
    default: break;
  }
}
