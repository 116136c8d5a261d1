// One AdamW step over many tensors: float32 weights, states in 32 or in 8 bits, and the int8 working copy of the weights.
// Bound: HBM.  A parameter moves 8 bytes of weight, its gradient, its states twice (2 x 8 bytes, or 2 x 2) and a byte of
// working copy; all of a network's tensors share launches, and a tensor list travels with the launch.
#include "niti_float.cuh"
#include "niti_tcgen05.cuh"
#include <math.h>

namespace {

constexpr int BLOCK = NITI_STATE_BLOCK;            // elements that share the exponent of an 8-bit state: a warp's share
static_assert(BLOCK == 256, "eight elements a lane");
constexpr int WARPS = 8;
constexpr int CHUNK = WARPS * BLOCK;               // elements that a CTA works on at a time
constexpr int STAGES = 2;
constexpr int GROUP = 4;                           // chunks that a CTA takes in a row where there are many
// bytes of a chunk in shared memory: weights, gradients (room for 32 bits), both states
__host__ __device__ constexpr int stage_bytes(bool eight) { return CHUNK * (4 + 4 + (eight ? 2 : 8)); }
__host__ __device__ constexpr int ctas_per_sm(bool eight) { return eight ? 4 : 3; }
constexpr float TOO_LARGE = 9.223372036854775808e18f;   // 2^63: the square of a smaller gradient is finite, and so is every state
constexpr int LIST_SMALL = 16, LIST_MOST = 256;    // tensors a launch takes (its parameters: 1.4 and 22 KB)

struct Tensor {
  float *p;
  const void *g;
  void *m, *v;
  int8_t *s_m, *s_v, *w8;
  const int32_t *s_w;
  long long n;
  float decay;                                     // 1 - lr * weight decay
  short g_type, vec;                               // vec: whole chunks may be copied to shared memory in bulk
};
template <int MOST>
struct List {
  int n;
  int first[MOST + 1];                             // first group of each tensor, all tensors' groups counted through
  Tensor t[MOST];
};
struct Hyper {
  float lr, b1, b2, c1, c2, eps;                   // c = 1 - b
  float log_b1, log_b2;
  int group;                                       // chunks of a group
};

__device__ __forceinline__ float load_grad(const void *g, int type, long long i) {
  if (type == NITI_F32) return reinterpret_cast<const float *>(g)[i];
  if (type == NITI_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(g)[i]);
  return __half2float(reinterpret_cast<const __half *>(g)[i]);
}

__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Roots of two values: the hardware's approximation r and a step of Heron's method, r + (v - r^2) / (2 r), whose residual a fused
// multiply-add has exactly as long as r^2 has no bits below 2^-149.  The step squares a relative error of 2^-22, so that what is
// left decides the rounding only within 2^-20 of a step of a tie: as __fsqrt_rn() (compared by the tests), in half of its
// instructions.  0 stays 0.  For values of 0 and from SMALL_V on: below it the residual loses bits, and below 2^-126 the
// approximation is 0.
constexpr float SMALL_V = 7.888609052210118e-31f;  // 2^-100
__device__ __forceinline__ F2 root2(float v0, float v1, F2 v) {
  float r0, r1;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(v0));
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(v1));
  const F2 r(r0, r1), d = fma2(F2(-r0, -r1), r, v);
  return fma2(d, F2(0.5f * reciprocal(fmaxf(r0, 1e-30f)), 0.5f * reciprocal(fmaxf(r1, 1e-30f))), r);
}
// The same for any values, small ones times 2^80 beforehand (exact, and so is the root's way back: it is at least 2^-75).
__device__ __forceinline__ F2 root2_scaled(float v0, float v1) {
  const bool s0 = v0 < SMALL_V, s1 = v1 < SMALL_V;
  const float w0 = s0 ? v0 * 1.2089258196146292e24f : v0, w1 = s1 ? v1 * 1.2089258196146292e24f : v1;
  return mul2(root2(w0, w1, F2(w0, w1)), F2(s0 ? 9.094947017729282e-13f : 1.0f, s1 ? 9.094947017729282e-13f : 1.0f));
}
// In bits 20 .. 27, the code below a magnitude t < 256, given as t 2^-24, plus what 16 random bits (times 16: `sixteen` is 16
// in a register, which keeps the multiply-add from becoming a shift and an addition on the busier integer pipe) carry into it.
// The last four bits of a float's exponent and its first three fraction bits are the code: exponent fields of codes 8 .. 120
// (2^-6 .. 2^8) end in 00001 .. 01111 after the multiplication by 2^-24.  SMALL: below 2^-6, where codes are multiples of
// 2^-9, adding 2^-6 puts the number into a binade with that spacing, eight codes too high.
constexpr float LEAST_NORMAL = 9.313225746154785e-10f;                  // 2^-6 2^-24
constexpr float LEAST_CODE = 1.1641532182693481e-10f;                   // 2^-9 2^-24
template <bool SMALL>
__device__ __forceinline__ unsigned draw_e4m3(float t, unsigned draw, unsigned sixteen) {
  unsigned b = __float_as_uint(t);
  if (SMALL && t < LEAST_NORMAL) b = __float_as_uint(__fadd_rz(t, LEAST_NORMAL)) - (8u << 20);
  return draw * sixteen + b;
}
// The codes of four such words in one
__device__ __forceinline__ unsigned pack_codes(unsigned a, unsigned b, unsigned c, unsigned d) {
  return __byte_perm(__byte_perm(a, b, 0x7632) >> 4, __byte_perm(c, d, 0x7632) >> 4, 0x6420);
}
// Values of the four codes in a word (the conversion to half precision is exact: 2^-9 .. 448)
__device__ __forceinline__ void values_e4m3(unsigned w, float (&v)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    unsigned p;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(p) : "h"((unsigned short)(h ? w >> 16 : w & 0xffffu)));
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&p));
    v[2 * h] = f.x;
    v[2 * h + 1] = f.y;
  }
}
// 32 random bits for an element of a tensor in a step (multiply and shift mixing, constants of C. Wellons' search for
// 32-bit mixing functions of low bias).
__device__ __forceinline__ unsigned random_bits(unsigned index, unsigned key) {
  unsigned x = index ^ key;
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x = (x ^ (x >> 15)) * 0x846CA68Bu;
  return x ^ (x >> 16);
}

struct Step {                                      // of this step and tensor
  float den_r, den_1;                              // the step is m / (r den_r + den_1)
  float decay, gs, w_scale;
  unsigned key, sixteen;
  bool scaled;                                     // gs is not simply 1
};

// A warp works on one block of 256 elements at a time, a lane on eight (two vectors of four, or every 32nd element).  8-bit
// states are codes of the first moment and of the root of the second, r = sqrt(v): the root halves the range that a code has to
// span, and it is what the step divides by.  Both round stochastically, since to nearest a state that changes by a thousandth a
// step would never leave its code.  The random bits come from the element's index and the step, not from discarded bits as in
// the integer calls: m mixes a short code and a short gradient with weights 9/10 and 1/10, whose binary expansions repeat the
// same four bits, and without a gradient a code meets the same constant, and so the same discarded bits, in every step.  A root
// that is not zero does not round to zero (the next step divides by it).  s_m, s_v: the block's exponents, before and after.
// Returns whether a gradient was not finite, or too large, or a weight is not finite now.
// VEC: the operands are in shared memory at `stage` (the barrier `empty` is told when they have been read), else everything
// goes by elements.
template <bool EIGHT, bool VEC>
__device__ __forceinline__ bool adamw_block(const Tensor &T, const Hyper &hy, const Step &st, long long blk, int warp, int lane, int &s_m, int &s_v,
                                            const char *stage, unsigned empty) {
  const long long base = blk * BLOCK, at = base + (VEC ? 4 * lane : lane);
  const int live = VEC ? 8 : (int)min(max((T.n - at + 31) / 32, 0LL), 8LL);
  auto offset = [](int j) { return VEC ? (j & 3) + (j >> 2) * 128 : 32 * j; };      // of the lane's j-th element
  float p[8], g[8], m[8], v[8], r[8];
  unsigned cm[2], cv[2];                           // the codes, four a word
  if constexpr (VEC) {
    const char *sp = stage + warp * BLOCK * 4, *sg = stage + CHUNK * 4 + warp * BLOCK * (T.g_type == NITI_F32 ? 4 : 2);
    const char *sm = stage + CHUNK * 8 + warp * BLOCK * (EIGHT ? 1 : 4), *sv = sm + CHUNK * (EIGHT ? 1 : 4);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = 32 * h + lane;
      *reinterpret_cast<float4 *>(p + 4 * h) = reinterpret_cast<const float4 *>(sp)[i];
      if (EIGHT) {
        cm[h] = reinterpret_cast<const unsigned *>(sm)[i];
        cv[h] = reinterpret_cast<const unsigned *>(sv)[i];
      } else {
        *reinterpret_cast<float4 *>(m + 4 * h) = reinterpret_cast<const float4 *>(sm)[i];
        *reinterpret_cast<float4 *>(v + 4 * h) = reinterpret_cast<const float4 *>(sv)[i];
      }
      if (T.g_type == NITI_F32) {
        *reinterpret_cast<float4 *>(g + 4 * h) = reinterpret_cast<const float4 *>(sg)[i];
      } else {
        const uint2 w = reinterpret_cast<const uint2 *>(sg)[i];
        if (T.g_type == NITI_BF16) {
          g[4 * h] = __uint_as_float(w.x << 16); g[4 * h + 1] = __uint_as_float(w.x & 0xffff0000u);
          g[4 * h + 2] = __uint_as_float(w.y << 16); g[4 * h + 3] = __uint_as_float(w.y & 0xffff0000u);
        } else {
          const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&w.x)), b = __half22float2(*reinterpret_cast<const __half2 *>(&w.y));
          g[4 * h] = a.x; g[4 * h + 1] = a.y; g[4 * h + 2] = b.x; g[4 * h + 3] = b.y;
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty);
  } else {
    cm[0] = cm[1] = cv[0] = cv[1] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const long long e = at + offset(j);
      const bool in = j < live;
      p[j] = in ? T.p[e] : 0.0f;
      g[j] = in ? load_grad(T.g, T.g_type, e) : 0.0f;
      if (EIGHT) {
        if (in) {
          cm[j >> 2] |= (unsigned)((const uint8_t *)T.m)[e] << (8 * (j & 3));
          cv[j >> 2] |= (unsigned)((const uint8_t *)T.v)[e] << (8 * (j & 3));
        }
      } else {
        m[j] = in ? ((const float *)T.m)[e] : 0.0f;
        v[j] = in ? ((const float *)T.v)[e] : 0.0f;
      }
    }
  }
  if (EIGHT) {
    const float k_m = niti_pow2(s_m), k_v = niti_pow2(s_v);
    values_e4m3(cm[0], *reinterpret_cast<float (*)[4]>(m));
    values_e4m3(cm[1], *reinterpret_cast<float (*)[4]>(m + 4));
    values_e4m3(cv[0], *reinterpret_cast<float (*)[4]>(v));
    values_e4m3(cv[1], *reinterpret_cast<float (*)[4]>(v + 4));
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      mul2(F2(m[j], m[j + 1]), F2(k_m)).get(m[j], m[j + 1]);
      const F2 t = mul2(F2(v[j], v[j + 1]), F2(k_v));
      mul2(t, t).get(v[j], v[j + 1]);
    }
  }
  if (st.scaled) {
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] *= st.gs;
  }
  float worst = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) worst = niti_absmax(worst, g[j]);
  const bool bad = !(worst < TOO_LARGE);
  // The states are products and sums rounded one by one, without fused multiply-adds, and a correctly rounded root: a code
  // follows from them alone, and so from the formulas, whatever computes them.  (By single instructions: the assembler fuses
  // packed multiplications and additions.)
  auto update = [&](int j) {
    m[j] = __fadd_rn(__fmul_rn(hy.b1, m[j]), __fmul_rn(hy.c1, g[j]));
    v[j] = __fadd_rn(__fmul_rn(hy.b2, v[j]), __fmul_rn(__fmul_rn(hy.c2, g[j]), g[j]));
  };
  if (!bad) {
    float least = TOO_LARGE;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      update(j);
      least = fminf(least, v[j]);
    }
    if (least < SMALL_V) {                         // (zeros, too; rare in a network that learns)
#pragma unroll
      for (int j = 0; j < 8; j += 2) root2_scaled(v[j], v[j + 1]).get(r[j], r[j + 1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; j += 2) root2(v[j], v[j + 1], F2(v[j], v[j + 1])).get(r[j], r[j + 1]);
    }
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const F2 mm(m[j], m[j + 1]), rr(r[j], r[j + 1]);
      float d0, d1;
      fma2(rr, F2(st.den_r), F2(st.den_1)).get(d0, d1);
      fma2(mm, F2(reciprocal(d0), reciprocal(d1)), mul2(F2(p[j], p[j + 1]), F2(st.decay))).get(p[j], p[j + 1]);
    }
  } else {                                         // (elements without a usable gradient keep what they have)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool ok = fabsf(g[j]) < TOO_LARGE;
      if (ok) update(j);
      r[j] = __fsqrt_rn(v[j]);
      if (ok) p[j] = fmaf(m[j], reciprocal(fmaf(r[j], st.den_r, st.den_1)), p[j] * st.decay);
    }
  }
  float top = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = niti_absmax(top, p[j]);
  if (EIGHT) {
    float am = 0.0f, ar = 0.0f, lm = fabsf(m[0]), lr = r[0];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      am = fmaxf(am, fabsf(m[j]));
      ar = fmaxf(ar, r[j]);
      lm = fminf(lm, fabsf(m[j]));
      lr = fminf(lr, r[j]);
    }
    const int e_m = niti_exponent_of(__reduce_max_sync(0xffffffffu, __float_as_uint(am)), 8);
    const int e_r = niti_exponent_of(__reduce_max_sync(0xffffffffu, __float_as_uint(ar)), 8);
    const float q_m = niti_pow2(-e_m - 24), q_r = niti_pow2(-e_r - 24);
    unsigned qm[8], qr[8];
    // (few blocks hold a value below 2^-13 of their largest)
    if (__any_sync(0xffffffffu, lm * q_m < LEAST_NORMAL || lr * q_r < LEAST_NORMAL)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned x = random_bits((unsigned)at + (unsigned)offset(j), st.key);
        qm[j] = draw_e4m3<true>(fabsf(m[j]) * q_m, x >> 16, st.sixteen);
        // (at least the smallest code unless r is 0)
        qr[j] = draw_e4m3<true>(r[j] > 0.0f ? fmaxf(r[j] * q_r, LEAST_CODE) : 0.0f, x & 0xffffu, st.sixteen);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned x = random_bits((unsigned)at + (unsigned)offset(j), st.key);
        qm[j] = draw_e4m3<false>(fabsf(m[j]) * q_m, x >> 16, st.sixteen);
        qr[j] = draw_e4m3<false>(r[j] * q_r, x & 0xffffu, st.sixteen);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      unsigned s01, s23;                           // sign bytes of the moments
      asm("prmt.b32 %0, %1, %2, 0x00fb;" : "=r"(s01) : "r"(__float_as_uint(m[4 * h])), "r"(__float_as_uint(m[4 * h + 1])));
      asm("prmt.b32 %0, %1, %2, 0x00fb;" : "=r"(s23) : "r"(__float_as_uint(m[4 * h + 2])), "r"(__float_as_uint(m[4 * h + 3])));
      cm[h] = pack_codes(qm[4 * h], qm[4 * h + 1], qm[4 * h + 2], qm[4 * h + 3]) | (__byte_perm(s01, s23, 0x5410) & 0x80808080u);
      cv[h] = pack_codes(qr[4 * h], qr[4 * h + 1], qr[4 * h + 2], qr[4 * h + 3]);
    }
    s_m = e_m;
    s_v = e_r;
  }
  if constexpr (VEC) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const long long e = at + 128 * h;
      *reinterpret_cast<float4 *>(T.p + e) = *reinterpret_cast<float4 *>(p + 4 * h);
      if (EIGHT) {
        *reinterpret_cast<unsigned *>((uint8_t *)T.m + e) = cm[h];
        *reinterpret_cast<unsigned *>((uint8_t *)T.v + e) = cv[h];
      } else {
        *reinterpret_cast<float4 *>((float *)T.m + e) = *reinterpret_cast<float4 *>(m + 4 * h);
        *reinterpret_cast<float4 *>((float *)T.v + e) = *reinterpret_cast<float4 *>(v + 4 * h);
      }
      if (T.w8) *reinterpret_cast<unsigned *>(T.w8 + e) = niti_payload4<false>(p[4 * h], p[4 * h + 1], p[4 * h + 2], p[4 * h + 3], st.w_scale);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= live) continue;
      const long long e = at + offset(j);
      T.p[e] = p[j];
      if (EIGHT) {
        ((uint8_t *)T.m)[e] = (uint8_t)(cm[j >> 2] >> (8 * (j & 3)));
        ((uint8_t *)T.v)[e] = (uint8_t)(cv[j >> 2] >> (8 * (j & 3)));
      } else {
        ((float *)T.m)[e] = m[j];
        ((float *)T.v)[e] = v[j];
      }
      if (T.w8) T.w8[e] = (int8_t)niti_payload<false>(p[j], st.w_scale);
    }
  }
  return bad || !(top < __int_as_float(0x7f800000));
}

__device__ __forceinline__ void bulk_load(unsigned dst, const void *src, unsigned bytes, unsigned bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Persistent: a CTA takes every n-th group of chunks, finds the step's constants once, and a warp of its own keeps the next
// chunks' operands on their way into shared memory.  A group's block exponents are collected there, too, and stored by the warp
// that comes last (32 bytes at once: one byte a warp and block took 60 us of 138 million weights' 418).
template <int MOST, bool EIGHT>
__global__ void __launch_bounds__(32 * WARPS + 32, ctas_per_sm(EIGHT))
adamw_kernel(const __grid_constant__ List<MOST> l, const Hyper hy, const int32_t *step, const float *grad_scale, uint32_t *status) {
  extern __shared__ __align__(128) char smem[];
  __shared__ __align__(8) unsigned long long bars[2 * STAGES];            // a stage is full, and has been read by all warps
  __shared__ volatile int abort_flag;
  // exponents of both states for the groups with chunks that are copied in bulk, in turn: a warp that begins the (k + STAGES +
  // 1)th of those chunks waits until all have read the (k + 1)th, and so are done with the kth (other chunks make no warp wait,
  // and so take no turn)
  __shared__ int8_t exps[STAGES + 1][2][GROUP * WARPS];
  __shared__ int arrived[STAGES + 1];
  if (threadIdx.x <= STAGES) arrived[threadIdx.x] = 0;
  if (threadIdx.x < 2 * STAGES) {
    mbar_init(smem_u32(&bars[threadIdx.x]), threadIdx.x < STAGES ? 1 : WARPS);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (threadIdx.x == 0) abort_flag = 0;
  __syncthreads();
  niti_enter(step, grad_scale);
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = (int)threadIdx.x & 31;
  const int t_step = *step;
  if (t_step < 1) {                                // (1 - b^t would be no positive number)
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(status, NITI_DEV_BAD_STEP);
    return;
  }
  // (groups are dealt in turn, so that the grid works on neighbouring memory)
  const int begin = (int)blockIdx.x, step_g = (int)gridDim.x, end = l.first[l.n], group = hy.group;
  int lo = 0, hi = l.n;                            // the first group's tensor
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.first[mid] <= begin) lo = mid; else hi = mid;
  }
  // chunks of a group from element `first` on that are copied in bulk
  auto bulk = [&](const Tensor &T, long long first) { return T.vec ? (int)min((T.n - first) / CHUNK, (long long)group) : 0; };
  const unsigned smem0 = smem_u32(smem);
  if (warp == WARPS) {                             // the copying warp (a copy takes its thread about 250 ns: not beside other work)
    int stage = 0;
    unsigned parity = 1u;
    bool ok = true;
    for (int gr = begin; lane == 0 && ok && gr < end; gr += step_g) {
      while (gr >= l.first[lo + 1]) ++lo;
      const Tensor &T = l.t[lo];
      long long first = (long long)(gr - l.first[lo]) * group * CHUNK;
      const unsigned gb = T.g_type == NITI_F32 ? 4 : 2, sb = EIGHT ? 1 : 4;
      for (int left = bulk(T, first); left > 0; --left, first += CHUNK) {
        if (!mbar_wait(smem_u32(&bars[STAGES + stage]), parity, &abort_flag, status)) { ok = false; break; }
        const unsigned bar = smem_u32(&bars[stage]), dst = smem0 + stage * stage_bytes(EIGHT);
        mbar_expect_tx(bar, CHUNK * (4 + gb + 2 * sb));
        bulk_load(dst, T.p + first, CHUNK * 4, bar);
        bulk_load(dst + CHUNK * 4, (const char *)T.g + first * gb, CHUNK * gb, bar);
        bulk_load(dst + CHUNK * 8, (const char *)T.m + first * sb, CHUNK * sb, bar);
        bulk_load(dst + CHUNK * (8 + sb), (const char *)T.v + first * sb, CHUNK * sb, bar);
        if (++stage == STAGES) { stage = 0; parity ^= 1u; }
      }
    }
    __syncwarp();
    if (abort_flag) {                              // copies in flight land before the shared memory goes away
      const long long t0 = clock64();
      while (clock64() - t0 < 20000000LL) {
      }
    }
    return;
  }
  Step st;
  // 1 - b^t without its cancellation
  // (with the bounds that the call puts on lr and eps every denominator is finite and not 0, so that an element without a
  // gradient does not become 0 / 0 or 0 times infinity; a learning rate of 0 has infinite ones, whose reciprocals are 0)
  const float lr_t = hy.lr / -expm1f((float)t_step * hy.log_b1), lr = fmaxf(lr_t, 1e-30f);
  st.den_r = -rsqrtf(-expm1f((float)t_step * hy.log_b2)) / lr;
  st.den_1 = lr_t < 1e-30f ? __int_as_float(0xff800000) : -fmaxf(hy.eps / lr, 1e-37f);          // (its reciprocal is finite)
  st.gs = grad_scale ? *grad_scale : 1.0f;
  st.scaled = grad_scale != nullptr;
  st.key = (unsigned)t_step * 0x9E3779B9u;
  st.sixteen = 16u;
  asm volatile("" : "+r"(st.sixteen));
  bool bad = false;
  int stage = 0;
  unsigned parity = 0;
  int next_m = 0, next_v = 0;                      // exponents of the warp's block of chunk `ready` of tensor `known`
  long long ready = -1;
  bool ok = true;
  for (int gr = begin, known = -1, turn = 0; ok && gr < end; gr += step_g) {
    while (gr >= l.first[lo + 1]) ++lo;
    const Tensor &T = l.t[lo];
    if (lo != known) {
      known = lo;
      ready = -1;
      const int s_w = T.w8 ? *T.s_w : 0;
      st.w_scale = s_w >= 127 ? __int_as_float(0x00400000) : niti_pow2(s_w < -127 ? 127 : -s_w);       // (2^-127 is subnormal)
      st.decay = T.decay;
    }
    const long long chunk0 = (long long)(gr - l.first[lo]) * group;
    const int whole = bulk(T, chunk0 * CHUNK);
    for (int j = 0; j < group; ++j) {
      const long long chunk = chunk0 + j, blk = chunk * WARPS + warp;
      if (chunk * CHUNK >= T.n) break;
      int s_m = next_m, s_v = next_v;
      if (EIGHT) {
        if (ready != chunk && blk * BLOCK < T.n) {
          s_m = T.s_m[blk];
          s_v = T.s_v[blk];
        }
        ready = j + 1 < group ? chunk + 1 : chunk + 1 + (long long)(step_g - 1) * group;
        const long long next = ready * WARPS + warp;
        if (next * BLOCK < T.n) {
          next_m = T.s_m[next];
          next_v = T.s_v[next];
        }
      }
      if (j < whole) {
        if (!mbar_wait_warp(smem_u32(&bars[stage]), parity, &abort_flag, status)) { ok = false; break; }
        bad |= adamw_block<EIGHT, true>(T, hy, st, blk, warp, lane, s_m, s_v, smem + stage * stage_bytes(EIGHT), smem_u32(&bars[STAGES + stage]));
        if (++stage == STAGES) { stage = 0; parity ^= 1u; }
        if (EIGHT) {
          int before = 0;
          if (lane == 0) {
            exps[turn][0][j * WARPS + warp] = (int8_t)s_m;
            exps[turn][1][j * WARPS + warp] = (int8_t)s_v;
            __threadfence_block();
            before = atomicAdd(&arrived[turn], 1);
          }
          if (__shfl_sync(0xffffffffu, before, 0) == whole * WARPS - 1) {
            __threadfence_block();
            if (lane < whole * WARPS) {
              T.s_m[chunk0 * WARPS + lane] = *(volatile int8_t *)&exps[turn][0][lane];
              T.s_v[chunk0 * WARPS + lane] = *(volatile int8_t *)&exps[turn][1][lane];
            }
            if (lane == 0) arrived[turn] = 0;
            __threadfence_block();
          }
        }
      } else if (blk * BLOCK < T.n) {
        bad |= adamw_block<EIGHT, false>(T, hy, st, blk, warp, lane, s_m, s_v, nullptr, 0u);
        if (EIGHT && lane == 0) {
          T.s_m[blk] = (int8_t)s_m;
          T.s_v[blk] = (int8_t)s_v;
        }
      }
    }
    if (whole > 0) turn = turn == STAGES ? 0 : turn + 1;
  }
  if (abort_flag) {                                // (as above)
    const long long t0 = clock64();
    while (clock64() - t0 < 20000000LL) {
    }
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(status, NITI_DEV_NONFINITE);
}

template <int MOST>
int launch(niti_ctx *ctx, cudaStream_t st, const niti_adamw_tensor *t, int n, bool eight, Hyper hy, double lr, const int32_t *step,
           const float *grad_scale) {
  List<MOST> l;
  long long chunks = 0, groups = 0;
  for (int i = 0; i < n; ++i) chunks += (t[i].n + CHUNK - 1) / CHUNK;
  const long long most = (long long)ctx->sm_count * ctas_per_sm(eight);
  hy.group = chunks >= 4 * GROUP * most ? GROUP : 1;           // (few chunks: one for every CTA)
  l.n = n;
  for (int i = 0; i < n; ++i) {
    const niti_adamw_tensor &a = t[i];
    Tensor &b = l.t[i];
    b.p = a.p; b.g = a.g; b.m = a.m; b.v = a.v;
    b.s_m = a.s_m; b.s_v = a.s_v; b.w8 = a.w8; b.s_w = a.s_w;
    b.n = a.n;
    b.decay = (float)(1.0 - lr * (double)a.weight_decay);
    b.g_type = (short)a.g_type;
    b.vec = (((uintptr_t)a.p | (uintptr_t)a.g | (uintptr_t)a.m | (uintptr_t)a.v) & 15) == 0 && ((uintptr_t)a.w8 & 3) == 0;
    l.first[i] = (int)groups;
    groups += (a.n + (long long)CHUNK * hy.group - 1) / ((long long)CHUNK * hy.group);
    if (groups >= (1LL << 30)) return niti_fail(ctx, NITI_ERR_SHAPE, "niti_adamw: too many elements in one list");
  }
  for (int i = n; i <= MOST; ++i) l.first[i] = (int)groups;
  if (!groups) return NITI_OK;
  const unsigned grid = (unsigned)(groups < most ? groups : most);
  auto go = [&](auto kernel) -> int {
    // (the device's limit, as for every kernel of the library: see niti_ctx::smem_optin)
    bool &ready = ctx->adamw_ready[(MOST == LIST_MOST ? 2 : 0) + (eight ? 1 : 0)];
    if (!ready) {
      cudaFuncAttributes fa;
      NITI_CUDA_TRY(ctx, cudaFuncGetAttributes(&fa, kernel));
      NITI_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(ctx->smem_optin - fa.sharedSizeBytes)));
      ready = true;
    }
    NITI_CUDA_TRY(ctx, niti_launch(st, grid, 32 * WARPS + 32, (size_t)STAGES * stage_bytes(eight), kernel, l, hy, step, grad_scale, ctx->d_status));
    return NITI_OK;
  };
  const int rc = eight ? go(adamw_kernel<MOST, true>) : go(adamw_kernel<MOST, false>);
  if (rc != NITI_OK) return rc;
  ctx->launches++;
  return NITI_OK;
}

}  // namespace

extern "C" int niti_adamw(niti_ctx *ctx, void *stream, const niti_adamw_tensor *t, int n, int state_bits, const int32_t *step, double lr,
                          double beta1, double beta2, double eps, const float *grad_scale) {
  if (!ctx) return NITI_ERR_ARG;
  if (n < 0 || (n > 0 && !t) || !step || ((uintptr_t)step & 3) || ((uintptr_t)grad_scale & 3) || (state_bits != 8 && state_bits != 32) ||
      !(lr >= 0.0 && lr <= 1e6) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 1e-20 && eps <= 1e6))
    return niti_fail(ctx, NITI_ERR_ARG, "niti_adamw: bad argument");
  const bool eight = state_bits == 8;
  for (int i = 0; i < n; ++i) {
    const niti_adamw_tensor &a = t[i];
    if (a.n < 0 || !niti_type_ok(a.g_type) || !(a.weight_decay >= 0.0f && a.weight_decay <= 1e6f))
      return niti_fail(ctx, NITI_ERR_ARG, "niti_adamw: bad argument (size, gradient type or weight decay of a tensor)");
    if (a.n == 0) continue;
    const uintptr_t words = (uintptr_t)a.p | (uintptr_t)a.s_w | (eight ? 0 : (uintptr_t)a.m | (uintptr_t)a.v);
    if (!a.p || !a.g || !a.m || !a.v || (eight && (!a.s_m || !a.s_v)) || (a.w8 && !a.s_w) || (words & 3) ||
        ((uintptr_t)a.g & (uintptr_t)(niti_type_size(a.g_type) - 1)))
      return niti_fail(ctx, NITI_ERR_ARG, "niti_adamw: bad argument (a pointer of a tensor is missing or not aligned to its type)");
  }
  Hyper hy;
  memset(&hy, 0, sizeof(hy));
  hy.lr = (float)lr;
  hy.b1 = (float)beta1; hy.b2 = (float)beta2;
  hy.c1 = (float)(1.0 - beta1); hy.c2 = (float)(1.0 - beta2);
  hy.eps = (float)eps;
  // (b = 0: 1 - b^t is 1 for every t >= 1)
  hy.log_b1 = beta1 > 0.0 ? (float)log(beta1) : -1e30f;
  hy.log_b2 = beta2 > 0.0 ? (float)log(beta2) : -1e30f;
  for (int i = 0; i < n; i += LIST_MOST) {
    const int k = n - i < LIST_MOST ? n - i : LIST_MOST;
    const int rc = k <= LIST_SMALL ? launch<LIST_SMALL>(ctx, (cudaStream_t)stream, t + i, k, eight, hy, lr, step, grad_scale)
                                   : launch<LIST_MOST>(ctx, (cudaStream_t)stream, t + i, k, eight, hy, lr, step, grad_scale);
    if (rc != NITI_OK) return rc;
  }
  return NITI_OK;
}
