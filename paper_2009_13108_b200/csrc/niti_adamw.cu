// One AdamW step over many tensors: float32 weights, states in 32 or in 8 bits, and the int8 working copy of the weights.
// Bound: HBM.  A parameter moves 8 bytes of weight, its gradient, its states twice (2 x 8 bytes, or 2 x 2) and a byte of
// working copy; all of a network's tensors share launches, and a tensor list travels with the launch.
#include "niti_float.cuh"
#include <math.h>

namespace {

constexpr int BLOCK = NITI_STATE_BLOCK;            // elements that share the exponent of an 8-bit state: a warp's share
static_assert(BLOCK == 256, "eight elements a lane");
constexpr int WARPS = 8;
constexpr int LIST_SMALL = 16, LIST_MOST = 256;    // tensors a launch takes (its parameters: 1.4 and 22 KB)

struct Tensor {
  float *p;
  const void *g;
  void *m, *v;
  int8_t *s_m, *s_v, *w8;
  const int32_t *s_w;
  long long n;
  float decay;                                     // 1 - lr * weight decay
  short g_type, vec;                               // vec: every pointer allows vectors of eight elements
};
template <int MOST>
struct List {
  int n;
  int first[MOST + 1];                             // first chunk of each tensor
  Tensor t[MOST];
};
struct Hyper {
  float lr, b1, b2, c1, c2, eps;                   // c = 1 - b
  float log_b1, log_b2;
  int blocks;                                      // 256-element blocks of a chunk
};

__device__ __forceinline__ float load_grad(const void *g, int type, long long i) {
  if (type == NITI_F32) return reinterpret_cast<const float *>(g)[i];
  if (type == NITI_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(g)[i]);
  return __half2float(reinterpret_cast<const __half *>(g)[i]);
}

// A scaled magnitude t < 256 as a code of three fraction bits, rounded down, and the 16 bits behind it.  Below 2^-6 codes
// are multiples of 2^-9.
__device__ __forceinline__ void split_e4m3(float t, unsigned &code, unsigned &rest) {
  const unsigned b = __float_as_uint(t);
  const unsigned small = __float2uint_rz(t * 33554432.0f);            // t 2^9 2^16
  const bool normal = b >= (121u << 23);
  code = normal ? (b >> 20) - 960u : small >> 16;
  rest = (normal ? b >> 4 : small) & 0xffffu;
}
__device__ __forceinline__ float root(float x) {                      // (within two steps of 2^-24)
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float value_e4m3(unsigned code) {          // of a code without its sign
  return __uint_as_float(code << 20) * 1.329227995784916e+36f;        // 2^120
}

// 32 random bits for an element of a tensor in a step (multiply and shift mixing, constants of C. Wellons' search for
// 32-bit mixing functions of low bias).
__device__ __forceinline__ unsigned random_bits(unsigned index, unsigned key) {
  unsigned x = index ^ key;
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x = (x ^ (x >> 15)) * 0x846CA68Bu;
  return x ^ (x >> 16);
}

// A warp works on one block of 256 elements at a time, a lane on eight (consecutive ones where the tensor allows vectors,
// else every 32nd).  8-bit states are codes of the first moment and of the root of the second, r = sqrt(v): the root
// halves the range that a code has to span, and it is what the step divides by.  Both round stochastically, since to
// nearest a state that changes by a thousandth a step would never leave its code.  The random bits come from the element's
// index and the step, not from discarded bits as in the integer calls: m mixes a short code and a short gradient with
// weights 9/10 and 1/10, whose binary expansions repeat the same four bits, and without a gradient a code meets the same
// constant, and so the same discarded bits, in every step.  A root that is not zero does not round to zero (the next step
// divides by it).
template <int MOST, bool EIGHT>
__global__ void __launch_bounds__(32 * WARPS)
adamw_kernel(const __grid_constant__ List<MOST> l, const Hyper hy, const int32_t *step, const float *grad_scale, uint32_t *status) {
  niti_enter(step, grad_scale);
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  int lo = 0, hi = l.n;                            // the tensor of this chunk
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.first[mid] <= (int)blockIdx.x) lo = mid; else hi = mid;
  }
  const Tensor &T = l.t[lo];
  const long long chunk = (long long)((int)blockIdx.x - l.first[lo]) * hy.blocks;
  const int t_step = *step;
  if (t_step < 1) {                                // (1 - b^t would be no positive number)
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(status, NITI_DEV_BAD_STEP);
    return;
  }
  const float fstep = (float)t_step, gs = grad_scale ? *grad_scale : 1.0f;
  // 1 - b^t without its cancellation
  const float lr_m = hy.lr / -expm1f(fstep * hy.log_b1), rs_v = rsqrtf(-expm1f(fstep * hy.log_b2));
  const float decay = T.decay;
  const bool with_w8 = T.w8 != nullptr;
  const int s_w = with_w8 ? *T.s_w : 0;
  const float w_scale = niti_pow2(s_w < -126 ? 126 : s_w > 126 ? -126 : -s_w);
  const unsigned key = (unsigned)t_step * 0x9E3779B9u;
  bool bad = false;
  for (int i = warp; i < hy.blocks; i += WARPS) {
    const long long blk = chunk + i, base = blk * BLOCK;
    if (base >= T.n) break;
    const bool vec = T.vec && base + BLOCK <= T.n;
    const long long at = base + (vec ? lane * 8 : lane);
    const int stride = vec ? 1 : 32;
    const int live = vec ? 8 : (int)((T.n - at + 31) / 32 < 0 ? 0 : (T.n - at + 31) / 32 > 8 ? 8 : (T.n - at + 31) / 32);
    float p[8], g[8], m[8], v[8];
    unsigned cm[8], cv[8];
    if (vec) {
      *reinterpret_cast<float4 *>(p) = __ldcs(reinterpret_cast<const float4 *>(T.p + at));
      *reinterpret_cast<float4 *>(p + 4) = __ldcs(reinterpret_cast<const float4 *>(T.p + at) + 1);
      if (T.g_type == NITI_F32) {
        *reinterpret_cast<float4 *>(g) = __ldcs(reinterpret_cast<const float4 *>((const float *)T.g + at));
        *reinterpret_cast<float4 *>(g + 4) = __ldcs(reinterpret_cast<const float4 *>((const float *)T.g + at) + 1);
      } else if (T.g_type == NITI_BF16) {
        Pack<NITI_BF16, 8> k;
        k.load(T.g, at);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = k.get(j);
      } else {
        Pack<NITI_F16, 8> k;
        k.load(T.g, at);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = k.get(j);
      }
      if (EIGHT) {
        const uint2 a = __ldcs(reinterpret_cast<const uint2 *>((const uint8_t *)T.m + at));
        const uint2 b = __ldcs(reinterpret_cast<const uint2 *>((const uint8_t *)T.v + at));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          cm[j] = ((j < 4 ? a.x : a.y) >> (8 * (j & 3))) & 255u;
          cv[j] = ((j < 4 ? b.x : b.y) >> (8 * (j & 3))) & 255u;
        }
      } else {
        *reinterpret_cast<float4 *>(m) = __ldcs(reinterpret_cast<const float4 *>((const float *)T.m + at));
        *reinterpret_cast<float4 *>(m + 4) = __ldcs(reinterpret_cast<const float4 *>((const float *)T.m + at) + 1);
        *reinterpret_cast<float4 *>(v) = __ldcs(reinterpret_cast<const float4 *>((const float *)T.v + at));
        *reinterpret_cast<float4 *>(v + 4) = __ldcs(reinterpret_cast<const float4 *>((const float *)T.v + at) + 1);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const long long e = at + j * stride;
        const bool in = j < live;
        p[j] = in ? T.p[e] : 0.0f;
        g[j] = in ? load_grad(T.g, T.g_type, e) : 0.0f;
        if (EIGHT) {
          cm[j] = in ? ((const uint8_t *)T.m)[e] : 0u;
          cv[j] = in ? ((const uint8_t *)T.v)[e] : 0u;
        } else {
          m[j] = in ? ((const float *)T.m)[e] : 0.0f;
          v[j] = in ? ((const float *)T.v)[e] : 0.0f;
        }
      }
    }
    if (EIGHT) {
      const float k_m = niti_pow2((int)T.s_m[blk]), k_v = niti_pow2((int)T.s_v[blk]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float mm = value_e4m3(cm[j] & 127u) * k_m, r = value_e4m3(cv[j] & 127u) * k_v;
        m[j] = (cm[j] & 128u) ? -mm : mm;
        v[j] = r * r;
      }
    }
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float gj = g[j] * gs;
      const bool ok = fabsf(gj) < __int_as_float(0x7f800000);
      if (ok) {
        m[j] = fmaf(hy.b1, m[j], hy.c1 * gj);
        v[j] = fmaf(hy.b2, v[j], hy.c2 * gj * gj);
      }
      r[j] = root(v[j]);
      if (ok) p[j] = fmaf(p[j], decay, -lr_m * __fdividef(m[j], fmaf(r[j], rs_v, hy.eps)));
      bad |= !ok;
    }
    if (EIGHT) {
      unsigned am = 0, ar = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        am = max(am, __float_as_uint(m[j]) & 0x7fffffffu);
        ar = max(ar, __float_as_uint(r[j]));
      }
      const int e_m = niti_exponent_of(__reduce_max_sync(0xffffffffu, am), 8), e_r = niti_exponent_of(__reduce_max_sync(0xffffffffu, ar), 8);
      const float k_m = niti_pow2(-e_m), k_r = niti_pow2(-e_r);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        unsigned fm, fr;
        split_e4m3(fabsf(m[j]) * k_m, cm[j], fm);
        split_e4m3(r[j] * k_r, cv[j], fr);
        const unsigned x = random_bits((unsigned)(at + j * stride), key);
        cm[j] += (fm + (x >> 16)) >> 16;
        cv[j] += (fr + (x & 0xffffu)) >> 16;
        if (cv[j] == 0u && r[j] > 0.0f) cv[j] = 1u;
        if (m[j] < 0.0f) cm[j] |= 128u;
      }
      if (lane == 0) {
        T.s_m[blk] = (int8_t)e_m;
        T.s_v[blk] = (int8_t)e_r;
      }
    }
    if (vec) {
      reinterpret_cast<float4 *>(T.p + at)[0] = *reinterpret_cast<float4 *>(p);
      reinterpret_cast<float4 *>(T.p + at)[1] = *reinterpret_cast<float4 *>(p + 4);
      if (EIGHT) {
        *reinterpret_cast<uint2 *>((uint8_t *)T.m + at) =
            make_uint2(cm[0] | cm[1] << 8 | cm[2] << 16 | cm[3] << 24, cm[4] | cm[5] << 8 | cm[6] << 16 | cm[7] << 24);
        *reinterpret_cast<uint2 *>((uint8_t *)T.v + at) =
            make_uint2(cv[0] | cv[1] << 8 | cv[2] << 16 | cv[3] << 24, cv[4] | cv[5] << 8 | cv[6] << 16 | cv[7] << 24);
      } else {
        reinterpret_cast<float4 *>((float *)T.m + at)[0] = *reinterpret_cast<float4 *>(m);
        reinterpret_cast<float4 *>((float *)T.m + at)[1] = *reinterpret_cast<float4 *>(m + 4);
        reinterpret_cast<float4 *>((float *)T.v + at)[0] = *reinterpret_cast<float4 *>(v);
        reinterpret_cast<float4 *>((float *)T.v + at)[1] = *reinterpret_cast<float4 *>(v + 4);
      }
      if (with_w8) {
        int q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = niti_payload(p[j], w_scale, NITI_ROUND_NEAREST);
        niti_store_payload<8>(T.w8, at, q);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= live) continue;
        const long long e = at + j * stride;
        T.p[e] = p[j];
        if (EIGHT) {
          ((uint8_t *)T.m)[e] = (uint8_t)cm[j];
          ((uint8_t *)T.v)[e] = (uint8_t)cv[j];
        } else {
          ((float *)T.m)[e] = m[j];
          ((float *)T.v)[e] = v[j];
        }
        if (with_w8) T.w8[e] = (int8_t)niti_payload(p[j], w_scale, NITI_ROUND_NEAREST);
      }
    }
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(status, NITI_DEV_NONFINITE);
}

template <int MOST>
int launch(niti_ctx *ctx, cudaStream_t st, const niti_adamw_tensor *t, int n, bool eight, const Hyper &hyper, double lr, const int32_t *step,
           const float *grad_scale) {
  List<MOST> l;
  Hyper hy = hyper;
  long long total = 0;
  for (int i = 0; i < n; ++i) total += (t[i].n + BLOCK - 1) / BLOCK;
  // a chunk of several blocks a warp shares the set-up between them; with few blocks every warp has one
  hy.blocks = total >= 16LL * WARPS * ctx->sm_count ? 4 * WARPS : WARPS;
  long long chunks = 0;
  l.n = n;
  for (int i = 0; i < n; ++i) {
    const niti_adamw_tensor &a = t[i];
    Tensor &b = l.t[i];
    b.p = a.p; b.g = a.g; b.m = a.m; b.v = a.v;
    b.s_m = a.s_m; b.s_v = a.s_v; b.w8 = a.w8; b.s_w = a.s_w;
    b.n = a.n;
    b.decay = (float)(1.0 - lr * (double)a.weight_decay);
    b.g_type = (short)a.g_type;
    const uintptr_t wide = (uintptr_t)a.p | (uintptr_t)a.g | (eight ? 0 : (uintptr_t)a.m | (uintptr_t)a.v);
    const uintptr_t narrow = (uintptr_t)a.w8 | (eight ? (uintptr_t)a.m | (uintptr_t)a.v : 0);
    b.vec = (wide & 15) == 0 && (narrow & 7) == 0;
    l.first[i] = (int)chunks;
    chunks += ((a.n + BLOCK - 1) / BLOCK + hy.blocks - 1) / hy.blocks;
    if (chunks >= (1LL << 31)) return niti_fail(ctx, NITI_ERR_SHAPE, "niti_adamw: too many elements in one list");
  }
  for (int i = n; i <= MOST; ++i) l.first[i] = (int)chunks;
  if (!chunks) return NITI_OK;
  if (eight)
    NITI_CUDA_TRY(ctx, niti_launch(st, (unsigned)chunks, 32 * WARPS, 0, adamw_kernel<MOST, true>, l, hy, step, grad_scale, ctx->d_status));
  else
    NITI_CUDA_TRY(ctx, niti_launch(st, (unsigned)chunks, 32 * WARPS, 0, adamw_kernel<MOST, false>, l, hy, step, grad_scale, ctx->d_status));
  ctx->launches++;
  return NITI_OK;
}

}  // namespace

extern "C" int niti_adamw(niti_ctx *ctx, void *stream, const niti_adamw_tensor *t, int n, int state_bits, const int32_t *step, double lr,
                          double beta1, double beta2, double eps, const float *grad_scale) {
  if (!ctx) return NITI_ERR_ARG;
  if (n < 0 || (n > 0 && !t) || !step || ((uintptr_t)step & 3) || ((uintptr_t)grad_scale & 3) || (state_bits != 8 && state_bits != 32) ||
      !(lr >= 0.0) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps > 0.0))
    return niti_fail(ctx, NITI_ERR_ARG, "niti_adamw: bad argument");
  const bool eight = state_bits == 8;
  for (int i = 0; i < n; ++i) {
    const niti_adamw_tensor &a = t[i];
    if (a.n < 0 || !niti_type_ok(a.g_type) || !(a.weight_decay >= 0.0f))
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
