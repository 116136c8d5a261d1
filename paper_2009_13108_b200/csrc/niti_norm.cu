// Root-mean-square norm with the residual's addition and an int8 result, its backward pass, and the conversions between
// float tensors and payloads.  All of these are bound by HBM: a row is read once and stays in registers while its sums are
// taken.
#include "niti_div.h"
#include "niti_float.cuh"
#include "niti_sums.cuh"
#include <type_traits>

namespace {

constexpr int ROW_THREADS = 256;      // threads of a block where a row takes fewer
constexpr int ROW_MOST = 512;         // and at most (a thread keeps up to 32 values of a row and as many gains)
constexpr unsigned INF_BITS = 0x7f800000u;

struct RowShape {
  int M, C;
  int tpr;                            // threads of a row (a multiple of 32)
  int rpb;                            // rows of a block
};

// Sum of `ss` and maximum of `am` over the threads of a row, in a fixed order.  buf: per warp of the block.  One barrier a
// row: consecutive rows use the two halves of `buf` in turn.
__device__ __forceinline__ void row_reduce(float &ss, unsigned &am, int tpr, int warp, int lane, float2 (*buf)[32], int turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  am = __reduce_max_sync(0xffffffffu, am);
  if (tpr == 32) return;
  const int wpr = tpr >> 5, first = warp / wpr * wpr;
  if (lane == 0) buf[turn][warp] = make_float2(ss, __uint_as_float(am));
  __syncthreads();
  const float2 v = lane < wpr ? buf[turn][first + lane] : make_float2(0.0f, 0.0f);
  ss = v.x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  am = __reduce_max_sync(0xffffffffu, __float_as_uint(v.y));
}

// Rounding of a launch: a template parameter where a thread has vectors, looked up where it has single elements.
enum { ROUND_BY_ARGUMENT = 2 };
template <int VEC, int MODE>
__device__ __forceinline__ void store_payload(int8_t *y, long long at, const float (&x)[VEC], float scale, int round_mode) {
  if constexpr (MODE == ROUND_BY_ARGUMENT) {
    if (round_mode == NITI_ROUND_PSR) niti_store_payload<VEC, true>(y, at, x, scale);
    else niti_store_payload<VEC, false>(y, at, x, scale);
  } else {
    niti_store_payload<VEC, MODE == NITI_ROUND_PSR>(y, at, x, scale);
  }
}
// The bits of the largest magnitude of a row, INF_BITS or more where something is not finite: a value, or the squares' sum
// (then r is 0 or NaN, and nothing of the row means anything).
__device__ __forceinline__ unsigned row_top(unsigned am, float ss, float r) {
  return am >= INF_BITS || !(ss < __uint_as_float(INF_BITS)) ? INF_BITS : __float_as_uint(__uint_as_float(am) * r);
}

// r and the factor from payload units usually scale a value in one product.  Where r is large (rows near zero with a tiny eps)
// that factor can leave float32: r is applied first then.  2^11 2^100 2^16 is 2^127.
constexpr float LARGE_R = 2048.0f;

// y = h r gain with h = x + residual, r = 1 / sqrt(mean(h^2) + eps); without NORM y = x.  A thread holds NV vectors of its
// row, and the next row's are on their way while this one's sums are taken.  The maximum that fixes the exponent is taken
// of |h gain| beside the sum of squares, since r only scales it: one reduction a row.
// SHARED: only h, r and the maximum over the tensor; norm_round_kernel follows.
// 8192 x 4096 bfloat16 with a residual: 235 MB in 38 us, 6.2 TB/s (0.96 of the measured copy rate), with 768 threads an SM (a
// fourth block of 256 does not fit the registers and ran a wave of its own: 43 us), 26 instructions an element.
template <int T, int VEC, int NV, bool NORM, bool SHARED, int MODE>
__global__ void __launch_bounds__(ROW_MOST)
norm_rows_kernel(const void *x, const void *res, const float *gain, void *h, int8_t *y, int32_t *s_y, float *rstd,
                 WsHeader *hdr, WsHeader *next, uint32_t *status, RowShape sh, float eps, int round_mode) {
  __shared__ float2 buf[2][32];
  niti_enter(x, res, gain);
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  const int grp = (int)threadIdx.x / sh.tpr, t = (int)threadIdx.x - grp * sh.tpr;
  if (next && blockIdx.x == 0 && warp == 0) niti_zero_header(next, lane);
  float g[NV][VEC];
  Pack<T, VEC> px[NV], pr[NV];
  bool in[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * sh.tpr + t) * VEC;
    in[v] = c < sh.C;
    px[v].zero(); pr[v].zero();
#pragma unroll
    for (int j = 0; j < VEC; ++j) g[v][j] = NORM && in[v] ? gain[c + j] : 1.0f;
  }
  const int step = (int)gridDim.x * sh.rpb;
  auto fetch = [&](int row) {
    const long long at = (long long)row * sh.C + t * VEC;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (in[v] && row < sh.M) {
        px[v].template load<SHARED>(x, at + (long long)v * sh.tpr * VEC);
        if (NORM && res) pr[v].load(res, at + (long long)v * sh.tpr * VEC);
      }
  };
  int row = (int)blockIdx.x * sh.rpb + grp;
  fetch(row);
  unsigned most = 0;
  const float inv_c = 1.0f / (float)sh.C;
  for (int turn = 0, base = (int)blockIdx.x * sh.rpb; base < sh.M; base += step, row += step, turn ^= 1) {
    const bool rok = row < sh.M;
    const long long at = (long long)row * sh.C + t * VEC;
    float hv[NV][VEC];
    float ss = 0.0f, am = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (NORM && res) {                               // (the norm is that of the stored row)
        px[v].add(pr[v]);
        if (in[v] && rok) px[v].store(h, at + (long long)v * sh.tpr * VEC);
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) hv[v][j] = px[v].get(j);
    }
    fetch(row + step < sh.M ? row + step : sh.M);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if (NORM) {
          ss = fmaf(hv[v][j], hv[v][j], ss);
          hv[v][j] *= g[v][j];
        }
        am = niti_absmax(am, hv[v][j]);              // (0 where the thread has no columns)
      }
    unsigned ab = __float_as_uint(am);
    row_reduce(ss, ab, sh.tpr, warp, lane, buf, turn);
    const float r = NORM ? rsqrtf(fmaf(ss, inv_c, eps)) : 1.0f;
    const unsigned top = row_top(ab, ss, r);
    if (t == 0 && rok) {
      if (top >= INF_BITS) atomicOr(status, NITI_DEV_NONFINITE);
      if (NORM && rstd) rstd[row] = r;
    }
    if (SHARED) {
      if (rok) most = max(most, top);
      continue;
    }
    const int s = niti_exponent_of(top);
    const bool large = NORM && r > LARGE_R;
    if (large) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < VEC; ++j) hv[v][j] *= r;
    }
    const float scale = niti_payload_scale((large ? 1.0f : r) * niti_pow2(-s), round_mode);
    if (t == 0 && rok) s_y[row] = s;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (in[v] && rok) store_payload<VEC, MODE>(y, at + (long long)v * sh.tpr * VEC, hv[v], scale, round_mode);
  }
  if (SHARED) {
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0 && most) atomicMax(&hdr->maxabs32, most);
  }
}

// Payload of a whole tensor with the exponent of its maximum, from h (or x) and r.  The rows that norm_rows_kernel read
// last come first: they are still in L2.
template <int T, int VEC, bool NORM, int MODE>
__global__ void __launch_bounds__(ROW_THREADS)
norm_round_kernel(const void *h, const float *gain, const float *rstd, int8_t *y, int32_t *s_y, const WsHeader *hdr, int M, int C,
                  int parts, int round_mode) {
  niti_enter(h, gain, rstd, hdr);
  const int s = niti_exponent_of(hdr->maxabs32);
  const float p2 = niti_pow2(-s);
  if (blockIdx.x == 0 && threadIdx.x == 0) *s_y = s;
  const long long items = (long long)M * parts;
  for (long long it = (long long)gridDim.x - 1 - blockIdx.x; it < items; it += gridDim.x) {
    const int row = M - 1 - (int)(it / parts), part = (int)(it % parts);
    const int c = (part * ROW_THREADS + (int)threadIdx.x) * VEC;
    if (c >= C) continue;
    const float r = NORM ? rstd[row] : 1.0f;
    const bool large = NORM && r > LARGE_R;
    const float scale = niti_payload_scale((large ? 1.0f : r) * p2, round_mode);
    Pack<T, VEC> p;
    p.load(h, (long long)row * C + c);
    float v[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[j] = NORM ? p.get(j) * gain[c + j] : p.get(j);
    if (large) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[j] *= r;
    }
    store_payload<VEC, MODE>(y, (long long)row * C + c, v, scale, round_mode);
  }
}

// The same for aligned tensors whose rows are not whole vectors: vectors run over the tensor as one row, and may hold the end of a
// row and the beginning of the next (C >= VEC).  The elements behind the last vector go to the first block's threads.
template <int T, int VEC, bool NORM>
__global__ void __launch_bounds__(ROW_THREADS)
norm_round_flat_kernel(const void *h, const float *gain, const float *rstd, int8_t *y, int32_t *s_y, const WsHeader *hdr, long long n, int C, Div d_c,
                       int round_mode) {
  niti_enter(h, gain, rstd, hdr);
  const int s = niti_exponent_of(hdr->maxabs32);
  const float scale = niti_payload_scale(niti_pow2(-s), round_mode);
  if (blockIdx.x == 0 && threadIdx.x == 0) *s_y = s;
  const long long items = n / VEC;
  for (long long i = (long long)(gridDim.x - 1 - blockIdx.x) * ROW_THREADS + threadIdx.x; i < items; i += (long long)gridDim.x * ROW_THREADS) {
    Pack<T, VEC> p;
    p.load(h, i * VEC);
    float v[VEC];
    if (NORM) {
      const long long row = d_c.s >= 0 ? (long long)div_by((int)(i * VEC), d_c) : i * VEC / C;
      const int c = (int)(i * VEC - row * C);
      const float r0 = rstd[row], r1 = c + VEC > C ? rstd[row + 1] : 0.0f;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const bool here = c + j < C;
        v[j] = p.get(j) * gain[here ? c + j : c + j - C] * (here ? r0 : r1);
      }
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[j] = p.get(j);
    }
    store_payload<VEC, ROUND_BY_ARGUMENT>(y, i * VEC, v, scale, round_mode);
  }
  const long long at = items * VEC + threadIdx.x;
  if (blockIdx.x == 0 && at < n) {
    Pack<T, 1> p;
    p.load(h, at);
    const long long row = at / C;
    const float v[1] = {NORM ? p.get(0) * gain[at - row * C] * rstd[row] : p.get(0)};
    store_payload<1, ROUND_BY_ARGUMENT>(y, at, v, scale, round_mode);
  }
}

// Rows that are longer than a block's registers: the row is read again (from L2) for the rounding.  2048 x 16384
// float32 with a residual 109 us, 4.0 TB/s; by single elements 123.
template <int T, int VEC, bool NORM, bool SHARED>
__global__ void __launch_bounds__(1024)
norm_wide_kernel(const void *x, const void *res, const float *gain, void *h, int8_t *y, int32_t *s_y, float *rstd,
                 WsHeader *hdr, WsHeader *next, uint32_t *status, int M, int C, float eps, int round_mode) {
  __shared__ float2 buf[2][32];
  niti_enter(x, res, gain);
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  if (next && blockIdx.x == 0 && warp == 0) niti_zero_header(next, lane);
  unsigned most = 0;
  int turn = 0;
  for (int row = (int)blockIdx.x; row < M; row += (int)gridDim.x, turn ^= 1) {
    const long long at = (long long)row * C;
    float ss = 0.0f, am = 0.0f;
#pragma unroll 4
    for (int c = (int)threadIdx.x * VEC; c < C; c += 1024 * VEC) {
      Pack<T, VEC> p;
      p.template load<true>(x, at + c);
      if (NORM && res) {
        Pack<T, VEC> pr;
        pr.load(res, at + c);
        p.add(pr);
        p.store(h, at + c);
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float v = p.get(j);
        if (NORM) ss = fmaf(v, v, ss);
        am = niti_absmax(am, NORM ? v * gain[c + j] : v);
      }
    }
    unsigned ab = __float_as_uint(am);
    row_reduce(ss, ab, 1024, warp, lane, buf, turn);
    const float r = NORM ? rsqrtf(ss / (float)C + eps) : 1.0f;
    const unsigned top = row_top(ab, ss, r);
    if (threadIdx.x == 0) {
      if (top >= INF_BITS) atomicOr(status, NITI_DEV_NONFINITE);
      if (NORM && rstd) rstd[row] = r;
    }
    if (SHARED) {
      most = max(most, top);
      continue;
    }
    const int s = niti_exponent_of(top);
    const bool large = NORM && r > LARGE_R;
    const float scale = niti_payload_scale((large ? 1.0f : r) * niti_pow2(-s), round_mode);
    if (threadIdx.x == 0) s_y[row] = s;
    const void *src = NORM && res ? h : x;            // (each thread reads what it has written itself)
#pragma unroll 2
    for (int c = (int)threadIdx.x * VEC; c < C; c += 1024 * VEC) {
      Pack<T, VEC> p;
      p.load(src, at + c);
      float v[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[j] = NORM ? p.get(j) * gain[c + j] * (large ? r : 1.0f) : p.get(j);
      store_payload<VEC, ROUND_BY_ARGUMENT>(y, at + c, v, scale, round_mode);
    }
  }
  if (SHARED && threadIdx.x == 0 && most) atomicMax(&hdr->maxabs32, most);
}

// Backward: with G = gain dy and c = sum_c(G h) r^3 / C:  dx = dh + r G - c h;  dgain = sum over the rows of dy h r.  The
// columns of a thread are the same in every row, so the gain's gradient stays in its registers; each block leaves its sums
// in `part` and column_sum_kernel adds them up in a fixed order.  8192 x 4096 bfloat16 with dh: 268 MB in 42 us, 6.4 TB/s (0.99
// of the measured copy rate), and 5 us for the sums of 296 blocks.
// At most 16 columns of a thread in 16 bits: with 32 their operands, gains and sums do not fit 128 registers (4096 x 8192 bfloat16
// as 256 threads of 32 columns took 513 us in spilled registers, as 512 of 16 it takes 57).  float32 with 16 columns spills 80
// bytes a thread.
template <int T, int VEC, int NV>
__global__ void __launch_bounds__(ROW_MOST, 1)
norm_bwd_kernel(const void *dy, const void *h, const float *gain, const float *rstd, const void *dh, void *dx, float *part,
                RowShape sh) {
  __shared__ float2 buf[2][32];
  niti_enter(dy, h, gain, rstd, dh);
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  const int grp = (int)threadIdx.x / sh.tpr, t = (int)threadIdx.x - grp * sh.tpr;
  float g[NV][VEC], dg[NV][VEC];
  Pack<T, VEC> py[NV], ph[NV], pd[NV];
  bool in[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * sh.tpr + t) * VEC;
    in[v] = c < sh.C;
    py[v].zero(); ph[v].zero(); pd[v].zero();
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      g[v][j] = in[v] ? gain[c + j] : 0.0f;
      dg[v][j] = 0.0f;
    }
  }
  const int step = (int)gridDim.x * sh.rpb;
  float r_next = 0.0f;
  auto fetch = [&](int row) {
    if (row >= sh.M) return;
    const long long at = (long long)row * sh.C + t * VEC;
    r_next = rstd[row];
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (in[v]) {
        py[v].load(dy, at + (long long)v * sh.tpr * VEC);
        ph[v].load(h, at + (long long)v * sh.tpr * VEC);
        if (dh) pd[v].load(dh, at + (long long)v * sh.tpr * VEC);
      }
  };
  int row = (int)blockIdx.x * sh.rpb + grp;
  fetch(row);
  for (int turn = 0, base = (int)blockIdx.x * sh.rpb; base < sh.M; base += step, row += step, turn ^= 1) {
    const bool rok = row < sh.M;
    const float r = r_next;
    Pack<T, VEC> qy[NV], qh[NV], qd[NV];
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      qy[v] = py[v]; qh[v] = ph[v]; qd[v] = pd[v];
    }
    fetch(row + step);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float y = qy[v].get(j), hh = qh[v].get(j);
        dot = fmaf(y * g[v][j], hh, dot);
        if (rok) dg[v][j] = fmaf(y, hh * r, dg[v][j]);
      }
    unsigned none = 0;
    row_reduce(dot, none, sh.tpr, warp, lane, buf, turn);
    const float c = dot / (float)sh.C * r * r * r;   // (r^3 alone can leave float32)
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float d[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) d[j] = qd[v].get(j) + (r * (qy[v].get(j) * g[v][j]) - c * qh[v].get(j));
      Pack<T, VEC> o;
      o.set(d);
      if (in[v] && rok) o.store(dx, (long long)row * sh.C + (v * sh.tpr + t) * VEC);
    }
  }
  if (!part) return;
  extern __shared__ float sums[];                    // (several rows a block: theirs first)
  float *mine = sh.rpb > 1 ? sums + grp * sh.C : part + (long long)blockIdx.x * sh.C;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (in[v]) mine[(v * sh.tpr + t) * VEC + j] = dg[v][j];
  if (sh.rpb == 1) return;
  __syncthreads();
  for (int c = (int)threadIdx.x; c < sh.C; c += (int)blockDim.x) {
    float sum = sums[c];
    for (int k = 1; k < sh.rpb; ++k) sum += sums[k * sh.C + c];
    part[(long long)blockIdx.x * sh.C + c] = sum;
  }
}

// Backward of rows longer than a block's registers: one block per row reads it twice (the second time from L2) and leaves dy h r
// to be summed by columns in another pass (norm_wide_gain_kernel).  2048 x 16384 float32 144 us, single elements 222.
template <int T, int VEC>
__global__ void __launch_bounds__(1024)
norm_bwd_wide_kernel(const void *dy, const void *h, const float *gain, const float *rstd, const void *dh, void *dx, int M, int C) {
  __shared__ float2 buf[2][32];
  niti_enter(dy, h, gain, rstd, dh);
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  int turn = 0;
  for (int row = (int)blockIdx.x; row < M; row += (int)gridDim.x, turn ^= 1) {
    const long long at = (long long)row * C;
    const float r = rstd[row];
    float dot = 0.0f;
    unsigned none = 0;
    Pack<T, VEC> a, b, d;
    d.zero();
#pragma unroll 4
    for (int c = (int)threadIdx.x * VEC; c < C; c += 1024 * VEC) {
      a.template load<true>(dy, at + c);
      b.template load<true>(h, at + c);
#pragma unroll
      for (int j = 0; j < VEC; ++j) dot = fmaf(a.get(j) * gain[c + j], b.get(j), dot);
    }
    row_reduce(dot, none, 1024, warp, lane, buf, turn);
    const float k = dot / (float)C * r * r * r;
#pragma unroll 2
    for (int c = (int)threadIdx.x * VEC; c < C; c += 1024 * VEC) {
      a.load(dy, at + c);
      b.load(h, at + c);
      if (dh) d.load(dh, at + c);
      float o[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) o[j] = d.get(j) + (r * (a.get(j) * gain[c + j]) - k * b.get(j));
      Pack<T, VEC> po;
      po.set(o);
      po.store(dx, at + c);
    }
  }
}
// Column sums of dy h r over a share of the rows (blockIdx.y), VEC columns a thread; in front of norm_bwd_wide_kernel, which
// may write dx over dy.
template <int T, int VEC>
__global__ void __launch_bounds__(256)
norm_wide_gain_kernel(const void *dy, const void *h, const float *rstd, float *part, int M, int C) {
  niti_enter(dy, h, rstd);
  const int c = (int)(blockIdx.x * 256 + threadIdx.x) * VEC;
  if (c >= C) return;
  float sum[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] = 0.0f;
#pragma unroll 4
  for (int row = (int)blockIdx.y; row < M; row += (int)gridDim.y) {
    Pack<T, VEC> a, b;
    a.load(dy, (long long)row * C + c);
    b.load(h, (long long)row * C + c);
    const float r = rstd[row];
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] = fmaf(a.get(j), b.get(j) * r, sum[j]);
  }
#pragma unroll
  for (int j = 0; j < VEC; ++j) part[(long long)blockIdx.y * C + c + j] = sum[j];
}

template <int W>
__global__ void __launch_bounds__(256 * 4 / W)
column_sum_kernel(const float *part, float *dst, int n, int C) {
  __shared__ float buf[32 * 33];
  niti_enter(part);
  niti_column_sums<W, 32>(part, dst, n, C, (int)blockIdx.x, buf);
}

// 2^e, e clamped to the format's -128 .. 127
__device__ __forceinline__ float exponent_scale(int e) {
  return e >= 127 ? niti_pow2(127) : e >= -126 ? niti_pow2(e) : __int_as_float(e == -127 ? 0x00400000 : 0x00200000);
}
// (an e4m3 code's exponent and fraction, moved into place, are the value over 2^120; exact, the small ones too)
template <bool E4M3>
__device__ __forceinline__ float code_value(unsigned b) {
  if (!E4M3) return (float)(int)(int8_t)b;
  const float v = __uint_as_float((b & 127u) << 20) * 1.329227995784916e+36f;
  return (b & 128u) ? -v : v;
}
// values = payload * 2^s, or the value of an 8-bit code times 2^s; one exponent for every `per` elements (0: one in all).
// WIDE: 16 elements a thread, of at most two exponents (per >= 16), in 32-byte stores (whole sectors: half of one a store took
// 21 us for 8192 x 4096 payloads to bfloat16, this 16); the elements behind the last 16 go to the block behind the others.
template <int T, bool E4M3, typename S, bool WIDE>
__global__ void __launch_bounds__(256)
dequantize_kernel(const uint8_t *q, const S *s, void *out, long long n, Div d_per, long long per, int blocks) {
  niti_enter(q, s);
  typedef typename FloatOf<T>::type FT;
  if (WIDE && (int)blockIdx.x < blocks) {
    const long long items = n / 16, stride = (long long)blocks * 256;
    long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    uint4 ahead = make_uint4(0, 0, 0, 0);            // (the next vector is on its way while this one is converted)
    if (i < items) ahead = __ldcs(reinterpret_cast<const uint4 *>(q) + i);
    for (; i < items; i += stride) {
      const uint4 w4 = ahead;
      if (i + stride < items) ahead = __ldcs(reinterpret_cast<const uint4 *>(q) + i + stride);
      const long long at = i * 16;
      // (indices below 2^31 are divided by multiplication)
      const long long row = per == 0 ? 0 : d_per.s >= 0 ? (long long)div_by((int)at, d_per) : at / per;
      const int split = per == 0 || (row + 1) * per - at > 16 ? 16 : (int)((row + 1) * per - at);
      const float k0 = exponent_scale((int)s[row]), k1 = split < 16 ? exponent_scale((int)s[row + 1]) : k0;
      const unsigned w[4] = {w4.x, w4.y, w4.z, w4.w};
      float v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = code_value<E4M3>((w[j >> 2] >> (8 * (j & 3))) & 255u) * (j < split ? k0 : k1);
      constexpr int PV = 32 / (int)sizeof(FT);
#pragma unroll
      for (int k = 0; k < 16 / PV; ++k) {
        unsigned o[8];
        pack32<T, PV>(v + PV * k, o);
        store32(reinterpret_cast<FT *>(out) + at + PV * k, o);
      }
    }
    return;
  }
  const long long from = WIDE ? n / 16 * 16 : 0, step = WIDE ? 256 : (long long)gridDim.x * 256;
  for (long long at = from + (WIDE ? 0 : (long long)blockIdx.x * 256) + threadIdx.x; at < n; at += step) {
    const float v[1] = {code_value<E4M3>(q[at]) * exponent_scale((int)s[per == 0 ? 0 : at / per])};
    Pack<T, 1> p;
    p.set(v);
    p.store(out, at);
  }
}

inline bool misaligned(const void *a, uintptr_t bytes) { return ((uintptr_t)a & (bytes - 1)) != 0; }

// How a row of C elements is dealt to threads: vectors of 16 bytes where rows and pointers allow them; as few vectors a
// thread as keep a row within ROW_THREADS threads, then within ROW_MOST.
struct RowPlan { int vec, nv; RowShape sh; };
RowPlan plan_rows(int M, int C, int type, bool aligned, int nv_most) {
  RowPlan p;
  const int v16 = 16 / niti_type_size(type);
  p.vec = aligned && C % v16 == 0 ? v16 : 1;
  const int nvec = (C + p.vec - 1) / p.vec;
  p.nv = 0;
  p.sh.M = M; p.sh.C = C; p.sh.tpr = 0; p.sh.rpb = 1;
  for (int limit = ROW_THREADS; limit <= ROW_MOST && !p.nv; limit *= 2)
    for (int nv = 1; nv <= nv_most && !p.nv; nv *= 2)
      if ((nvec + nv - 1) / nv <= limit) p.nv = nv;
  if (!p.nv) return p;                               // (wide rows)
  p.sh.tpr = ((nvec + p.nv - 1) / p.nv + 31) / 32 * 32;
  p.sh.rpb = p.sh.tpr >= ROW_THREADS ? 1 : ROW_THREADS / p.sh.tpr;
  return p;
}

template <typename F>
int with_type(int type, F f) {
  if (type == NITI_F32) return f(std::integral_constant<int, NITI_F32>{});
  if (type == NITI_BF16) return f(std::integral_constant<int, NITI_BF16>{});
  return f(std::integral_constant<int, NITI_F16>{});
}

unsigned row_blocks(const niti_ctx *ctx, const RowShape &sh, int threads, int per_sm_threads) {
  const long long want = ((long long)sh.M + sh.rpb - 1) / sh.rpb;
  const long long cap = (long long)ctx->sm_count * (per_sm_threads / threads > 0 ? per_sm_threads / threads : 1);
  return (unsigned)(want < cap ? want : cap);
}

struct NormCall {
  const void *x, *res;
  const float *gain;
  void *h;
  int8_t *y;
  int32_t *s_y;
  float *rstd;
  int type, M, C, rows, round_mode;
  float eps;
};

template <bool NORM>
int run_norm(niti_ctx *ctx, cudaStream_t st, const NormCall &c, void *ws) {
  const uintptr_t all = (uintptr_t)c.x | (uintptr_t)c.res | (uintptr_t)c.h;
  const bool aligned = (all & 15) == 0 && !misaligned(c.y, 8);
  // (at most 16 columns a thread before 32: 8192 x 5120 bfloat16 66 -> 55 us; float32 as 512 threads of 8, 8192 x 4096 shared 73
  // -> 89.  Single elements: up to 16 a thread)
  RowPlan pl = plan_rows(c.M, c.C, c.type, aligned, c.type == NITI_F32 ? 4 : 2);
  if (!pl.nv) pl = plan_rows(c.M, c.C, c.type, aligned, pl.vec == 1 ? 16 : 4);
  WsHeader *hdr = nullptr, *next = nullptr;
  float *rstd = c.rstd;
  if (!c.rows) {
    hdr = niti_take_header(ctx, st, ws);
    const int rc = niti_clear(ctx, st, nullptr, 0, &next);
    if (rc != NITI_OK) return rc;
    if (NORM && !rstd) rstd = (float *)((char *)ws + NITI_WS_HEADER);
  }
  const int threads = pl.nv ? pl.sh.tpr * pl.sh.rpb : 1024;
  const int rc = with_type(c.type, [&](auto t) -> int {
    constexpr int T = decltype(t)::value;
    constexpr int V16 = 16 / (int)sizeof(typename FloatOf<T>::type);
    auto go = [&](auto shared) -> int {
      constexpr bool SHARED = decltype(shared)::value;
      auto rows_as = [&](auto vec, auto nv, auto mode) -> int {
        NITI_CUDA_TRY(ctx, niti_launch(st, row_blocks(ctx, pl.sh, threads, 768), threads, 0,
                                       norm_rows_kernel<T, decltype(vec)::value, decltype(nv)::value, NORM, SHARED, decltype(mode)::value>, c.x, c.res,
                                       c.gain, c.h, c.y, c.s_y, rstd, hdr, next, ctx->d_status, pl.sh, c.eps, c.round_mode));
        return NITI_OK;
      };
      auto rows = [&](auto vec, auto nv) -> int {
        if constexpr (SHARED || decltype(vec)::value == 1) return rows_as(vec, nv, std::integral_constant<int, ROUND_BY_ARGUMENT>{});
        else if (c.round_mode == NITI_ROUND_PSR) return rows_as(vec, nv, std::integral_constant<int, NITI_ROUND_PSR>{});
        else return rows_as(vec, nv, std::integral_constant<int, NITI_ROUND_NEAREST>{});
      };
      auto pick = [&](auto vec) -> int {
        if (pl.nv == 1) return rows(vec, std::integral_constant<int, 1>{});
        if (pl.nv == 2) return rows(vec, std::integral_constant<int, 2>{});
        if constexpr (decltype(vec)::value == 1) {
          if (pl.nv == 8) return rows(vec, std::integral_constant<int, 8>{});
          if (pl.nv == 16) return rows(vec, std::integral_constant<int, 16>{});
        }
        return rows(vec, std::integral_constant<int, 4>{});
      };
      if (!pl.nv) {
        auto wide = [&](auto vec) -> int {
          NITI_CUDA_TRY(ctx, niti_launch(st, (unsigned)(c.M < 2 * ctx->sm_count ? c.M : 2 * ctx->sm_count), 1024, 0,
                                         norm_wide_kernel<T, decltype(vec)::value, NORM, SHARED>, c.x, c.res, c.gain, c.h, c.y, c.s_y, rstd, hdr, next,
                                         ctx->d_status, c.M, c.C, c.eps, c.round_mode));
          return NITI_OK;
        };
        return pl.vec == 1 ? wide(std::integral_constant<int, 1>{}) : wide(std::integral_constant<int, V16>{});
      }
      return pl.vec == 1 ? pick(std::integral_constant<int, 1>{}) : pick(std::integral_constant<int, V16>{});
    };
    int r = c.rows ? go(std::false_type{}) : go(std::true_type{});
    ctx->launches++;
    if (r != NITI_OK || c.rows) return r;
    niti_header_passed_on(ctx, next);
    const void *src = NORM && c.res ? c.h : c.x;
    auto second_as = [&](auto vec, auto mode) -> int {
      constexpr int VEC = decltype(vec)::value;
      const int parts = (c.C + ROW_THREADS * VEC - 1) / (ROW_THREADS * VEC);
      const long long items = (long long)c.M * parts, cap = 8LL * ctx->sm_count;
      NITI_CUDA_TRY(ctx, niti_launch(st, (unsigned)(items < cap ? items : cap), ROW_THREADS, 0, norm_round_kernel<T, VEC, NORM, decltype(mode)::value>, src,
                                     c.gain, (const float *)rstd, c.y, c.s_y, (const WsHeader *)hdr, c.M, c.C, parts, c.round_mode));
      return NITI_OK;
    };
    auto second = [&](auto vec) -> int {
      if constexpr (decltype(vec)::value == 1) return second_as(vec, std::integral_constant<int, ROUND_BY_ARGUMENT>{});
      else if (c.round_mode == NITI_ROUND_PSR) return second_as(vec, std::integral_constant<int, NITI_ROUND_PSR>{});
      else return second_as(vec, std::integral_constant<int, NITI_ROUND_NEAREST>{});
    };
    if (aligned && c.C % V16 != 0 && c.C >= V16) {   // (8192 x 4095 bfloat16 15 us, by single elements 95)
      const long long n = (long long)c.M * c.C, want = (n / V16 + ROW_THREADS - 1) / ROW_THREADS, cap = 8LL * ctx->sm_count;
      const Div d = n < (1LL << 31) ? make_div(c.C) : Div{0u, -1};
      NITI_CUDA_TRY(ctx, niti_launch(st, (unsigned)(want < cap ? want : cap), ROW_THREADS, 0, norm_round_flat_kernel<T, V16, NORM>, src, c.gain,
                                     (const float *)rstd, c.y, c.s_y, (const WsHeader *)hdr, n, c.C, d, c.round_mode));
      ctx->launches++;
      return NITI_OK;
    }
    r = aligned && c.C % V16 == 0 ? second(std::integral_constant<int, V16>{}) : second(std::integral_constant<int, 1>{});
    ctx->launches++;
    return r;
  });
  return rc;
}

// Blocks of norm_bwd_kernel, whose gain sums the workspace has to hold: at most this many rows of C floats.
constexpr int BWD_PARTS = 320;

}  // namespace

size_t niti_norm_ws_bytes(int op, long long M, long long C) {
  if (op == NITI_OP_RMSNORM_BWD) return NITI_WS_HEADER + ((size_t)BWD_PARTS * 4 * (size_t)C + 255) / 256 * 256;
  return NITI_WS_HEADER + ((size_t)M * 4 + 255) / 256 * 256;
}

static int norm_args(niti_ctx *ctx, const char *name, int type, int M, int C, void *ws, size_t ws_bytes, int op) {
  if (!niti_type_ok(type) || M < 0 || C <= 0) {
    snprintf(ctx->err, sizeof(ctx->err), "%s: bad argument (type, or a size that is not positive)", name);
    return NITI_ERR_ARG;
  }
  if (M > (1 << 30) || C > (1 << 30)) return niti_fail(ctx, NITI_ERR_SHAPE, "more than 2^30 rows or columns");    // (32-bit counters)
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < niti_norm_ws_bytes(op, M, C))
    return niti_fail(ctx, NITI_ERR_WORKSPACE, "workspace missing, misaligned or too small");
  return NITI_OK;
}

// A tensor without rows has the exponent of one of zeros.
static int exponent_of_nothing(niti_ctx *ctx, void *stream, int32_t *s, int row_exponents) {
  if (row_exponents || !s) return NITI_OK;
  if (misaligned(s, 4)) return niti_fail(ctx, NITI_ERR_ARG, "bad argument (pointers are aligned to their type)");
  NITI_CUDA_TRY(ctx, cudaMemsetAsync(s, 0, 4, (cudaStream_t)stream));
  return NITI_OK;
}

extern "C" int niti_rmsnorm_fwd(niti_ctx *ctx, void *stream, const void *x, const void *residual, const float *gain, void *h, int8_t *y,
                                int32_t *s_y, float *rstd, int type, int M, int C, int row_exponents, float eps, int round_mode, void *ws,
                                size_t ws_bytes) {
  if (!ctx) return NITI_ERR_ARG;
  const int rc = norm_args(ctx, "niti_rmsnorm_fwd", type, M, C, ws, ws_bytes, NITI_OP_RMSNORM_FWD);
  if (rc != NITI_OK) return rc;
  if (M == 0) return exponent_of_nothing(ctx, stream, s_y, row_exponents);
  const uintptr_t es = (uintptr_t)niti_type_size(type);
  if (!x || !gain || !y || !s_y || (residual && !h) || !(eps >= 0.0f) || (round_mode != NITI_ROUND_PSR && round_mode != NITI_ROUND_NEAREST) ||
      (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)h) & (es - 1)) || (((uintptr_t)gain | (uintptr_t)s_y | (uintptr_t)rstd) & 3))
    return niti_fail(ctx, NITI_ERR_ARG, "niti_rmsnorm_fwd: bad argument (a residual needs h; pointers are aligned to their type)");
  const NormCall c = {x, residual, gain, residual ? h : nullptr, y, s_y, rstd, type, M, C, row_exponents, round_mode, eps};
  return run_norm<true>(ctx, (cudaStream_t)stream, c, ws);
}

extern "C" int niti_quantize(niti_ctx *ctx, void *stream, const void *x, int8_t *q, int32_t *s, int type, int M, int C, int row_exponents,
                             int round_mode, void *ws, size_t ws_bytes) {
  if (!ctx) return NITI_ERR_ARG;
  const int rc = norm_args(ctx, "niti_quantize", type, M, C, ws, ws_bytes, NITI_OP_QUANTIZE);
  if (rc != NITI_OK) return rc;
  if (M == 0) return exponent_of_nothing(ctx, stream, s, row_exponents);
  if (!x || !q || !s || misaligned(x, (uintptr_t)niti_type_size(type)) || misaligned(s, 4) ||
      (round_mode != NITI_ROUND_PSR && round_mode != NITI_ROUND_NEAREST))
    return niti_fail(ctx, NITI_ERR_ARG, "niti_quantize: bad argument (pointers are aligned to their type)");
  if (round_mode == NITI_ROUND_PSR && type != NITI_F32)
    return niti_fail(ctx, NITI_ERR_ARG, "niti_quantize: 16-bit values have too few discarded bits for pseudo-stochastic rounding");
  const NormCall c = {x, nullptr, nullptr, nullptr, q, s, nullptr, type, M, C, row_exponents, round_mode, 0.0f};
  return run_norm<false>(ctx, (cudaStream_t)stream, c, ws);
}

static int launch_column_sums(niti_ctx *ctx, cudaStream_t st, const float *part, float *dst, int n, int C);

extern "C" int niti_rmsnorm_bwd(niti_ctx *ctx, void *stream, const void *dy, const void *h, const float *gain, const float *rstd, const void *dh,
                                void *dx, float *dgain, int type, int M, int C, void *ws, size_t ws_bytes) {
  if (!ctx) return NITI_ERR_ARG;
  int rc = norm_args(ctx, "niti_rmsnorm_bwd", type, M, C, ws, ws_bytes, NITI_OP_RMSNORM_BWD);
  if (rc != NITI_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (misaligned(dgain, 4)) return niti_fail(ctx, NITI_ERR_ARG, "niti_rmsnorm_bwd: bad argument (pointers are aligned to their type)");
  if (M == 0) {
    if (dgain) NITI_CUDA_TRY(ctx, cudaMemsetAsync(dgain, 0, (size_t)C * 4, st));
    return NITI_OK;
  }
  const uintptr_t es = (uintptr_t)niti_type_size(type);
  if (!dy || !h || !gain || !rstd || !dx || (((uintptr_t)dy | (uintptr_t)h | (uintptr_t)dh | (uintptr_t)dx) & (es - 1)) ||
      (((uintptr_t)gain | (uintptr_t)rstd) & 3))
    return niti_fail(ctx, NITI_ERR_ARG, "niti_rmsnorm_bwd: bad argument (pointers are aligned to their type)");
  float *part = dgain ? (float *)((char *)ws + NITI_WS_HEADER) : nullptr;
  const bool aligned = (((uintptr_t)dy | (uintptr_t)h | (uintptr_t)dh | (uintptr_t)dx) & 15) == 0;
  // (512 threads with two vectors before 256 with four)
  RowPlan pl = plan_rows(M, C, type, aligned, 2);
  if (!pl.nv && pl.vec < 8) pl = plan_rows(M, C, type, aligned, pl.vec == 1 ? 8 : 4);
  int nparts = 0;
  rc = with_type(type, [&](auto t) -> int {
    constexpr int T = decltype(t)::value;
    constexpr int V16 = 16 / (int)sizeof(typename FloatOf<T>::type);
    if (!pl.nv) {
      auto wide = [&](auto vec) -> int {
        constexpr int VEC = decltype(vec)::value;
        if (dgain) {
          const int strips = (C + 256 * VEC - 1) / (256 * VEC), most = 8 * ctx->sm_count / strips;     // (one wave)
          nparts = most < 1 ? 1 : most < BWD_PARTS ? most : BWD_PARTS;
          if (nparts > M) nparts = M;
          NITI_CUDA_TRY(ctx, niti_launch(st, dim3((unsigned)strips, (unsigned)nparts), 256, 0, norm_wide_gain_kernel<T, VEC>, dy, h, rstd, part, M, C));
          ctx->launches++;
        }
        NITI_CUDA_TRY(ctx, niti_launch(st, (unsigned)(M < 2 * ctx->sm_count ? M : 2 * ctx->sm_count), 1024, 0, norm_bwd_wide_kernel<T, VEC>, dy, h, gain,
                                       rstd, dh, dx, M, C));
        return NITI_OK;
      };
      return pl.vec == 1 ? wide(std::integral_constant<int, 1>{}) : wide(std::integral_constant<int, V16>{});
    }
    const int threads = pl.sh.tpr * pl.sh.rpb;
    unsigned blocks = row_blocks(ctx, pl.sh, threads, 512);
    if (blocks > BWD_PARTS) blocks = BWD_PARTS;
    nparts = (int)blocks;
    const size_t smem = part && pl.sh.rpb > 1 ? (size_t)pl.sh.rpb * C * 4 : 0;       // (at most 8 rows of 1024)
    auto rows = [&](auto vec, auto nv) -> int {
      NITI_CUDA_TRY(ctx, niti_launch(st, blocks, threads, smem, norm_bwd_kernel<T, decltype(vec)::value, decltype(nv)::value>, dy, h, gain, rstd, dh,
                                     dx, part, pl.sh));
      return NITI_OK;
    };
    auto pick = [&](auto vec) -> int {
      if (pl.nv == 1) return rows(vec, std::integral_constant<int, 1>{});
      constexpr int VEC = decltype(vec)::value;
      if constexpr (VEC < 8)
        if (pl.nv == 4) return rows(vec, std::integral_constant<int, 4>{});
      if constexpr (VEC == 1)
        if (pl.nv == 8) return rows(vec, std::integral_constant<int, 8>{});
      return rows(vec, std::integral_constant<int, 2>{});
    };
    return pl.vec == 1 ? pick(std::integral_constant<int, 1>{}) : pick(std::integral_constant<int, V16>{});
  });
  ctx->launches++;
  if (rc != NITI_OK || !dgain) return rc;
  return launch_column_sums(ctx, st, part, dgain, nparts, C);
}

// dst[c] = sum over n rows of part[n][C], in a fixed order
static int launch_column_sums(niti_ctx *ctx, cudaStream_t st, const float *part, float *dst, int n, int C) {
  const unsigned grid = (unsigned)((C + 31) / 32);
  if (C % 4 == 0) NITI_CUDA_TRY(ctx, niti_launch(st, grid, 256, 0, column_sum_kernel<4>, part, dst, n, C));
  else NITI_CUDA_TRY(ctx, niti_launch(st, grid, 1024, 0, column_sum_kernel<1>, part, dst, n, C));
  ctx->launches++;
  return NITI_OK;
}

extern "C" int niti_dequantize(niti_ctx *ctx, void *stream, const void *q, const void *s, void *out, int format, int exponent_bytes, int type,
                               int64_t n, int64_t per) {
  if (!ctx) return NITI_ERR_ARG;
  if (n == 0 && niti_type_ok(type)) return NITI_OK;
  if (!q || !s || !out || !niti_type_ok(type) || n < 0 || per < 0 || (format != NITI_I8 && format != NITI_E4M3) ||
      (exponent_bytes != 1 && exponent_bytes != 4) || misaligned(out, (uintptr_t)niti_type_size(type)) || misaligned(s, (uintptr_t)exponent_bytes))
    return niti_fail(ctx, NITI_ERR_ARG, "niti_dequantize: bad argument (pointers are aligned to their type)");
  const bool wide = n >= 16 && (per == 0 || per >= 16) && !misaligned(q, 16) && !misaligned(out, 32);
  const long long want = ((wide ? n / 16 : n) + 255) / 256, cap = 16LL * ctx->sm_count;
  const int blocks = (int)(want < cap ? want : cap);
  const unsigned grid = (unsigned)(blocks + (wide && n % 16 ? 1 : 0));
  const Div d = per > 0 && n < (1LL << 31) ? make_div(per < (1LL << 31) ? per : (1LL << 31)) : Div{0u, -1};
  const int rc = with_type(type, [&](auto t) -> int {
    constexpr int T = decltype(t)::value;
    auto go = [&](auto e4m3, auto sv, auto w) -> int {
      typedef decltype(sv) S;
      NITI_CUDA_TRY(ctx, niti_launch((cudaStream_t)stream, grid, 256, 0, dequantize_kernel<T, decltype(e4m3)::value, S, decltype(w)::value>,
                                     (const uint8_t *)q, (const S *)s, out, (long long)n, d, (long long)per, blocks));
      return NITI_OK;
    };
    auto by_exponent = [&](auto e4m3, auto w) -> int { return exponent_bytes == 1 ? go(e4m3, (int8_t)0, w) : go(e4m3, (int32_t)0, w); };
    auto by_width = [&](auto e4m3) -> int { return wide ? by_exponent(e4m3, std::true_type{}) : by_exponent(e4m3, std::false_type{}); };
    return format == NITI_E4M3 ? by_width(std::true_type{}) : by_width(std::false_type{});
  });
  ctx->launches++;
  return rc;
}
