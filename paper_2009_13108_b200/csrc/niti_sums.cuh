// Sums over the rows of a matrix of partial sums, as a part of any kernel.
#pragma once
#include "niti_common.cuh"

// dst[c] = sum over the rows of part[n][C], in a fixed order, for the 32 columns of `block`: LANES threads for every W of them
// (a block of LANES * 32 / W threads; buf: LANES * 33 floats).  Bound: the latency of a few loads.  (One thread for a column
// and eight for its rows took 6.4 us of 296 rows of 4096.)
template <int W, int LANES>
__device__ __forceinline__ void niti_column_sums(const float *part, float *dst, int n, int C, int block, float *buf) {
  constexpr int PER = 32 / W;                      // threads side by side
  const int tx = (int)threadIdx.x % PER, ty = (int)threadIdx.x / PER;
  const int c = block * 32 + tx * W;
  float sum[W];
#pragma unroll
  for (int j = 0; j < W; ++j) sum[j] = 0.0f;
  if (c < C) {
#pragma unroll 8
    for (int i = ty; i < n; i += LANES) {
      if constexpr (W == 4) {
        const float4 v = *reinterpret_cast<const float4 *>(part + (long long)i * C + c);
        sum[0] += v.x; sum[1] += v.y; sum[2] += v.z; sum[3] += v.w;
      } else {
        sum[0] += part[(long long)i * C + c];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < W; ++j) buf[ty * 33 + tx * W + j] = sum[j];
  __syncthreads();
  if (threadIdx.x < 32 && block * 32 + (int)threadIdx.x < C) {
    float all = 0.0f;
#pragma unroll
    for (int k = 0; k < LANES; ++k) all += buf[k * 33 + threadIdx.x];
    dst[block * 32 + threadIdx.x] = all;
  }
}
