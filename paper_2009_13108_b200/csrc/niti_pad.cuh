// Rows of n bytes copied to rows of `pitch` bytes (see pad_pitch_kernel), as a part of any kernel.
#pragma once
#include "niti_common.cuh"

struct PadJob {
  const int8_t *src;
  int8_t *dst;
  long long rows;
  int n, pitch;
};
static inline unsigned niti_pad_blocks(const PadJob &j, int threads, long long most) {
  const long long want = (j.rows * (j.pitch >> 4) + threads - 1) / threads;
  return (unsigned)(want < most ? want : most);
}
// The share of block `block` of `blocks`.
__device__ __forceinline__ void niti_pad_rows(const PadJob &j, unsigned block, unsigned blocks) {
  const unsigned parts = (unsigned)j.pitch >> 4;
  for (long long base = (long long)block * blockDim.x; base < j.rows * parts; base += (long long)blocks * blockDim.x) {
    // (the division is by thread and 32 bits wide: the block's first row is found once)
    const long long r0 = base / parts;
    const unsigned t = (unsigned)(base - r0 * parts) + threadIdx.x, dr = t / parts, part = t - dr * parts;
    const long long r = r0 + dr;
    if (r >= j.rows) continue;
    const int left = j.n - 16 * (int)part;                // valid bytes of this part
    const long long o = r * j.n + 16 * part;
    const int mis = (int)(o & 3);
    const unsigned *p = reinterpret_cast<const unsigned *>(j.src) + (o >> 2);
    unsigned v[5], out[4];
#pragma unroll
    for (int k = 0; k < 5; ++k) v[k] = left > 0 && 4 * k < mis + (left < 16 ? left : 16) ? p[k] : 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int have = left - 4 * k;
      const unsigned w = __funnelshift_r(v[k], v[k + 1], 8u * (unsigned)mis);
      out[k] = have >= 4 ? w : (have <= 0 ? 0u : w & (0xffffffffu >> (32 - 8 * have)));
    }
    *reinterpret_cast<uint4 *>(j.dst + r * j.pitch + 16 * part) = make_uint4(out[0], out[1], out[2], out[3]);
  }
}
