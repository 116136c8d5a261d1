// Internal interface of the fully connected layers with a float epilogue.
#pragma once
#include "niti_common.cuh"

// out = act(sum * 2^(s0 + s1) + bias) + res; z (optional) receives the argument of act.
struct LinearEpilogue {
  const int32_t *s0;       // exponents: one, or (s0_rows) one for every row of the output
  const int32_t *s1;       // one
  const float *bias;       // per column, may be null
  const void *res;         // may be null
  void *out, *z;           // z may be null
  int s0_rows, act;
};

// Contractions are split only where all shares run at once, so that their sums take at most a tile of 128 x 256 words an SM.
#define NITI_LINEAR_MAX_SMS 160
// A multiply on the tensor cores; operands with 16-byte aligned rows of pitch ld0, ld1.  kind: GK_FC_FWD (A [gm][gk], B
// [gn][gk]), GK_FC_DGRAD (A [gm][gk], B [gk][gn]) or GK_FC_WGRAD (A [gk][gm], B [gk][gn]).  e.out null: not wanted.
struct LinearMultiply {
  int kind, type;
  const int8_t *p0, *p1;
  long long ld0, ld1, gm, gn, gk;
  LinearEpilogue e;
};
// Words of a zeroed header that count the arrivals of a multiply's split tiles.
#define NITI_LINEAR_COUNTERS 320
// The forward multiply of a few rows, at most NITI_LINEAR_ROWS: streams the weights, in the caller's layout whatever K is.
#define NITI_LINEAR_ROWS 32
int niti_linear_rows(niti_ctx *ctx, cudaStream_t st, const int8_t *a, const int8_t *w, int M, int N, int K, const LinearEpilogue &e, int type);
