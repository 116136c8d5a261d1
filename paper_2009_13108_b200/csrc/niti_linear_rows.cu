// The fully connected layer with a float epilogue for a few rows: decoding tokens, where the weights are read once and
// nothing else counts.  Bound: HBM (or L2, where the weights fit it).
#include "niti_act.cuh"
#include "niti_linear_act.h"
#include <type_traits>

namespace {

constexpr int DEEP = 4;                            // blocks of 64 contraction elements that a warp has in flight

// 16 bytes of a row from element k on; elements from K on are zero.  ALIGNED: rows are whole 16-byte vectors.
template <bool ALIGNED>
__device__ __forceinline__ uint4 load16(const int8_t *row, int k, int K, bool ok) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (!ok || k >= K) return v;
  if (ALIGNED) return __ldg(reinterpret_cast<const uint4 *>(row + k));
  v.x = niti_load_bytes4(row + k, K - k);
  v.y = niti_load_bytes4(row + k + 4, K - k - 4);
  v.z = niti_load_bytes4(row + k + 8, K - k - 8);
  v.w = niti_load_bytes4(row + k + 12, K - k - 12);
  return v;
}

__device__ __forceinline__ void mma_i8(int (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A block has 16 rows of the weights; its warps deal the contraction among them in pieces of 64 elements and add their sums
// in shared memory.  The weights are the multiply's 16 rows and the tokens its 8 columns (NT times).  Which contraction
// element sits in which place of a fragment does not matter as long as both operands agree, so a lane loads 16 consecutive
// bytes of its weight rows (g and g + 8) and of its token and uses them as the fragments of two multiplies.
// Weights from HBM: 1 x 8192 x 4096 9.0 us, of which a launch of nothing takes about 1.8 (4.7 TB/s while it streams), 1 x 4096 x
// 4096 5.6, 32 x 4096 x 4096 9.8 (the tokens come through L2 for every block).  The tiled kernel takes 17.5 us for the first.
template <int T, int NT, bool ALIGNED, int WARPS>
__global__ void __launch_bounds__(32 * WARPS)
linear_rows_kernel(const int8_t *a, const int8_t *w, int M, int N, int K, const LinearEpilogue e, uint32_t *status) {
  __shared__ int part[WARPS][16][8 * NT + 1];
  niti_enter(a, w);
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n0 = (int)blockIdx.x * 16;
  const bool ok0 = n0 + g < N, ok1 = n0 + g + 8 < N;
  const int8_t *w0 = w + (long long)(n0 + g) * K, *w1 = w0 + 8LL * K;
  int acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0;
  for (int k0 = warp * 64 + 16 * t; k0 - 16 * t < K; k0 += DEEP * WARPS * 64) {
    uint4 x0[DEEP], x1[DEEP];
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
      x0[d] = load16<ALIGNED>(w0, k0 + d * WARPS * 64, K, ok0);
      x1[d] = load16<ALIGNED>(w1, k0 + d * WARPS * 64, K, ok1);
    }
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
      uint4 y[NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) y[i] = load16<ALIGNED>(a + (long long)(8 * i + g) * K, k0 + d * WARPS * 64, K, 8 * i + g < M);
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        mma_i8(acc[i], x0[d].x, x1[d].x, x0[d].y, x1[d].y, y[i].x, y[i].y);
        mma_i8(acc[i], x0[d].z, x1[d].z, x0[d].w, x1[d].w, y[i].z, y[i].w);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    part[warp][g][8 * i + 2 * t] = acc[i][0];
    part[warp][g][8 * i + 2 * t + 1] = acc[i][1];
    part[warp][g + 8][8 * i + 2 * t] = acc[i][2];
    part[warp][g + 8][8 * i + 2 * t + 1] = acc[i][3];
  }
  __syncthreads();
  const int s1 = *e.s1;
  for (int i = (int)threadIdx.x; i < 16 * M; i += 32 * WARPS) {
    const int n = i & 15, m = i >> 4;
    if (n0 + n >= N) continue;
    int sum = 0;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) sum += part[k][n][m];
    const int s = e.s0[e.s0_rows ? m : 0] + s1;
    if (s < -128 || s > 127) atomicOr(status, NITI_DEV_EXP_RANGE);
    const long long at = (long long)m * N + n0 + n;
    float x[1] = {(float)sum * linear_scale(s)};
    if (e.bias) x[0] += e.bias[n0 + n];
    Pack<T, 1> p;
    if (e.z) {
      p.set(x);
      p.store(e.z, at);
    }
    x[0] = act_one(x[0], e.act);
    if (e.res) {
      p.load(e.res, at);
      x[0] += p.get(0);
    }
    p.set(x);
    p.store(e.out, at);
  }
}

}  // namespace

int niti_linear_rows(niti_ctx *ctx, cudaStream_t st, const int8_t *a, const int8_t *w, int M, int N, int K, const LinearEpilogue &e, int type) {
  const unsigned grid = (unsigned)((N + 15) / 16);
  auto go_as = [&](auto tc, auto nt, auto al, auto wc) -> int {
    constexpr int WARPS = decltype(wc)::value;
    NITI_CUDA_TRY(ctx, niti_launch(st, grid, 32 * WARPS, 0, linear_rows_kernel<decltype(tc)::value, decltype(nt)::value, decltype(al)::value, WARPS>, a, w,
                                   M, N, K, e, ctx->d_status));
    ctx->launches++;
    ctx->tc_launches++;
    return NITI_OK;
  };
  // Sixteen warps a block where the contraction feeds them and all blocks still run at once (three an SM), else eight: weights
  // beyond L2, 8 -> 16 warps, 1 x 4096 x 4096 7.5 -> 5.3 us, 32 x 4096 x 4096 13.2 -> 9.9, 1 x 4096 x 16384 25.3 -> 15.4; outside
  // the rule 1 x 8192 x 4096 9.0 -> 9.2, 16 x 4096 x 1024 3.3 -> 3.9.
  const bool wide = K >= 2048 && (long long)grid <= 3LL * ctx->sm_count;
  auto go = [&](auto tc, auto nt, auto al) -> int {
    if constexpr (decltype(al)::value)
      if (wide) return go_as(tc, nt, al, std::integral_constant<int, 16>{});
    return go_as(tc, nt, al, std::integral_constant<int, 8>{});
  };
  auto by_rows = [&](auto tc, auto al) -> int {
    if (M <= 8) return go(tc, std::integral_constant<int, 1>{}, al);
    if (M <= 16) return go(tc, std::integral_constant<int, 2>{}, al);
    return go(tc, std::integral_constant<int, 4>{}, al);
  };
  auto by_type = [&](auto tc) -> int { return K % 16 == 0 ? by_rows(tc, std::true_type{}) : by_rows(tc, std::false_type{}); };
  if (type == NITI_F32) return by_type(std::integral_constant<int, NITI_F32>{});
  if (type == NITI_BF16) return by_type(std::integral_constant<int, NITI_BF16>{});
  return by_type(std::integral_constant<int, NITI_F16>{});
}
