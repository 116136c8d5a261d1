// Fully connected layers whose results leave the integer format in the multiply's epilogue: scale by the operands' exponents,
// bias, activation and residual, stored in 16 or 32 bits; and their backward pass, an error that is rounded to int8 with one
// exponent and the two multiplies that it enters.
#include "niti_act.cuh"
#include "niti_div.h"
#include "niti_linear_act.h"
#include "niti_tcgen05.cuh"
#include <type_traits>

namespace {

constexpr int BM = 128;                            // rows of a tile = TMEM lanes
constexpr int PROD_WARPS = 3, MMA_WARP = 3, EPI_WARP0 = 4;
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 32 * (EPI_WARP0 + EPI_WARPS);
constexpr int MAX_STAGES = 8, MAX_TBUF = 4;
constexpr int STG_FLOATS = 32 * 33;                // a warp's buffer for rows that are not whole, aligned vectors

struct Params {
  int gm, gn;
  int bn, nbuf, tmem_cols;
  int kdepth, ksteps, kb_total, kb_per_split, splits;
  int stages, nprod;
  int a_bytes, b_bytes, a_boxes, b_boxes, a_box_bytes, b_box_bytes, a_box_step, b_box_step;
  unsigned idesc;
  unsigned long long a_desc, b_desc;
  unsigned a_kstep16, b_kstep16;
  int n_tiles_n, m_units, raster_g, last_group, items;
  Div d_split, d_group, d_units, d_last;
  int stg_off;                                     // byte offset of the warps' buffers, behind the stages
  int direct;                                      // rows are whole, aligned pieces of 32 bytes
  LinearEpilogue e;
};

__device__ __forceinline__ void decode(const Params &p, int item, int &mu, int &nt, int &split, int &tile) {
  tile = item;
  split = 0;
  if (p.splits > 1) {
    tile = div_by(item, p.d_split);
    split = item - tile * p.splits;
  }
  const int g = div_by(tile, p.d_group);
  const int rem = tile - g * p.raster_g * p.n_tiles_n;
  const bool last = g == p.last_group;
  nt = div_by(rem, last ? p.d_last : p.d_units);
  mu = g * p.raster_g + rem - nt * (last ? p.m_units - g * p.raster_g : p.raster_g);
}

// What follows the multiply, for 32 columns from n0 of a tile's rows; a lane holds the int32 sums of its row.
template <int T>
__device__ __forceinline__ void finish_chunk(const Params &p, int (&v)[32], int row0, int n0, float f, float *stg, int lane) {
  const LinearEpilogue &e = p.e;
  typedef typename FloatOf<T>::type FT;
  constexpr int N32 = 32 / (int)sizeof(FT);
  if (p.direct) {
    const int row = row0 + lane;
    const long long at = (long long)row * p.gn + n0;
    const bool rok = row < p.gm;
    float x[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) x[j] = (float)v[j] * f;
    if (e.bias) {
#pragma unroll
      for (int j = 0; j < 32; j += 4)
        if (n0 + j < p.gn) {
          const float4 b = *reinterpret_cast<const float4 *>(e.bias + n0 + j);
          x[j] += b.x; x[j + 1] += b.y; x[j + 2] += b.z; x[j + 3] += b.w;
        }
    }
    if (e.z) {
#pragma unroll
      for (int j = 0; j < 32; j += N32) {
        unsigned w[8];
        pack32<T, N32>(x + j, w);
        if (rok && n0 + j < p.gn) store32((FT *)e.z + at + j, w);
      }
    }
    act_all(x, e.act);
#pragma unroll
    for (int j = 0; j < 32; j += N32) {
      unsigned w[8];
      if (rok && n0 + j < p.gn) {
        if (e.res) {
          load32((const FT *)e.res + at + j, w);
#pragma unroll
          for (int i = 0; i < N32; ++i) x[j + i] += get32<T, N32>(w, i);
        }
        pack32<T, N32>(x + j, w);
        store32((FT *)e.out + at + j, w);
      }
    }
    return;
  }
  // through shared memory, so that a lane has a column and an instruction whole rows
#pragma unroll
  for (int j = 0; j < 32; ++j) stg[lane * 33 + j] = __int_as_float(v[j]);
  __syncwarp();
  const int col = n0 + lane;
  const bool cok = col < p.gn;
  const float b = e.bias && cok ? e.bias[col] : 0.0f;
#pragma unroll 4
  for (int r = 0; r < 32; ++r) {
    const float fr = __shfl_sync(0xffffffffu, f, r);
    if (row0 + r >= p.gm || !cok) continue;
    const long long at = (long long)(row0 + r) * p.gn + col;
    float x[1] = {(float)__float_as_int(stg[r * 33 + lane]) * fr + b};
    Pack<T, 1> k;
    if (e.z) {
      k.set(x);
      k.store(e.z, at);
    }
    x[0] = act_one(x[0], e.act);
    if (e.res) {
      k.load(e.res, at);
      x[0] += k.get(0);
    }
    k.set(x);
    k.store(e.out, at);
  }
  __syncwarp();
}

// Do all epilogue warps say so?
__device__ __forceinline__ bool epilogue_all(bool ok) {
  int all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, %2, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
               : "=r"(all)
               : "r"((int)ok), "n"(32 * EPI_WARPS)
               : "memory");
  return all != 0;
}

// One persistent CTA (or pair on a 256-row tile) per SM; warps 0 - 2 copy, warp 3 multiplies, the others finish tiles.  The
// pipeline is the one of the integer layers' kernel; nothing here depends on the whole tensor, so that a tile is final when
// its sums are.  A contraction that is split over CTAs leaves its sums in slabs; the CTA that comes last adds them up, in the
// order of the splits (integers: any order gives the same), and finishes the tile.
template <int KIND, int CTAS, int T>
__global__ void __launch_bounds__(THREADS, 1)
linear_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Params p, int *slabs,
              unsigned *counters, WsHeader *next, uint32_t *status) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ __align__(8) unsigned long long bars[2 * MAX_STAGES + 2 * MAX_TBUF];
  __shared__ unsigned tmem_slot;
  __shared__ volatile int abort_flag;
  __shared__ int is_last;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = (int)threadIdx.x & 31;
  const unsigned rank = CTAS == 2 ? cluster_ctarank() : 0u;
  const unsigned smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int stage_bytes = p.a_bytes + p.b_bytes;
  const unsigned full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[MAX_STAGES]);
  const unsigned tfull0 = smem_u32(&bars[2 * MAX_STAGES]), tempty0 = smem_u32(&bars[2 * MAX_STAGES + MAX_TBUF]);
  const unsigned lead_full0 = CTAS == 2 ? map_to_cta(full0, 0) : full0;
  const unsigned lead_tempty0 = CTAS == 2 ? map_to_cta(tempty0, 0) : tempty0;
  const int first_item = (int)blockIdx.x / CTAS, item_step = (int)gridDim.x / CTAS;

  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
  }
  if (threadIdx.x == 0) abort_flag = 0;
  if (threadIdx.x < 2 * MAX_STAGES + 2 * MAX_TBUF) {
    mbar_init(smem_u32(&bars[threadIdx.x]), threadIdx.x >= 2 * MAX_STAGES + MAX_TBUF ? EPI_WARPS * CTAS : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == MMA_WARP) {
    if (CTAS == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"((unsigned)p.tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"((unsigned)p.tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync_all();
  tc_fence_after();
  const unsigned tmem_base = tmem_slot;
  niti_enter(slabs);
  if (next && blockIdx.x == 0 && warp == EPI_WARP0 + EPI_WARPS - 1) niti_zero_header(next, lane);

  if (warp < PROD_WARPS) {
    const bool leader = elect_one();
    int stage = 0, owner = 0;
    unsigned phase = 0;
    bool ok = true;
    const int bn_cta = p.bn / CTAS;
    const unsigned tx = (unsigned)(CTAS * (p.a_boxes * p.a_box_bytes + p.b_boxes * p.b_box_bytes));
    for (int item = first_item; ok && item < p.items; item += item_step) {
      int mu, nt, split, tile;
      decode(p, item, mu, nt, split, tile);
      const int m0 = (mu * CTAS + (int)rank) * BM, n0 = nt * p.bn + (int)rank * bn_cta;
      const int kb0 = split * p.kb_per_split, kb1 = min(kb0 + p.kb_per_split, p.kb_total);
      for (int kb = kb0; kb < kb1; ++kb) {
        if (owner == warp) {
          if (!mbar_wait_warp(empty0 + 8 * stage, phase ^ 1, &abort_flag, status)) { ok = false; break; }
          const unsigned full = lead_full0 + 8 * stage, sa = smem_base + stage * stage_bytes, sb = sa + p.a_bytes;
          if (leader) {
            if (rank == 0) mbar_expect_tx(full0 + 8 * stage, tx);
            const int k = kb * p.kdepth;
            if (KIND == GK_FC_WGRAD) {
              for (int j = 0; j < p.a_boxes; ++j) load2<CTAS>(sa + j * p.a_box_bytes, &map_a, full, m0 + j * p.a_box_step, k);
            } else {
              load2<CTAS>(sa, &map_a, full, k, m0);
            }
            if (KIND == GK_FC_FWD) {
              load2<CTAS>(sb, &map_b, full, k, n0);
            } else {
              for (int j = 0; j < p.b_boxes; ++j) load2<CTAS>(sb + j * p.b_box_bytes, &map_b, full, n0 + j * p.b_box_step, k);
            }
          }
        }
        if (++owner == p.nprod) owner = 0;
        if (++stage == p.stages) { stage = 0; phase ^= 1; }
      }
    }
  } else if (warp == MMA_WARP) {
    if (rank == 0) {
      const bool leader = elect_one();
      int stage = 0;
      unsigned phase = 0, buf = 0, par = 0;
      bool ok = true;
      const unsigned a_lo0 = (unsigned)p.a_desc, b_lo0 = (unsigned)p.b_desc, a_hi = (unsigned)(p.a_desc >> 32), b_hi = (unsigned)(p.b_desc >> 32);
      const unsigned ak = p.a_kstep16, bk = p.b_kstep16, idesc = p.idesc, a_bytes = (unsigned)p.a_bytes;
      const int ksteps = p.ksteps;
      for (int item = first_item; ok && item < p.items; item += item_step) {
        const int split = p.splits > 1 ? item - div_by(item, p.d_split) * p.splits : 0;
        const int kb0 = split * p.kb_per_split, kb1 = min(kb0 + p.kb_per_split, p.kb_total);
        if (!mbar_wait_warp(tempty0 + 8 * buf, par ^ 1u, &abort_flag, status)) { ok = false; break; }
        const unsigned tfull = tfull0 + 8 * buf, tmem_d = tmem_base + buf * (unsigned)p.bn;
        if (++buf == (unsigned)p.nbuf) { buf = 0; par ^= 1u; }
        tc_fence_after();
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait_warp(full0 + 8 * stage, phase, &abort_flag, status)) { ok = false; break; }
          tc_fence_after();
          const unsigned sa = smem_base + stage * stage_bytes;
          const unsigned a_lo = a_lo0 + ((sa >> 4) & 0x3fff), b_lo = b_lo0 + (((sa + a_bytes) >> 4) & 0x3fff);
          const unsigned acc = kb > kb0 ? 1u : 0u;
          if (leader) {
            if (ksteps == 4) issue_kblock<CTAS, 4>(tmem_d, a_lo, a_hi, b_lo, b_hi, ak, bk, idesc, acc);
            else if (ksteps == 2) issue_kblock<CTAS, 2>(tmem_d, a_lo, a_hi, b_lo, b_hi, ak, bk, idesc, acc);
            else issue_kblock<CTAS, 1>(tmem_d, a_lo, a_hi, b_lo, b_hi, ak, bk, idesc, acc);
            if (CTAS == 2) tc_commit_pair(empty0 + 8 * stage); else tc_commit(empty0 + 8 * stage);
          }
          if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        if (ok && leader) {
          if (CTAS == 2) tc_commit_pair(tfull); else tc_commit(tfull);
        }
      }
    }
  } else {
    const int ew = warp - EPI_WARP0, quarter = warp & 3, part = ew >> 2;
    float *stg = reinterpret_cast<float *>(smem_raw + (smem_base - smem_u32(smem_raw)) + p.stg_off) + ew * STG_FLOATS;
    const LinearEpilogue &e = p.e;
    const int s_col = (e.s1 ? *e.s1 : 0);
    unsigned buf = 0, par = 0;
    bool wide_exp = false;
    for (int item = first_item; item < p.items; item += item_step) {
      int mu, nt, split, tile;
      decode(p, item, mu, nt, split, tile);
      const int row0 = (mu * CTAS + (int)rank) * BM + 32 * quarter, n0 = nt * p.bn;
      const int row = row0 + lane < p.gm ? row0 + lane : p.gm - 1;
      const int s = e.s0[e.s0_rows ? row : 0] + s_col;
      wide_exp |= s < -128 || s > 127;
      const float f = linear_scale(s);
      bool ok = mbar_wait_warp(tfull0 + 8 * buf, par, &abort_flag, status);
      if (p.splits > 1) ok = epilogue_all(ok);     // (they meet at barriers below: all go on, or none)
      if (!ok) break;
      tc_fence_after();
      const unsigned tm = tmem_base + buf * (unsigned)p.bn + ((unsigned)(32 * quarter) << 16);
      const unsigned tempty = lead_tempty0 + 8 * buf;
      if (++buf == (unsigned)p.nbuf) { buf = 0; par ^= 1u; }
      auto drained = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) { if (CTAS == 2) mbar_arrive_cluster(tempty); else mbar_arrive(tempty); }
      };
      if (p.splits == 1) {
        for (int c = part; c < p.bn / 32; c += EPI_WARPS / 4) {
          int v[32];
          if (n0 + 32 * c < p.gn) {
            tc_ld32(tm + 32u * (unsigned)c, v);
            finish_chunk<T>(p, v, row0, n0 + 32 * c, f, stg, lane);
          }
        }
        drained();
        continue;
      }
      // a share of a split contraction: 32 columns x 128 rows of sums in column order
      const int slot = tile * CTAS + (int)rank, words = p.bn * BM;
      int *mine = slabs + ((long long)slot * p.splits + split) * words + 32 * quarter + lane;
      for (int c = part; c < p.bn / 32; c += EPI_WARPS / 4) {
        int v[32];
        tc_ld32(tm + 32u * (unsigned)c, v);
#pragma unroll
        for (int j = 0; j < 32; ++j) mine[(32 * c + j) * BM] = v[j];
      }
      drained();
      __threadfence();
      asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory");
      if (ew == 0 && lane == 0) {
        const unsigned before = atomicAdd(counters + slot, 1u);
        __threadfence();
        is_last = before == (unsigned)p.splits - 1u;
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory");
      if (is_last) {
        const int *all = slabs + (long long)slot * p.splits * words + 32 * quarter + lane;
        for (int c = part; c < p.bn / 32; c += EPI_WARPS / 4) {
          if (n0 + 32 * c >= p.gn) continue;
          int v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0;
          for (int k = 0; k < p.splits; ++k) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += __ldcg(all + (long long)k * words + (32 * c + j) * BM);
          }
          finish_chunk<T>(p, v, row0, n0 + 32 * c, f, stg, lane);
        }
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory");          // (is_last has been read by all)
    }
    if (__any_sync(0xffffffffu, wide_exp) && lane == 0) atomicOr(status, NITI_DEV_EXP_RANGE);
  }

  tc_fence_before();
  __syncthreads();
  if (abort_flag) {                                // copies and multiplies in flight land before the memories go away
    const long long t0 = clock64();
    while (clock64() - t0 < 20000000LL) {
    }
    __syncthreads();
  }
  if (CTAS == 2) cluster_sync_all();
  if (warp == MMA_WARP) {
    tc_fence_after();
    if (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((unsigned)p.tmem_cols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((unsigned)p.tmem_cols) : "memory");
  }
}

// ---- host ------------------------------------------------------------------------------------
// Cycles of a k-block of 128 contraction elements: multiplies, or the operand copies (constants as measured for the integer
// layers' kernel: 84 bytes a clock into one SM, 9000 into all).
double kblock_cycles(int ctas, int bn, int ksteps, long long running) {
  const double mma = bn / 2.0, smem = 32.0 + bn / (4.0 * ctas), bytes = (128.0 + (double)bn / ctas) * 32.0 * ksteps;
  double c = ksteps * (mma > smem ? mma : smem);
  if (c < bytes / 84.0) c = bytes / 84.0;
  if (c < bytes * (double)running / 9000.0) c = bytes * (double)running / 9000.0;
  return c < 100.0 * ksteps ? 100.0 * ksteps : c;
}

struct Choice { int ctas, bn, splits; };
// Tile width, pairs and splits with the least modelled time: k-blocks of a wave, the epilogue of its tiles (about 20 issue
// slots an element, hidden behind the next tile's main loop), and for splits the slabs' way through L2.
Choice choose(const niti_ctx *ctx, int kind, long long gm, long long gn, int kb, int ksteps, int pairs) {
  Choice best = {1, 32, 1};
  double least = 1e300;
  const long long mt = (gm + BM - 1) / BM;
  const int unit = kind == GK_FC_FWD ? 32 : 64;
  for (int ctas = 1; ctas <= 2; ++ctas) {
    if (ctas == 2 && mt < 2) break;
    const long long mu = (mt + ctas - 1) / ctas, units = ctas == 2 ? pairs : ctx->sm_count;
    for (int bn = 256; bn >= unit; bn -= unit) {
      if (bn > 32 && bn - unit >= gn && bn > unit) continue;
      if (bn / ctas % 16) continue;
      const long long tiles = mu * ((gn + bn - 1) / bn);
      const double epi = 20.0 * bn;
      for (int s = 1; s <= 32; s += s < 4 ? 1 : s < 8 ? 2 : 4) {
        if (s > 1 && (tiles * s > units || kb / s < 4 || tiles * ctas > NITI_LINEAR_COUNTERS || ctx->sm_count > NITI_LINEAR_MAX_SMS)) break;
        const long long items = tiles * s, waves = (items + units - 1) / units;
        const double main = ((kb + s - 1) / s) * kblock_cycles(ctas, bn, ksteps, (items < units ? items : units) * ctas);
        double t = main + (double)(waves - 1) * (main > epi ? main : epi) + epi + (ctas == 2 ? 1500.0 : 0.0);
        if (s > 1) t += 3000.0 + 8.0 * bn * (s + 1);
        if (t < least * 0.98) { least = t; best = {ctas, bn, s}; }
      }
    }
  }
  return best;
}

template <int KIND, int CTAS, int T>
int set_up(niti_ctx *ctx) {
  // (per device and instance, the same value in every context: see niti_ctx::smem_optin)
  bool &ready = ctx->linear_ready[(KIND * 2 + CTAS - 1) * 3 + T];
  if (ready) return NITI_OK;
  cudaFuncAttributes fa;
  NITI_CUDA_TRY(ctx, cudaFuncGetAttributes(&fa, linear_kernel<KIND, CTAS, T>));
  NITI_CUDA_TRY(ctx, cudaFuncSetAttribute(linear_kernel<KIND, CTAS, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                          (int)(ctx->smem_optin - fa.sharedSizeBytes)));
  ready = true;
  return NITI_OK;
}

// CTA pairs that run at once (SMs pair up inside a GPC, so there can be fewer than half of the SMs).
int ask_pairs(niti_ctx *ctx) {
  if (ctx->linear_pairs) return NITI_OK;
  const int rc = set_up<GK_FC_FWD, 2, NITI_BF16>(ctx);
  if (rc != NITI_OK) return rc;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)(ctx->sm_count / 2 * 2), 1, 1);
  cfg.blockDim = dim3(THREADS, 1, 1);
  cfg.dynamicSmemBytes = 200 * 1024;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  NITI_CUDA_TRY(ctx, cudaOccupancyMaxActiveClusters(&n, linear_kernel<GK_FC_FWD, 2, NITI_BF16>, &cfg));
  ctx->linear_pairs = n < 1 ? 1 : n < ctx->sm_count / 2 ? n : ctx->sm_count / 2;
  return NITI_OK;
}

template <int KIND, int CTAS, int T>
int launch_as(niti_ctx *ctx, cudaStream_t st, const Params &p, const CUtensorMap &ma, const CUtensorMap &mb, size_t smem, unsigned grid, int *slabs,
              unsigned *counters, WsHeader *next) {
  const int rc = set_up<KIND, CTAS, T>(ctx);
  if (rc != NITI_OK) return rc;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(THREADS, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CTAS;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  NITI_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, linear_kernel<KIND, CTAS, T>, ma, mb, p, slabs, counters, next, ctx->d_status));
  ctx->launches++;
  ctx->tc_launches++;
  if (CTAS == 2) ctx->tc2_launches++;
  return NITI_OK;
}

}  // namespace

int niti_linear_gemm(niti_ctx *ctx, cudaStream_t st, int kind, const int8_t *p0, long long ld0, const int8_t *p1, long long ld1, long long gm,
                     long long gn, long long gk, const LinearEpilogue &e, int type, int *slabs, unsigned *counters, WsHeader *next) {
  Params p;
  memset(&p, 0, sizeof(p));
  p.gm = (int)gm; p.gn = (int)gn;
  p.e = e;
  p.kdepth = pick_swizzle(gk);
  p.ksteps = p.kdepth / 32;
  p.kb_total = (int)((gk + p.kdepth - 1) / p.kdepth);
  const int rc = ask_pairs(ctx);
  if (rc != NITI_OK) return rc;
  const int pairs = ctx->linear_pairs;
  const Choice c = choose(ctx, kind, gm, gn, p.kb_total, p.ksteps, pairs);
  const int ctas = c.ctas;
  p.bn = c.bn;
  p.kb_per_split = (p.kb_total + c.splits - 1) / c.splits;
  p.splits = (p.kb_total + p.kb_per_split - 1) / p.kb_per_split;
  const int bn_cta = p.bn / ctas;
  MapSpec sa, sb;
  memset(&sa, 0, sizeof(sa));
  memset(&sb, 0, sizeof(sb));
  const bool a_mn = kind == GK_FC_WGRAD, b_mn = kind != GK_FC_FWD;
  int a_sw = p.kdepth, b_sw = p.kdepth;
  if (a_mn) {
    a_sw = pick_swizzle(gm);
    sa = {2, {(cuuint64_t)gm, (cuuint64_t)gk}, {(cuuint64_t)ld0}, {(cuuint32_t)a_sw, (cuuint32_t)p.kdepth}, a_sw, p0};
    p.a_boxes = BM / a_sw;
    if ((long long)p.a_boxes * a_sw > (gm + a_sw - 1) / a_sw * a_sw) p.a_boxes = (int)((gm + a_sw - 1) / a_sw);
    p.a_box_bytes = p.kdepth * a_sw;
    p.a_box_step = a_sw;
    p.a_bytes = (BM / a_sw) * p.a_box_bytes;
    p.a_desc = desc_mnmajor(a_sw, p.kdepth);
    p.a_kstep16 = (unsigned)((32 * a_sw) >> 4);
  } else {
    sa = {2, {(cuuint64_t)gk, (cuuint64_t)gm}, {(cuuint64_t)ld0}, {(cuuint32_t)p.kdepth, BM}, a_sw, p0};
    p.a_boxes = 1;
    p.a_box_bytes = p.a_bytes = BM * p.kdepth;
    p.a_desc = desc_kmajor(a_sw);
    p.a_kstep16 = 2;
  }
  if (b_mn) {
    b_sw = pick_swizzle_mn(bn_cta);
    sb = {2, {(cuuint64_t)gn, (cuuint64_t)gk}, {(cuuint64_t)ld1}, {(cuuint32_t)b_sw, (cuuint32_t)p.kdepth}, b_sw, p1};
    p.b_boxes = (bn_cta + b_sw - 1) / b_sw;
    p.b_box_bytes = p.kdepth * b_sw;
    p.b_box_step = b_sw;
    p.b_bytes = p.b_boxes * p.b_box_bytes;
    p.b_desc = desc_mnmajor(b_sw, p.kdepth);
    p.b_kstep16 = (unsigned)((32 * b_sw) >> 4);
  } else {
    sb = {2, {(cuuint64_t)gk, (cuuint64_t)gn}, {(cuuint64_t)ld1}, {(cuuint32_t)p.kdepth, (cuuint32_t)bn_cta}, b_sw, p1};
    p.b_boxes = 1;
    p.b_box_bytes = p.b_bytes = bn_cta * p.kdepth;
    p.b_desc = desc_kmajor(b_sw);
    p.b_kstep16 = 2;
  }
  p.a_bytes = (p.a_bytes + 1023) / 1024 * 1024;
  p.b_bytes = (p.b_bytes + 1023) / 1024 * 1024;
  const int es = niti_type_size(type);
  const uintptr_t ptrs = (uintptr_t)e.out | (uintptr_t)e.res | (uintptr_t)e.z;
  p.direct = (gn * es) % 32 == 0 && (ptrs & 31) == 0 && ((uintptr_t)e.bias & 15) == 0;
  const int stg = p.direct ? 0 : EPI_WARPS * STG_FLOATS * 4;
  const int stage = p.a_bytes + p.b_bytes;
  p.stages = (216 * 1024 - stg) / stage;
  if (p.stages > MAX_STAGES) p.stages = MAX_STAGES;
  if (p.stages == 5 || p.stages == 7) p.stages -= 1;
  if (p.stages < 2) return niti_fail(ctx, NITI_ERR_SHAPE, "linear layer: no room for two stages");
  p.stg_off = p.stages * stage;
  p.nprod = 1;
  for (int d = 2; d <= PROD_WARPS; ++d)
    if (p.stages % d == 0) p.nprod = d;
  p.nbuf = 512 / p.bn > MAX_TBUF ? MAX_TBUF : 512 / p.bn;
  p.tmem_cols = 32;
  while (p.tmem_cols < p.nbuf * p.bn) p.tmem_cols <<= 1;
  // instruction descriptor: s32 accumulate, signed 8-bit operands, majorness, N, M
  p.idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((unsigned)a_mn << 15) | ((unsigned)b_mn << 16) | ((unsigned)(p.bn >> 3) << 17) |
            ((unsigned)((BM * ctas) >> 4) << 24);
  const long long mt = (gm + BM - 1) / BM;
  p.m_units = (int)((mt + ctas - 1) / ctas);
  p.n_tiles_n = (int)((gn + p.bn - 1) / p.bn);
  const long long items = (long long)p.m_units * p.n_tiles_n * p.splits;
  if (items >= (1LL << 30)) return niti_fail(ctx, NITI_ERR_SHAPE, "linear layer: too many tiles");
  p.items = (int)items;
  p.raster_g = ctas == 2 ? 8 : 12;
  p.last_group = (p.m_units - 1) / p.raster_g;
  p.d_split = make_div(p.splits);
  p.d_group = make_div((long long)p.raster_g * p.n_tiles_n);
  p.d_units = make_div(p.raster_g);
  p.d_last = make_div(p.m_units - p.last_group * p.raster_g);
  CUtensorMap ma, mb;
  if (!encode(ctx, &ma, sa) || !encode(ctx, &mb, sb)) return niti_fail(ctx, NITI_ERR_CUDA, "linear layer: no tensor map for an operand");
  const size_t smem = (size_t)p.stg_off + stg + 1024;
  const long long units = ctas == 2 ? pairs : ctx->sm_count;
  const unsigned grid = (unsigned)((items < units ? items : units) * ctas);
  auto with_kind = [&](auto kc) -> int {
    constexpr int KIND = decltype(kc)::value;
    auto with = [&](auto tc) -> int {
      constexpr int T = decltype(tc)::value;
      return ctas == 2 ? launch_as<KIND, 2, T>(ctx, st, p, ma, mb, smem, grid, slabs, counters, next)
                       : launch_as<KIND, 1, T>(ctx, st, p, ma, mb, smem, grid, slabs, counters, next);
    };
    if (type == NITI_F32) return with(std::integral_constant<int, NITI_F32>{});
    if (type == NITI_BF16) return with(std::integral_constant<int, NITI_BF16>{});
    return with(std::integral_constant<int, NITI_F16>{});
  };
  if (kind == GK_FC_FWD) return with_kind(std::integral_constant<int, GK_FC_FWD>{});
  if (kind == GK_FC_DGRAD) return with_kind(std::integral_constant<int, GK_FC_DGRAD>{});
  return with_kind(std::integral_constant<int, GK_FC_WGRAD>{});
}

// ---- the error of the backward pass ---------------------------------------------------------
namespace {

constexpr int ERR_THREADS = 128;
constexpr unsigned INF_BITS = 0x7f800000u;

// e = dout act'(z) of a block's rows and columns, a thread on the same VEC columns in every row.
template <int T, int VEC, int ACT, typename F>
__device__ __forceinline__ void error_rows(const void *dout, const void *z, int N, int r0, int r1, int c, F take) {
  constexpr int DEEP = 4;                          // rows in flight
  for (int r = r0; r < r1; r += DEEP) {
    Pack<T, VEC> d[DEEP], zz[DEEP];
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
      if (r + k < r1) {
        d[k].load(dout, (long long)(r + k) * N + c);
        if (ACT != NITI_ACT_NONE) zz[k].load(z, (long long)(r + k) * N + c);
      }
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
      if (r + k < r1) {
        float e[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) e[j] = ACT == NITI_ACT_NONE ? d[k].get(j) : d[k].get(j) * act_slope(zz[k].get(j), ACT);
        take(r + k, e);
      }
  }
}

// Largest |e| of the tensor, and the column sums of every block's rows.  Bound: HBM (dout and z are read once here; the
// rounding pass finds what fits of them in L2).
template <int T, int VEC, int ACT>
__global__ void __launch_bounds__(ERR_THREADS)
error_max_kernel(const void *dout, const void *z, float *part, WsHeader *hdr, WsHeader *next, int M, int N, int rows) {
  niti_enter(dout, z);
  const int c = ((int)blockIdx.x * ERR_THREADS + (int)threadIdx.x) * VEC, r0 = (int)blockIdx.y * rows, r1 = min(r0 + rows, M);
  if (next && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 32) niti_zero_header(next, (int)threadIdx.x);
  float sum[VEC];
  float largest = 0.0f;
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] = 0.0f;
  if (c < N) {
    error_rows<T, VEC, ACT>(dout, z, N, r0, r1, c, [&](int, const float (&e)[VEC]) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        sum[j] += e[j];
        largest = niti_absmax(largest, e[j]);
      }
    });
    if (part) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) part[(long long)blockIdx.y * N + c + j] = sum[j];
    }
  }
  const unsigned most = __reduce_max_sync(0xffffffffu, __float_as_uint(largest));
  if ((threadIdx.x & 31) == 0 && most) atomicMax(&hdr->maxabs32, most);
}

// e as payload with the exponent of its maximum, rows of `pitch` bytes.  The rows that the pass before read last come first.
template <int T, int VEC, int ACT, bool PSR>
__global__ void __launch_bounds__(ERR_THREADS)
error_round_kernel(const void *dout, const void *z, int8_t *e8, int32_t *s_e, const WsHeader *hdr, uint32_t *status, int M, int N, int rows,
                   int pitch) {
  niti_enter(dout, z, hdr);
  const unsigned most = hdr->maxabs32;
  const int s = niti_exponent_of(most);
  const float scale = niti_payload_scale(niti_pow2(-s), PSR ? NITI_ROUND_PSR : NITI_ROUND_NEAREST);
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    *s_e = s;
    if (most >= INF_BITS) atomicOr(status, NITI_DEV_NONFINITE);
  }
  const int by = (int)(gridDim.y - 1 - blockIdx.y);
  const int c = ((int)blockIdx.x * ERR_THREADS + (int)threadIdx.x) * VEC, r0 = by * rows, r1 = min(r0 + rows, M);
  if (c >= N) return;
  error_rows<T, VEC, ACT>(dout, z, N, r0, r1, c, [&](int r, const float (&e)[VEC]) {
    niti_store_payload<VEC, PSR>(e8, (long long)r * pitch + c, e, scale);
  });
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
long long pitch16(long long n) { return (n + 15) / 16 * 16; }
size_t pad_bytes(long long rows, long long width) { return width % 16 ? up256((size_t)rows * (size_t)pitch16(width)) : 0; }

// Row blocks of the error passes: about 1024 blocks of 1024 columns in all, of 16 rows or more.
int error_blocks(long long M, long long N) {
  const long long strips = (N + 1023) / 1024, most = strips >= 1024 ? 1 : 1024 / strips, want = (M + 15) / 16;
  return (int)(want < most ? want : most);
}

}  // namespace

int niti_launch_pad_pitch(niti_ctx *ctx, cudaStream_t st, const int8_t *src, int8_t *dst, long long rows, int n, int pitch);
int niti_launch_column_sums(niti_ctx *ctx, cudaStream_t st, const float *part, float *dst, int n, int C);

size_t niti_linear_act_ws_bytes(int op, long long M, long long N, long long K) {
  size_t b = NITI_WS_HEADER + pad_bytes(M, K) + pad_bytes(N, K) + (size_t)NITI_LINEAR_MAX_SMS * BM * 256 * 4;
  if (op == NITI_OP_LINEAR_ACT_BWD) b += 256 + up256((size_t)error_blocks(M, N) * (size_t)N * 4) + up256((size_t)M * (size_t)pitch16(N));
  return b;
}

// Longest contraction whose int32 sums cannot wrap (127^2 a term).
#define NITI_LINEAR_MAX_K 131072

static int linear_args(niti_ctx *ctx, const char *name, int type, int M, int N, int K, int act, const void *a, const void *w, long long contraction,
                       void *ws, size_t ws_bytes, int op) {
  if (!niti_type_ok(type) || M < 0 || N <= 0 || K <= 0 || act < NITI_ACT_NONE || act > NITI_ACT_SILU) {
    snprintf(ctx->err, sizeof(ctx->err), "%s: bad argument (type, activation, or a size that is not positive)", name);
    return NITI_ERR_ARG;
  }
  if (M > (1 << 30) || N > (1 << 30) || K > (1 << 30) || contraction > NITI_LINEAR_MAX_K) {
    snprintf(ctx->err, sizeof(ctx->err), "%s: a sum over more than %d products could leave int32", name, NITI_LINEAR_MAX_K);
    return NITI_ERR_SHAPE;
  }
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < niti_linear_act_ws_bytes(op, M, N, K))
    return niti_fail(ctx, NITI_ERR_WORKSPACE, "workspace missing, misaligned or too small");
  if (M > 0 && (!a || !w || (((uintptr_t)a | (uintptr_t)w) & 15))) {
    snprintf(ctx->err, sizeof(ctx->err), "%s: bad argument (a and w must be 16-byte aligned)", name);
    return NITI_ERR_ARG;
  }
  return NITI_OK;
}

extern "C" int niti_linear_act_fwd(niti_ctx *ctx, void *stream, const int8_t *a, const int32_t *s_a, int row_exponents, const int8_t *w,
                                   const int32_t *s_w, const float *bias, const void *residual, void *out, void *z, int type, int M, int N, int K,
                                   int act, void *ws, size_t ws_bytes) {
  if (!ctx) return NITI_ERR_ARG;
  int rc = linear_args(ctx, "niti_linear_act_fwd", type, M, N, K, act, a, w, K, ws, ws_bytes, NITI_OP_LINEAR_ACT_FWD);
  if (rc != NITI_OK || M == 0) return rc;
  const uintptr_t es = (uintptr_t)niti_type_size(type);
  if (!s_a || !s_w || !out || (((uintptr_t)s_a | (uintptr_t)s_w | (uintptr_t)bias) & 3) ||
      (((uintptr_t)residual | (uintptr_t)out | (uintptr_t)z) & (es - 1)) || z == out || (z && z == residual))
    return niti_fail(ctx, NITI_ERR_ARG, "niti_linear_act_fwd: bad argument (z has a place of its own; pointers are aligned to their type)");
  cudaStream_t st = (cudaStream_t)stream;
  const LinearEpilogue e = {s_a, s_w, bias, residual, out, z, row_exponents ? 1 : 0, act};
  if (M <= NITI_LINEAR_ROWS) return niti_linear_rows(ctx, st, a, w, M, N, K, e, type);
  int8_t *pad = (int8_t *)ws + NITI_WS_HEADER;
  int *slabs = (int *)(pad + pad_bytes(M, K) + pad_bytes(N, K));
  const int pitch = (int)pitch16(K);
  if (pitch != K) {
    if ((rc = niti_launch_pad_pitch(ctx, st, a, pad, M, K, pitch)) != NITI_OK) return rc;
    if ((rc = niti_launch_pad_pitch(ctx, st, w, pad + pad_bytes(M, K), N, K, pitch)) != NITI_OK) return rc;
    a = pad;
    w = pad + pad_bytes(M, K);
  }
  WsHeader *hdr = niti_take_header(ctx, st, ws), *next = nullptr;
  if ((rc = niti_clear(ctx, st, nullptr, 0, &next)) != NITI_OK) return rc;
  rc = niti_linear_gemm(ctx, st, GK_FC_FWD, a, pitch, w, pitch, M, N, K, e, type, slabs, niti_split_max(hdr), next);
  if (rc == NITI_OK) niti_header_passed_on(ctx, next);
  return rc;
}

extern "C" int niti_linear_act_bwd(niti_ctx *ctx, void *stream, const int8_t *a, const int32_t *s_a, const int8_t *w, const int32_t *s_w,
                                   const void *z, const void *dout, void *dx, void *dw, float *dbias, int type, int dw_type, int M, int N, int K,
                                   int act, int round_mode, void *ws, size_t ws_bytes) {
  if (!ctx) return NITI_ERR_ARG;
  int rc = linear_args(ctx, "niti_linear_act_bwd", type, M, N, K, act, a, w, M > N ? M : N, ws, ws_bytes, NITI_OP_LINEAR_ACT_BWD);
  if (rc != NITI_OK) return rc;
  const uintptr_t es = (uintptr_t)niti_type_size(type);
  if (!niti_type_ok(dw_type) || (round_mode != NITI_ROUND_PSR && round_mode != NITI_ROUND_NEAREST) || ((uintptr_t)dbias & 3) ||
      ((uintptr_t)dw & (uintptr_t)(niti_type_size(dw_type) - 1)) || (((uintptr_t)dx | (uintptr_t)dout | (uintptr_t)z) & (es - 1)) ||
      (M > 0 && (!s_a || !s_w || !dout || (act != NITI_ACT_NONE && !z) || (((uintptr_t)s_a | (uintptr_t)s_w) & 3))))
    return niti_fail(ctx, NITI_ERR_ARG, "niti_linear_act_bwd: bad argument (an activation needs z; pointers are aligned to their type)");
  if (round_mode == NITI_ROUND_PSR && type != NITI_F32 && (act == NITI_ACT_NONE || act == NITI_ACT_RELU))
    return niti_fail(ctx, NITI_ERR_ARG, "niti_linear_act_bwd: 16-bit errors have too few discarded bits for pseudo-stochastic rounding");
  cudaStream_t st = (cudaStream_t)stream;
  if (M == 0) {
    if (dw) NITI_CUDA_TRY(ctx, cudaMemsetAsync(dw, 0, (size_t)N * K * niti_type_size(dw_type), st));
    if (dbias) NITI_CUDA_TRY(ctx, cudaMemsetAsync(dbias, 0, (size_t)N * 4, st));
    return NITI_OK;
  }
  if (!dx && !dw && !dbias) return NITI_OK;
  const int pitch = (int)pitch16(K), pitch_e = (int)pitch16(N), nblk = error_blocks(M, N);
  int8_t *pad_a = (int8_t *)ws + NITI_WS_HEADER, *pad_w = pad_a + pad_bytes(M, K);
  int *slabs = (int *)(pad_w + pad_bytes(N, K));
  int32_t *s_e = (int32_t *)(slabs + (size_t)NITI_LINEAR_MAX_SMS * BM * 256);
  float *part = (float *)((char *)s_e + 256);
  int8_t *e8 = (int8_t *)part + up256((size_t)nblk * (size_t)N * 4);
  WsHeader *hdr = niti_take_header(ctx, st, ws), *next = nullptr;
  if ((rc = niti_clear(ctx, st, nullptr, 0, &next)) != NITI_OK) return rc;
  const int rows = (M + nblk - 1) / nblk;
  const int v16 = 16 / (int)es;
  const bool vec = N % v16 == 0 && (((uintptr_t)dout | (uintptr_t)z) & 15) == 0;
  auto passes_as = [&](auto tc, auto vc, auto ac) -> int {
    constexpr int T = decltype(tc)::value, VEC = decltype(vc)::value, ACT = decltype(ac)::value;
    const dim3 grid((unsigned)((N + ERR_THREADS * VEC - 1) / (ERR_THREADS * VEC)), (unsigned)((M + rows - 1) / rows));
    NITI_CUDA_TRY(ctx, niti_launch(st, grid, ERR_THREADS, 0, error_max_kernel<T, VEC, ACT>, dout, z, dbias ? part : (float *)nullptr, hdr, next, M, N, rows));
    ctx->launches++;
    niti_header_passed_on(ctx, next);
    if (!dx && !dw) return NITI_OK;
    auto second = [&](auto psr) -> int {
      NITI_CUDA_TRY(ctx, niti_launch(st, grid, ERR_THREADS, 0, error_round_kernel<T, VEC, ACT, decltype(psr)::value>, dout, z, e8, s_e,
                                     (const WsHeader *)hdr, ctx->d_status, M, N, rows, pitch_e));
      ctx->launches++;
      return NITI_OK;
    };
    // (16-bit types without an activation or with a ReLU are not rounded pseudo-stochastically)
    if constexpr (T == NITI_F32 || ACT == NITI_ACT_GELU || ACT == NITI_ACT_SILU)
      if (round_mode == NITI_ROUND_PSR) return second(std::true_type{});
    return second(std::false_type{});
  };
  auto passes = [&](auto tc, auto vc) -> int {
    switch (act) {
      case NITI_ACT_RELU: return passes_as(tc, vc, std::integral_constant<int, NITI_ACT_RELU>{});
      case NITI_ACT_GELU: return passes_as(tc, vc, std::integral_constant<int, NITI_ACT_GELU>{});
      case NITI_ACT_SILU: return passes_as(tc, vc, std::integral_constant<int, NITI_ACT_SILU>{});
      default: return passes_as(tc, vc, std::integral_constant<int, NITI_ACT_NONE>{});
    }
  };
  auto by_type = [&](auto tc) -> int {
    constexpr int T = decltype(tc)::value;
    if (vec) return passes(tc, std::integral_constant<int, 16 / (int)sizeof(typename FloatOf<T>::type)>{});
    return passes(tc, std::integral_constant<int, 1>{});
  };
  rc = type == NITI_F32 ? by_type(std::integral_constant<int, NITI_F32>{}) : type == NITI_BF16 ? by_type(std::integral_constant<int, NITI_BF16>{})
                        : by_type(std::integral_constant<int, NITI_F16>{});
  if (rc != NITI_OK) return rc;
  if (dbias && (rc = niti_launch_column_sums(ctx, st, part, dbias, (M + rows - 1) / rows, N)) != NITI_OK) return rc;
  if (dx) {
    const int8_t *q = w;
    if (pitch != K) {
      if ((rc = niti_launch_pad_pitch(ctx, st, w, pad_w, N, K, pitch)) != NITI_OK) return rc;
      q = pad_w;
    }
    const LinearEpilogue e = {s_e, s_w, nullptr, nullptr, dx, nullptr, 0, NITI_ACT_NONE};
    if ((rc = niti_linear_gemm(ctx, st, GK_FC_DGRAD, e8, pitch_e, q, pitch, M, K, N, e, type, slabs, niti_split_max(hdr), nullptr)) != NITI_OK) return rc;
  }
  if (dw) {
    const int8_t *q = a;
    if (pitch != K) {
      if ((rc = niti_launch_pad_pitch(ctx, st, a, pad_a, M, K, pitch)) != NITI_OK) return rc;
      q = pad_a;
    }
    const LinearEpilogue e = {s_e, s_a, nullptr, nullptr, dw, nullptr, 0, NITI_ACT_NONE};
    if ((rc = niti_linear_gemm(ctx, st, GK_FC_WGRAD, e8, pitch_e, q, pitch, N, K, M, e, dw_type, slabs, niti_split_max(hdr) + NITI_LINEAR_COUNTERS,
                               nullptr)) != NITI_OK)
      return rc;
  }
  return NITI_OK;
}
