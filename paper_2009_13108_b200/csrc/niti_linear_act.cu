// Fully connected layers whose results leave the integer format in the multiply's epilogue: scale by the operands' exponents,
// bias, activation and residual, stored in 16 or 32 bits; and their backward pass, an error that is rounded to int8 with one
// exponent and the two multiplies that it enters.
#include "niti_act.cuh"
#include "niti_div.h"
#include "niti_linear_act.h"
#include "niti_pad.cuh"
#include "niti_sums.cuh"
#include "niti_tcgen05.cuh"
#include <type_traits>

namespace {

constexpr int BM = 128;                            // rows of a tile = TMEM lanes
constexpr int PROD_WARPS = 3, MMA_WARP = 3, EPI_WARP0 = 4;
constexpr int EPI_WARPS = 16;
constexpr int THREADS = 32 * (EPI_WARP0 + EPI_WARPS);
constexpr int MAX_STAGES = 8, MAX_TBUF = 4;
constexpr int STG_FLOATS = 32 * 33;                // a warp's buffer for rows that are not whole, aligned vectors

// A multiply of a launch.
struct Params {
  int kind;                                        // GK_FC_FWD, GK_FC_DGRAD or GK_FC_WGRAD
  int gm, gn;
  int bn;
  int kdepth, ksteps, kb_total, kb_per_split, splits;
  int a_bytes, b_bytes, a_boxes, b_boxes, a_box_bytes, b_box_bytes, a_box_step, b_box_step;
  unsigned idesc;
  unsigned long long a_desc, b_desc;
  unsigned a_kstep16, b_kstep16;
  int n_tiles_n, m_units, raster_g, last_group, items;
  Div d_split, d_group, d_units, d_last;
  int direct;                                      // rows are whole, aligned pieces of 32 bytes
  int *slabs;                                      // sums of split contractions, and what counts the arrivals of each tile
  unsigned *counters;
  LinearEpilogue e;
};
// A launch: one multiply (forward), or the two of a backward pass, whose items follow one another.
template <int N>
struct Launch {
  Params p[N];
  int items;
  int nbuf, bn_most, tmem_cols;                    // accumulators of bn_most columns
  int stages, nprod, stage_bytes;
  int stg_off;                                     // byte offset of the warps' buffers, behind the stages
};
template <int N>
struct Maps { CUtensorMap a[N], b[N]; };

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

// The copies of a k-block: A and B of this CTA from row m0 / column n0 and contraction element k.
template <int KIND, int CTAS>
__device__ __forceinline__ void copy_kblock(const Params &p, const CUtensorMap *ma, const CUtensorMap *mb, unsigned sa, unsigned full, int m0, int n0, int k) {
  const unsigned sb = sa + p.a_bytes;
  if (KIND == GK_FC_WGRAD) {
    for (int j = 0; j < p.a_boxes; ++j) load2<CTAS>(sa + j * p.a_box_bytes, ma, full, m0 + j * p.a_box_step, k);
  } else {
    load2<CTAS>(sa, ma, full, k, m0);
  }
  if (KIND == GK_FC_FWD) {
    load2<CTAS>(sb, mb, full, k, n0);
  } else {
    for (int j = 0; j < p.b_boxes; ++j) load2<CTAS>(sb + j * p.b_box_bytes, mb, full, n0 + j * p.b_box_step, k);
  }
}

// One persistent CTA (or pair on a 256-row tile) per SM; warps 0 - 2 copy, warp 3 multiplies, the others finish tiles.  The
// pipeline is the one of the integer layers' kernel; nothing here depends on the whole tensor, so that a tile is final when
// its sums are.  A contraction that is split over CTAs leaves its sums in slabs; the CTA that comes last adds them up, in the
// order of the splits (integers: any order gives the same), and finishes the tile.
// N = 2: the error's and the weights' multiply of a backward pass in one launch, whose tiles share the SMs (one after the
// other they left a seventh of them idle, twice, and each its first copies and its last epilogue uncovered: 4096 x 4096 x 1024
// 19 + 19 -> 30 us, 2000 x 520 x 777 15 + 15 -> 17).
// 8192 x 8192 x 8192 with bias, GELU, residual and z: 336 us alone, 3.27 POP/s, the tensor pipe busy for 90 % of it at the 1.5 GHz
// that the power cap leaves; in a long run 420 - 450.  Short contractions are bound by the epilogue, 11 instructions an
// element without an activation, 20 with SiLU, 23 with GELU: 4096 x 4096 x 1024 23, 28 and 30 us (with eight epilogue warps instead
// of sixteen 26 without one).
// (Measured and left out: outputs through shared memory in whole 128-byte rows, 4096 x 4096 x 128 16 -> 16 us and 8192^3 365 ->
// 400 for the stages that the buffers cost; copies by six threads instead of three, 11.7 -> 11.2 us at 64 x 4096 x 4096, slower
// elsewhere; sums turned into floats by integer additions, 25 -> 27 us.)
template <int N, int CTAS, int T0, int T1>
__global__ void __launch_bounds__(THREADS, 1)
linear_kernel(const __grid_constant__ Maps<N> maps, const __grid_constant__ Launch<N> g, WsHeader *next, uint32_t *status) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ __align__(8) unsigned long long bars[2 * MAX_STAGES + 2 * MAX_TBUF];
  __shared__ unsigned tmem_slot;
  __shared__ volatile int abort_flag;
  __shared__ int is_last;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = (int)threadIdx.x & 31;
  const unsigned rank = CTAS == 2 ? cluster_ctarank() : 0u;
  const unsigned smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const unsigned full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[MAX_STAGES]);
  const unsigned tfull0 = smem_u32(&bars[2 * MAX_STAGES]), tempty0 = smem_u32(&bars[2 * MAX_STAGES + MAX_TBUF]);
  const unsigned lead_full0 = CTAS == 2 ? map_to_cta(full0, 0) : full0;
  const unsigned lead_tempty0 = CTAS == 2 ? map_to_cta(tempty0, 0) : tempty0;
  const int first_item = (int)blockIdx.x / CTAS, item_step = (int)gridDim.x / CTAS;

  if (warp == 1 && lane < 2 * N && g.p[lane % N].items) {
    const CUtensorMap *m = lane < N ? &maps.a[lane] : &maps.b[lane - N];
    asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
  }
  if (threadIdx.x == 0) abort_flag = 0;
  if (threadIdx.x < 2 * MAX_STAGES + 2 * MAX_TBUF) {
    mbar_init(smem_u32(&bars[threadIdx.x]), threadIdx.x >= 2 * MAX_STAGES + MAX_TBUF ? EPI_WARPS * CTAS : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == MMA_WARP) {
    if (CTAS == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"((unsigned)g.tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"((unsigned)g.tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync_all();
  tc_fence_after();
  const unsigned tmem_base = tmem_slot;
  niti_enter(next);
  if (next && blockIdx.x == 0 && warp == EPI_WARP0 + EPI_WARPS - 1) niti_zero_header(next, lane);

  if (warp < PROD_WARPS) {
    const bool leader = elect_one();
    int stage = 0, owner = 0;
    unsigned phase = 0;
    bool ok = true;
    for (int item = first_item; ok && item < g.items; item += item_step) {
      const int which = N == 2 && item >= g.p[0].items ? 1 : 0;
      const Params &p = g.p[which];
      int mu, nt, split, tile;
      decode(p, which ? item - g.p[0].items : item, mu, nt, split, tile);
      const int bn_cta = p.bn / CTAS, m0 = (mu * CTAS + (int)rank) * BM, n0 = nt * p.bn + (int)rank * bn_cta;
      const int kb0 = split * p.kb_per_split, kb1 = min(kb0 + p.kb_per_split, p.kb_total);
      const unsigned tx = (unsigned)(CTAS * (p.a_boxes * p.a_box_bytes + p.b_boxes * p.b_box_bytes));
      for (int kb = kb0; kb < kb1; ++kb) {
        if (owner == warp) {
          if (!mbar_wait_warp(empty0 + 8 * stage, phase ^ 1, &abort_flag, status)) { ok = false; break; }
          if (leader) {
            const unsigned full = lead_full0 + 8 * stage, sa = smem_base + stage * g.stage_bytes;
            if (rank == 0) mbar_expect_tx(full0 + 8 * stage, tx);
            const int k = kb * p.kdepth;
            if (N == 1) copy_kblock<GK_FC_FWD, CTAS>(p, &maps.a[0], &maps.b[0], sa, full, m0, n0, k);
            else if (p.kind == GK_FC_DGRAD) copy_kblock<GK_FC_DGRAD, CTAS>(p, &maps.a[which], &maps.b[which], sa, full, m0, n0, k);
            else copy_kblock<GK_FC_WGRAD, CTAS>(p, &maps.a[which], &maps.b[which], sa, full, m0, n0, k);
          }
        }
        if (++owner == g.nprod) owner = 0;
        if (++stage == g.stages) { stage = 0; phase ^= 1; }
      }
    }
  } else if (warp == MMA_WARP) {
    if (rank == 0) {
      const bool leader = elect_one();
      int stage = 0;
      unsigned phase = 0, buf = 0, par = 0;
      bool ok = true;
      for (int item = first_item; ok && item < g.items; item += item_step) {
        const int which = N == 2 && item >= g.p[0].items ? 1 : 0;
        const Params &p = g.p[which];
        const int in = which ? item - g.p[0].items : item;
        const unsigned a_lo0 = (unsigned)p.a_desc, b_lo0 = (unsigned)p.b_desc, a_hi = (unsigned)(p.a_desc >> 32), b_hi = (unsigned)(p.b_desc >> 32);
        const unsigned ak = p.a_kstep16, bk = p.b_kstep16, idesc = p.idesc, a_bytes = (unsigned)p.a_bytes;
        const int ksteps = p.ksteps;
        const int split = p.splits > 1 ? in - div_by(in, p.d_split) * p.splits : 0;
        const int kb0 = split * p.kb_per_split, kb1 = min(kb0 + p.kb_per_split, p.kb_total);
        if (!mbar_wait_warp(tempty0 + 8 * buf, par ^ 1u, &abort_flag, status)) { ok = false; break; }
        const unsigned tfull = tfull0 + 8 * buf, tmem_d = tmem_base + buf * (unsigned)g.bn_most;
        if (++buf == (unsigned)g.nbuf) { buf = 0; par ^= 1u; }
        tc_fence_after();
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait_warp(full0 + 8 * stage, phase, &abort_flag, status)) { ok = false; break; }
          tc_fence_after();
          const unsigned sa = smem_base + stage * g.stage_bytes;
          const unsigned a_lo = a_lo0 + ((sa >> 4) & 0x3fff), b_lo = b_lo0 + (((sa + a_bytes) >> 4) & 0x3fff);
          const unsigned acc = kb > kb0 ? 1u : 0u;
          if (leader) {
            if (ksteps == 4) issue_kblock<CTAS, 4>(tmem_d, a_lo, a_hi, b_lo, b_hi, ak, bk, idesc, acc);
            else if (ksteps == 2) issue_kblock<CTAS, 2>(tmem_d, a_lo, a_hi, b_lo, b_hi, ak, bk, idesc, acc);
            else issue_kblock<CTAS, 1>(tmem_d, a_lo, a_hi, b_lo, b_hi, ak, bk, idesc, acc);
            if (CTAS == 2) tc_commit_pair(empty0 + 8 * stage); else tc_commit(empty0 + 8 * stage);
          }
          if (++stage == g.stages) { stage = 0; phase ^= 1; }
        }
        if (ok && leader) {
          if (CTAS == 2) tc_commit_pair(tfull); else tc_commit(tfull);
        }
      }
    }
  } else {
    const int ew = warp - EPI_WARP0, quarter = warp & 3, part = ew >> 2;
    float *stg = reinterpret_cast<float *>(smem_raw + (smem_base - smem_u32(smem_raw)) + g.stg_off) + ew * STG_FLOATS;
    unsigned buf = 0, par = 0;
    bool wide_exp = false;
    for (int item = first_item; item < g.items; item += item_step) {
      const int which = N == 2 && item >= g.p[0].items ? 1 : 0;
      const Params &p = g.p[which];
      const LinearEpilogue &e = p.e;
      int mu, nt, split, tile;
      decode(p, which ? item - g.p[0].items : item, mu, nt, split, tile);
      const int row0 = (mu * CTAS + (int)rank) * BM + 32 * quarter, n0 = nt * p.bn;
      const int row = row0 + lane < p.gm ? row0 + lane : p.gm - 1;
      const int s = e.s0[e.s0_rows ? row : 0] + *e.s1;
      wide_exp |= s < -128 || s > 127;
      const float f = linear_scale(s);
      bool ok = mbar_wait_warp(tfull0 + 8 * buf, par, &abort_flag, status);
      if (p.splits > 1) ok = epilogue_all(ok);     // (they meet at barriers below: all go on, or none)
      if (!ok) break;
      tc_fence_after();
      const unsigned tm = tmem_base + buf * (unsigned)g.bn_most + ((unsigned)(32 * quarter) << 16);
      const unsigned tempty = lead_tempty0 + 8 * buf;
      if (++buf == (unsigned)g.nbuf) { buf = 0; par ^= 1u; }
      auto drained = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) { if (CTAS == 2) mbar_arrive_cluster(tempty); else mbar_arrive(tempty); }
      };
      auto finish = [&](int (&v)[32], int c) {
        if (T0 == T1 || which == 0) finish_chunk<T0>(p, v, row0, n0 + 32 * c, f, stg, lane);
        else finish_chunk<T1>(p, v, row0, n0 + 32 * c, f, stg, lane);
      };
      if (p.splits == 1) {
        for (int c = part; c < p.bn / 32; c += EPI_WARPS / 4) {
          int v[32];
          if (n0 + 32 * c < p.gn) {
            tc_ld32(tm + 32u * (unsigned)c, v);
            finish(v, c);
          }
        }
        drained();
        continue;
      }
      // a share of a split contraction: 32 columns x 128 rows of sums in column order
      const int slot = tile * CTAS + (int)rank, words = p.bn * BM;
      int *mine = p.slabs + ((long long)slot * p.splits + split) * words + 32 * quarter + lane;
      for (int c = part; c < p.bn / 32; c += EPI_WARPS / 4) {
        if (row0 >= p.gm || n0 + 32 * c >= p.gn) continue;           // (nobody reads them)
        int v[32];
        tc_ld32(tm + 32u * (unsigned)c, v);
#pragma unroll
        for (int j = 0; j < 32; ++j) mine[(32 * c + j) * BM] = v[j];
      }
      drained();
      __threadfence();
      asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory");
      if (ew == 0 && lane == 0) {
        const unsigned before = atomicAdd(p.counters + slot, 1u);
        __threadfence();
        is_last = before == (unsigned)p.splits - 1u;
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory");
      if (is_last) {
        const int *all = p.slabs + (long long)slot * p.splits * words + 32 * quarter + lane;
        for (int c = part; c < p.bn / 32; c += EPI_WARPS / 4) {
          if (row0 >= p.gm || n0 + 32 * c >= p.gn) continue;
          int v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0;
#pragma unroll 2
          for (int k = 0; k < p.splits; ++k) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += __ldcg(all + (long long)k * words + (32 * c + j) * BM);
          }
          finish(v, c);
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
    if (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((unsigned)g.tmem_cols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((unsigned)g.tmem_cols) : "memory");
  }
}

// ---- host ------------------------------------------------------------------------------------
// Cycles of a k-block of 128 contraction elements: multiplies, or the operand copies (constants as measured for the integer
// layers' kernel: 84 bytes a clock into one SM, 9000 into all).
bool direct_rows(const LinearMultiply &x) {
  const uintptr_t ptrs = (uintptr_t)x.e.out | (uintptr_t)x.e.res | (uintptr_t)x.e.z;
  return (x.gn * niti_type_size(x.type)) % 32 == 0 && (ptrs & 31) == 0 && ((uintptr_t)x.e.bias & 15) == 0;
}
double kblock_cycles(int ctas, int bn, int ksteps, long long running) {
  const double mma = bn / 2.0, smem = 32.0 + bn / (4.0 * ctas), bytes = (128.0 + (double)bn / ctas) * 32.0 * ksteps;
  double c = ksteps * (mma > smem ? mma : smem);
  if (c < bytes / 84.0) c = bytes / 84.0;
  if (c < bytes * (double)running / 9000.0) c = bytes * (double)running / 9000.0;
  return c < 100.0 * ksteps ? 100.0 * ksteps : c;
}

struct Choice { int bn, splits; double cycles; };
// Tile width and splits with the least modelled time on `units` CTAs (pairs): k-blocks of a wave, the epilogue of its tiles
// (issue slots an element, hidden behind the next tile's main loop), and for splits the slabs' way through L2.
Choice choose(const niti_ctx *ctx, const LinearMultiply &x, int ctas, long long units, double epi_slots) {
  Choice best = {32, 1, 1e300};
  const int kdepth = pick_swizzle(x.gk), ksteps = kdepth / 32, kb = (int)((x.gk + kdepth - 1) / kdepth);
  const long long mu = ((x.gm + BM - 1) / BM + ctas - 1) / ctas;
  const int unit = x.kind == GK_FC_FWD ? 32 : 64;
  for (int bn = 256; bn >= unit; bn -= unit) {
    if (bn > unit && bn - unit >= x.gn) continue;
    if (bn / ctas % 16) continue;
    const long long tiles = mu * ((x.gn + bn - 1) / bn);
    const double epi = epi_slots * bn;
    for (int s = 1; s <= 32; s += s < 4 ? 1 : s < 8 ? 2 : 4) {
      if (s > 1 && (tiles * s > units || kb / s < 4 || tiles * ctas > NITI_LINEAR_COUNTERS || ctx->sm_count > NITI_LINEAR_MAX_SMS)) break;
      const long long items = tiles * s, waves = (items + units - 1) / units;
      const double main = ((kb + s - 1) / s) * kblock_cycles(ctas, bn, ksteps, (items < units ? items : units) * ctas);
      double t = main + (double)(waves - 1) * (main > epi ? main : epi) + epi + (ctas == 2 ? 1500.0 : 0.0);
      if (s > 1) t += 3000.0 + 8.0 * bn * (s + 1);
      if (t < best.cycles * 0.98) best = {bn, s, t};
    }
  }
  return best;
}

// The same for the sizes of an earlier call: the search takes longer than a small multiply.
Choice chosen(niti_ctx *ctx, const LinearMultiply &x, int ctas, long long units, bool direct) {
  const long long key[4] = {x.gm, x.gn, x.gk, ((x.kind * 2LL + direct) * 2 + ctas - 1) * 1024 + units};
  unsigned long long h = 0;
  for (int i = 0; i < 4; ++i) h = (h ^ (unsigned long long)key[i]) * 0x9E3779B97F4A7C15ull;
  NitiLinearPlan &e = ctx->linear_plans[(h >> 32) % NITI_LINEAR_PLANS];
  if (memcmp(e.key, key, sizeof(key)) != 0 || !e.bn) {
    const Choice c = choose(ctx, x, ctas, units, direct ? 20.0 : 40.0);
    memcpy(e.key, key, sizeof(key));
    e.bn = c.bn;
    e.splits = c.splits;
    e.cycles = c.cycles;
  }
  return Choice{e.bn, e.splits, e.cycles};
}

template <int N, int CTAS, int T0, int T1>
int set_up(niti_ctx *ctx) {
  // (per device and instance, the same value in every context: see niti_ctx::smem_optin)
  bool &ready = ctx->linear_ready[((N - 1) * 2 + CTAS - 1) * 9 + 3 * T0 + T1];
  if (ready) return NITI_OK;
  cudaFuncAttributes fa;
  NITI_CUDA_TRY(ctx, cudaFuncGetAttributes(&fa, linear_kernel<N, CTAS, T0, T1>));
  NITI_CUDA_TRY(ctx, cudaFuncSetAttribute(linear_kernel<N, CTAS, T0, T1>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                          (int)(ctx->smem_optin - fa.sharedSizeBytes)));
  ready = true;
  return NITI_OK;
}

// CTA pairs that run at once (SMs pair up inside a GPC, so there can be fewer than half of the SMs).
int ask_pairs(niti_ctx *ctx) {
  if (ctx->linear_pairs) return NITI_OK;
  const int rc = set_up<1, 2, NITI_BF16, NITI_BF16>(ctx);
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
  NITI_CUDA_TRY(ctx, cudaOccupancyMaxActiveClusters(&n, linear_kernel<1, 2, NITI_BF16, NITI_BF16>, &cfg));
  ctx->linear_pairs = n < 1 ? 1 : n < ctx->sm_count / 2 ? n : ctx->sm_count / 2;
  return NITI_OK;
}

template <int N, int CTAS, int T0, int T1>
int launch_as(niti_ctx *ctx, cudaStream_t st, const Launch<N> &g, const Maps<N> &maps, size_t smem, unsigned grid, WsHeader *next) {
  const int rc = set_up<N, CTAS, T0, T1>(ctx);
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
  NITI_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, linear_kernel<N, CTAS, T0, T1>, maps, g, next, ctx->d_status));
  ctx->launches++;
  ctx->tc_launches++;
  if (CTAS == 2) ctx->tc2_launches++;
  return NITI_OK;
}

// Parameters and tensor maps of one multiply; false: an operand has no tensor map.
bool fill(niti_ctx *ctx, const LinearMultiply &x, int ctas, const Choice &c, Params &p, CUtensorMap &ma, CUtensorMap &mb) {
  p.kind = x.kind;
  p.gm = (int)x.gm; p.gn = (int)x.gn;
  p.e = x.e;
  p.bn = c.bn;
  p.kdepth = pick_swizzle(x.gk);
  p.ksteps = p.kdepth / 32;
  p.kb_total = (int)((x.gk + p.kdepth - 1) / p.kdepth);
  p.kb_per_split = (p.kb_total + c.splits - 1) / c.splits;
  p.splits = (p.kb_total + p.kb_per_split - 1) / p.kb_per_split;
  const int bn_cta = p.bn / ctas;
  MapSpec sa, sb;
  memset(&sa, 0, sizeof(sa));
  memset(&sb, 0, sizeof(sb));
  const bool a_mn = x.kind == GK_FC_WGRAD, b_mn = x.kind != GK_FC_FWD;
  int a_sw = p.kdepth, b_sw = p.kdepth;
  if (a_mn) {
    a_sw = pick_swizzle(x.gm);
    sa = {2, {(cuuint64_t)x.gm, (cuuint64_t)x.gk}, {(cuuint64_t)x.ld0}, {(cuuint32_t)a_sw, (cuuint32_t)p.kdepth}, a_sw, x.p0};
    p.a_boxes = BM / a_sw;
    if ((long long)p.a_boxes * a_sw > (x.gm + a_sw - 1) / a_sw * a_sw) p.a_boxes = (int)((x.gm + a_sw - 1) / a_sw);
    p.a_box_bytes = p.kdepth * a_sw;
    p.a_box_step = a_sw;
    p.a_bytes = (BM / a_sw) * p.a_box_bytes;
    p.a_desc = desc_mnmajor(a_sw, p.kdepth);
    p.a_kstep16 = (unsigned)((32 * a_sw) >> 4);
  } else {
    sa = {2, {(cuuint64_t)x.gk, (cuuint64_t)x.gm}, {(cuuint64_t)x.ld0}, {(cuuint32_t)p.kdepth, BM}, a_sw, x.p0};
    p.a_boxes = 1;
    p.a_box_bytes = p.a_bytes = BM * p.kdepth;
    p.a_desc = desc_kmajor(a_sw);
    p.a_kstep16 = 2;
  }
  if (b_mn) {
    b_sw = pick_swizzle_mn(bn_cta);
    sb = {2, {(cuuint64_t)x.gn, (cuuint64_t)x.gk}, {(cuuint64_t)x.ld1}, {(cuuint32_t)b_sw, (cuuint32_t)p.kdepth}, b_sw, x.p1};
    p.b_boxes = (bn_cta + b_sw - 1) / b_sw;
    p.b_box_bytes = p.kdepth * b_sw;
    p.b_box_step = b_sw;
    p.b_bytes = p.b_boxes * p.b_box_bytes;
    p.b_desc = desc_mnmajor(b_sw, p.kdepth);
    p.b_kstep16 = (unsigned)((32 * b_sw) >> 4);
  } else {
    sb = {2, {(cuuint64_t)x.gk, (cuuint64_t)x.gn}, {(cuuint64_t)x.ld1}, {(cuuint32_t)p.kdepth, (cuuint32_t)bn_cta}, b_sw, x.p1};
    p.b_boxes = 1;
    p.b_box_bytes = p.b_bytes = bn_cta * p.kdepth;
    p.b_desc = desc_kmajor(b_sw);
    p.b_kstep16 = 2;
  }
  p.a_bytes = (p.a_bytes + 1023) / 1024 * 1024;
  p.b_bytes = (p.b_bytes + 1023) / 1024 * 1024;
  p.direct = direct_rows(x) ? 1 : 0;
  // instruction descriptor: s32 accumulate, signed 8-bit operands, majorness, N, M
  p.idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((unsigned)a_mn << 15) | ((unsigned)b_mn << 16) | ((unsigned)(p.bn >> 3) << 17) |
            ((unsigned)((BM * ctas) >> 4) << 24);
  const long long mt = (x.gm + BM - 1) / BM;
  p.m_units = (int)((mt + ctas - 1) / ctas);
  p.n_tiles_n = (int)((x.gn + p.bn - 1) / p.bn);
  p.items = (int)((long long)p.m_units * p.n_tiles_n * p.splits);
  p.raster_g = ctas == 2 ? 8 : 12;
  p.last_group = (p.m_units - 1) / p.raster_g;
  p.d_split = make_div(p.splits);
  p.d_group = make_div((long long)p.raster_g * p.n_tiles_n);
  p.d_units = make_div(p.raster_g);
  p.d_last = make_div(p.m_units - p.last_group * p.raster_g);
  return encode(ctx, &ma, sa) && encode(ctx, &mb, sb);
}

template <int N>
int run_multiplies(niti_ctx *ctx, cudaStream_t st, const LinearMultiply *x, int *slabs, unsigned *counters, WsHeader *next) {
  int rc = ask_pairs(ctx);
  if (rc != NITI_OK) return rc;
  // each of two multiplies is planned for its share of the SMs (they have the same number of operations)
  Choice c[2][N];
  double cycles[2] = {0.0, 0.0};
  int wanted = 0;
  for (int i = 0; i < N; ++i) wanted += x[i].e.out ? 1 : 0;
  for (int ctas = 1; ctas <= 2; ++ctas)
    for (int i = 0; i < N; ++i) {
      if (!x[i].e.out) continue;
      const long long units = (ctas == 2 ? ctx->linear_pairs : ctx->sm_count) / wanted;
      c[ctas - 1][i] = chosen(ctx, x[i], ctas, units < 1 ? 1 : units, direct_rows(x[i]));
      if (c[ctas - 1][i].cycles > cycles[ctas - 1]) cycles[ctas - 1] = c[ctas - 1][i].cycles;
      if (ctas == 2 && x[i].gm <= BM) cycles[1] = 1e300;
    }
  const int ctas = cycles[1] < cycles[0] ? 2 : 1;
  Launch<N> g;
  Maps<N> maps;
  memset(&g, 0, sizeof(g));
  bool staged = false;
  long long items = 0;
  for (int i = 0; i < N; ++i) {
    Params &p = g.p[i];
    if (((x[i].gm + BM - 1) / BM) * ((x[i].gn + 31) / 32) >= (1LL << 28)) return niti_fail(ctx, NITI_ERR_SHAPE, "linear layer: too many tiles");
    if (!x[i].e.out) {                             // (not wanted)
      memset(&maps.a[i], 0, sizeof(maps.a[i]));
      memset(&maps.b[i], 0, sizeof(maps.b[i]));
      continue;
    }
    if (!fill(ctx, x[i], ctas, c[ctas - 1][i], p, maps.a[i], maps.b[i])) return niti_fail(ctx, NITI_ERR_CUDA, "linear layer: no tensor map for an operand");
    p.slabs = slabs;
    p.counters = counters;
    if (p.splits > 1) {                            // (at most a tile of 128 x 256 words for every SM that the multiply was planned for)
      slabs += (size_t)p.items * ctas * BM * p.bn;
      counters += NITI_LINEAR_COUNTERS;
    }
    items += p.items;
    if (p.a_bytes + p.b_bytes > g.stage_bytes) g.stage_bytes = p.a_bytes + p.b_bytes;
    if (p.bn > g.bn_most) g.bn_most = p.bn;
    staged = staged || !p.direct;
  }
  g.items = (int)items;
  const int stg = staged ? EPI_WARPS * STG_FLOATS * 4 : 0;
  g.stages = (216 * 1024 - stg) / g.stage_bytes;
  if (g.stages > MAX_STAGES) g.stages = MAX_STAGES;
  if (g.stages == 5 || g.stages == 7) g.stages -= 1;
  if (g.stages < 2) return niti_fail(ctx, NITI_ERR_SHAPE, "linear layer: no room for two stages");
  g.stg_off = g.stages * g.stage_bytes;
  g.nprod = 1;
  for (int d = 2; d <= PROD_WARPS; ++d)
    if (g.stages % d == 0) g.nprod = d;
  g.nbuf = 512 / g.bn_most > MAX_TBUF ? MAX_TBUF : 512 / g.bn_most;
  g.tmem_cols = 32;
  while (g.tmem_cols < g.nbuf * g.bn_most) g.tmem_cols <<= 1;
  const size_t smem = (size_t)g.stg_off + stg + 1024;
  const long long units = ctas == 2 ? ctx->linear_pairs : ctx->sm_count;
  const unsigned grid = (unsigned)((items < units ? items : units) * ctas);
  auto go = [&](auto t0, auto t1) -> int {
    constexpr int T0 = decltype(t0)::value, T1 = decltype(t1)::value;
    return ctas == 2 ? launch_as<N, 2, T0, T1>(ctx, st, g, maps, smem, grid, next) : launch_as<N, 1, T0, T1>(ctx, st, g, maps, smem, grid, next);
  };
  auto with = [](int type, auto f) -> int {
    if (type == NITI_F32) return f(std::integral_constant<int, NITI_F32>{});
    if (type == NITI_BF16) return f(std::integral_constant<int, NITI_BF16>{});
    return f(std::integral_constant<int, NITI_F16>{});
  };
  return with(x[0].type, [&](auto t0) -> int {
    if constexpr (N == 1) return go(t0, t0);
    else return with(x[N - 1].type, [&](auto t1) -> int { return go(t0, t1); });
  });
}

}  // namespace

// ---- the error of the backward pass ---------------------------------------------------------
namespace {

constexpr int ERR_THREADS = 128;
constexpr unsigned INF_BITS = 0x7f800000u;

// e = dout act'(z) of a block's rows and columns, a thread on the same VEC columns in every row; two rows at work and two on
// their way.
template <int T, int VEC, int ACT, bool KEEP, typename F>
__device__ __forceinline__ void error_rows(const void *dout, const void *z, int N, int r0, int r1, int c, F take) {
  constexpr int DEEP = 2;
  Pack<T, VEC> d[2][DEEP], zz[2][DEEP];
  auto fetch = [&](int r, Pack<T, VEC> (&dd)[DEEP], Pack<T, VEC> (&zd)[DEEP]) {
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
      if (r + k < r1) {
        dd[k].template load<KEEP>(dout, (long long)(r + k) * N + c);
        if (ACT != NITI_ACT_NONE) zd[k].template load<KEEP>(z, (long long)(r + k) * N + c);
      }
  };
  auto work = [&](int r, const Pack<T, VEC> (&dd)[DEEP], const Pack<T, VEC> (&zd)[DEEP]) {
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
      if (r + k < r1) {
        float e[VEC];
        if constexpr (ACT == NITI_ACT_NONE) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) e[j] = dd[k].get(j);
        } else {
          float dv[VEC], zv[VEC];
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            dv[j] = dd[k].get(j);
            zv[j] = zd[k].get(j);
          }
          act_backward<ACT>(dv, zv, e);
        }
        take(r + k, e);
      }
  };
  fetch(r0, d[0], zz[0]);
  for (int r = r0; r < r1; r += 2 * DEEP) {
    fetch(r + DEEP, d[1], zz[1]);
    work(r, d[0], zz[0]);
    fetch(r + 2 * DEEP, d[0], zz[0]);
    work(r + DEEP, d[1], zz[1]);
  }
}

// How the blocks of the error passes are dealt: `strips` column strips times row blocks of `rows` rows, then what else a pass
// does beside them.
struct ErrorGrid { int strips, rows, main; };

// Largest |e| of the tensor, and the column sums of every block's rows; beside them, operands whose rows have to be padded for
// the multiplies.  Bound: HBM and, with an activation, the exponentials and reciprocals of its slope (dout and z are read once
// here; the rounding pass finds what fits of them in L2).  4096 x 4096 bfloat16 with GELU: 67 MB in 18.5 us from HBM, the
// rounding pass 22 where nothing is in L2; with SiLU 17 and 20.5 (one instance with the activation looked up for every element
// took 31 and 39).  A pass that keeps e instead of computing it again would have to keep it in 32 bits, as many
// bytes as both operands.
template <int T, int VEC, int ACT>
__global__ void __launch_bounds__(ERR_THREADS, 8)
error_max_kernel(const void *dout, const void *z, float *part, WsHeader *hdr, WsHeader *next, uint32_t *status, int M, int N, ErrorGrid g,
                 PadJob pad0, PadJob pad1, unsigned pad0_blocks) {
  niti_enter(dout, z, pad0.src, pad1.src);
  if ((int)blockIdx.x >= g.main) {
    const unsigned b = blockIdx.x - (unsigned)g.main, all = gridDim.x - (unsigned)g.main;
    if (b < pad0_blocks) niti_pad_rows(pad0, b, pad0_blocks);
    else niti_pad_rows(pad1, b - pad0_blocks, all - pad0_blocks);
    return;
  }
  const int by = (int)blockIdx.x / g.strips, bx = (int)blockIdx.x - by * g.strips;
  const int c = (bx * ERR_THREADS + (int)threadIdx.x) * VEC, r0 = by * g.rows, r1 = min(r0 + g.rows, M);
  if (next && blockIdx.x == 0 && threadIdx.x < 32) niti_zero_header(next, (int)threadIdx.x);
  float sum[VEC];
  float largest = 0.0f;
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] = 0.0f;
  if (c < N) {
    error_rows<T, VEC, ACT, true>(dout, z, N, r0, r1, c, [&](int, const float (&e)[VEC]) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        sum[j] += e[j];
        largest = niti_absmax(largest, e[j]);
      }
    });
    if (part) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) part[(long long)by * N + c + j] = sum[j];
    }
  }
  const unsigned most = __reduce_max_sync(0xffffffffu, __float_as_uint(largest));
  if ((threadIdx.x & 31) == 0 && most) atomicMax(&hdr->maxabs32, most);
  if ((threadIdx.x & 31) == 0 && most >= INF_BITS) atomicOr(status, NITI_DEV_NONFINITE);
}

// The bias gradient of 32 columns from the row blocks' column sums.
__device__ __forceinline__ void bias_sums(const float *part, float *dbias, int nblk, int N, int block) {
  __shared__ float buf[16 * 33];
  if (N % 4 == 0) niti_column_sums<4, 16>(part, dbias, nblk, N, block, buf);
  else niti_column_sums<1, 4>(part, dbias, nblk, N, block, buf);
}
// Where no multiply follows; the order of the sums is the same.
__global__ void __launch_bounds__(ERR_THREADS)
bias_sum_kernel(const float *part, float *dbias, int nblk, int N) {
  niti_enter(part);
  bias_sums(part, dbias, nblk, N, (int)blockIdx.x);
}

// e as payload with the exponent of its maximum, rows of `pitch` bytes.  The rows that the pass before read last come first.
// Beside it, the bias gradient from that pass' column sums (of `nblk` row blocks).
template <int T, int VEC, int ACT, bool PSR>
__global__ void __launch_bounds__(ERR_THREADS, 8)
error_round_kernel(const void *dout, const void *z, int8_t *e8, int32_t *s_e, const WsHeader *hdr, int M, int N, ErrorGrid g, int pitch,
                   const float *part, float *dbias, int nblk) {
  niti_enter(dout, z, hdr, part);
  const unsigned most = hdr->maxabs32;
  const int s = niti_exponent_of(most);
  const float scale = niti_payload_scale(niti_pow2(-s), PSR ? NITI_ROUND_PSR : NITI_ROUND_NEAREST);
  if (blockIdx.x == 0 && threadIdx.x == 0) *s_e = s;
  if ((int)blockIdx.x >= g.main) {
    bias_sums(part, dbias, nblk, N, (int)blockIdx.x - g.main);
    return;
  }
  const int b = g.main - 1 - (int)blockIdx.x, by = b / g.strips, bx = b - by * g.strips;
  const int c = (bx * ERR_THREADS + (int)threadIdx.x) * VEC, r0 = by * g.rows, r1 = min(r0 + g.rows, M);
  if (c >= N) return;
  error_rows<T, VEC, ACT, false>(dout, z, N, r0, r1, c, [&](int r, const float (&e)[VEC]) {
    niti_store_payload<VEC, PSR>(e8, (long long)r * pitch + c, e, scale);
  });
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
long long pitch16(long long n) { return (n + 15) / 16 * 16; }
size_t pad_bytes(long long rows, long long width) { return width % 16 ? up256((size_t)rows * (size_t)pitch16(width)) : 0; }

// Row blocks of the error passes: as many blocks of 1024 columns as run at once (eight on each of 148 SMs), of four rows or
// more.
int error_blocks(long long M, long long N) {
  const long long strips = (N + 1023) / 1024, most = strips >= 1184 ? 1 : 1184 / strips, want = (M + 3) / 4;
  return (int)(want < most ? want : most);
}

}  // namespace

int niti_launch_pad_pitch2(niti_ctx *ctx, cudaStream_t st, const PadJob &a, const PadJob &b);

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

// Are the weights streamed (niti_linear_rows)?  Up to eight rows always; beyond, every block's tokens come through L2 and the sizes
// from which on the tiles are faster were measured (us, streamed / tiles).  16 rows: 11008 x 4096 13.3 / 18.9, 8192 x 8192 21.1 /
// 18.9, 16384 x 16384 90 / 54.  32 rows: 4096 x 4096 9.9 / 11.6, 6144 x 4096 16.8 / 12.5, and where not all blocks run at once 8192 x
// 1024 7.1 / 7.7, 16384 x 1024 12.2 / 8.1.  Rows that are not whole vectors: 16 x 2000 x 2001 10.8 / 12.0, 16 x 8192 x 2001 25 / 20, 32 x
// 1000 x 777 7.3 / 11.1, 32 x 520 x 3001 22 / 16, 32 x 4096 x 1001 10.6 / 10.9.
static bool streams(const niti_ctx *ctx, int M, int N, int K) {
  if (M <= 8) return true;
  if (M > NITI_LINEAR_ROWS) return false;
  const long long weights = (long long)N * K, mega = 1 << 20;
  if (M <= 16) return weights < (K % 16 == 0 ? 48 : 12) * mega;
  if (K % 16 != 0) return weights < 3 * mega / 2;
  return weights < (N > 48LL * ctx->sm_count ? 12 : 24) * mega;
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
  if (streams(ctx, M, N, K)) return niti_linear_rows(ctx, st, a, w, M, N, K, e, type);
  int8_t *pad = (int8_t *)ws + NITI_WS_HEADER;
  int *slabs = (int *)(pad + pad_bytes(M, K) + pad_bytes(N, K));
  const int pitch = (int)pitch16(K);
  if (pitch != K) {
    rc = niti_launch_pad_pitch2(ctx, st, PadJob{a, pad, M, K, pitch}, PadJob{w, pad + pad_bytes(M, K), N, K, pitch});
    if (rc != NITI_OK) return rc;
    a = pad;
    w = pad + pad_bytes(M, K);
  }
  WsHeader *hdr = niti_take_header(ctx, st, ws), *next = nullptr;
  if ((rc = niti_clear(ctx, st, nullptr, 0, &next)) != NITI_OK) return rc;
  const LinearMultiply x = {GK_FC_FWD, type, a, w, pitch, pitch, M, N, K, e};
  rc = run_multiplies<1>(ctx, st, &x, slabs, niti_split_max(hdr), next);
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
  const int rows = (M + nblk - 1) / nblk, blocks = (M + rows - 1) / rows;
  const int v16 = 16 / (int)es;
  const bool vec = N % v16 == 0 && (((uintptr_t)dout | (uintptr_t)z) & 15) == 0;
  // operands with padded rows, copied beside the first pass
  const bool pads = pitch != K;
  const PadJob job_w = {w, pad_w, N, K, pitch}, job_a = {a, pad_a, M, K, pitch};
  const unsigned pad0 = pads && dx ? niti_pad_blocks(job_w, ERR_THREADS, 4LL * ctx->sm_count) : 0;
  const unsigned pad1 = pads && dw ? niti_pad_blocks(job_a, ERR_THREADS, 4LL * ctx->sm_count) : 0;
  auto passes_as = [&](auto tc, auto vc, auto ac) -> int {
    constexpr int T = decltype(tc)::value, VEC = decltype(vc)::value, ACT = decltype(ac)::value;
    ErrorGrid g;
    g.strips = (N + ERR_THREADS * VEC - 1) / (ERR_THREADS * VEC);
    g.rows = rows;
    g.main = g.strips * blocks;
    NITI_CUDA_TRY(ctx, niti_launch(st, (unsigned)g.main + pad0 + pad1, ERR_THREADS, 0, error_max_kernel<T, VEC, ACT>, dout, z,
                                   dbias ? part : (float *)nullptr, hdr, next, ctx->d_status, M, N, g, job_w, job_a, pad0));
    ctx->launches++;
    niti_header_passed_on(ctx, next);
    if (!dx && !dw) {
      NITI_CUDA_TRY(ctx, niti_launch(st, (unsigned)((N + 31) / 32), ERR_THREADS, 0, bias_sum_kernel, (const float *)part, dbias, blocks, N));
      ctx->launches++;
      return NITI_OK;
    }
    auto second = [&](auto psr) -> int {
      const unsigned extra = dbias ? (unsigned)((N + 31) / 32) : 0u;
      NITI_CUDA_TRY(ctx, niti_launch(st, (unsigned)g.main + extra, ERR_THREADS, 0, error_round_kernel<T, VEC, ACT, decltype(psr)::value>, dout, z, e8, s_e,
                                     (const WsHeader *)hdr, M, N, g, pitch_e, (const float *)part, dbias, blocks));
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
  if (rc != NITI_OK || (!dx && !dw)) return rc;
  const LinearEpilogue e_x = {s_e, s_w, nullptr, nullptr, dx, nullptr, 0, NITI_ACT_NONE}, e_w = {s_e, s_a, nullptr, nullptr, dw, nullptr, 0, NITI_ACT_NONE};
  const LinearMultiply both[2] = {{GK_FC_DGRAD, type, e8, pads ? pad_w : w, pitch_e, pitch, M, K, N, e_x},
                                  {GK_FC_WGRAD, dw_type, e8, pads ? pad_a : a, pitch_e, pitch, N, K, M, e_w}};
  unsigned *counters = niti_split_max(hdr);
  return run_multiplies<2>(ctx, st, both, slabs, counters, nullptr);          // (one without an output has no items)
}
