// Instructions and host-side pieces that the tensor-core kernels share: barriers with bounded waits, TMA copies, tcgen05
// multiplies on int8 operands, matrix descriptors and tensor maps.
#pragma once
#include "niti_common.cuh"

namespace {

constexpr long long WAIT_LIMIT_CYCLES = 2000000000LL;

// ------------------------------------------------------------------------------------------
// PTX wrappers
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned smem_u32(const void *p) {
  return (unsigned)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void mbar_init(unsigned bar, unsigned count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void mbar_expect_tx(unsigned bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(unsigned bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(unsigned bar, unsigned parity) {
  unsigned ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Same, but the thread may sleep in hardware for up to `ns` nanoseconds while the phase is pending
// (it is woken when the phase completes), so a waiting warp does not burn issue slots polling.
__device__ __forceinline__ bool mbar_try_sleep(unsigned bar, unsigned parity, unsigned ns) {
  unsigned ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity), "r"(ns)
      : "memory");
  return ok != 0;
}
// A waiting warp that keeps polling takes issue slots next to the working warps of its scheduler (the
// hardware wait above returns after a few tens of cycles: ncu counts a poll loop every ~70 cycles in a
// warp that waits through an epilogue-bound tile).  After two failed polls the warp sleeps between
// polls, 128 ns at first and 256 ns from the eighth poll on.  Run times with and without the sleep
// measured the same within 1 % on five layer shapes; the sleep is kept because it costs nothing and
// leaves the issue slots to the working warps.
__device__ __forceinline__ void wait_backoff(unsigned &polls) {
  ++polls;
  if (polls > 2) __nanosleep(polls > 8 ? 256u : 128u);
}
// Bounded wait.  Returns false (and raises the abort flag) if the barrier did not flip in time or
// another thread already gave up.
__device__ __forceinline__ bool mbar_wait(unsigned bar, unsigned parity, volatile int *abort_flag,
                                          uint32_t *status, long long limit_cycles = WAIT_LIMIT_CYCLES) {
  if (mbar_try(bar, parity)) return true;
  long long t0 = clock64();
  unsigned polls = 0;
  while (true) {
    if (mbar_try_sleep(bar, parity, 20000u)) return true;
    if (*abort_flag) return false;
    if (clock64() - t0 > limit_cycles) {
      *abort_flag = 1;
      atomicOr(status, NITI_DEV_TIMEOUT);
      return false;
    }
    wait_backoff(polls);
  }
}
// The same bounded wait for a whole converged warp: every lane polls, the votes make the outcome (and
// with it the caller's control flow) warp-uniform, so the compiler can keep the caller's address
// arithmetic in uniform registers.
__device__ __forceinline__ bool mbar_wait_warp(unsigned bar, unsigned parity, volatile int *abort_flag,
                                               uint32_t *status, long long limit_cycles = WAIT_LIMIT_CYCLES) {
  if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
  const long long t0 = clock64();
  unsigned polls = 0;
  while (true) {
    if (__all_sync(0xffffffffu, mbar_try_sleep(bar, parity, 20000u))) return true;
    if (__any_sync(0xffffffffu, *abort_flag != 0)) return false;
    if (__any_sync(0xffffffffu, clock64() - t0 > limit_cycles)) {
      *abort_flag = 1;
      atomicOr(status, NITI_DEV_TIMEOUT);
      return false;
    }
    wait_backoff(polls);
  }
}
// One lane of a converged warp (the same one every time it is asked).
__device__ __forceinline__ bool elect_one() {
  unsigned pred;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(pred));
  return pred != 0;
}
__device__ __forceinline__ void tma_load_2d(unsigned dst, const CUtensorMap *map, unsigned bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(unsigned dst, const CUtensorMap *map, unsigned bar, int c0, int c1,
                                            int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(unsigned dst, const CUtensorMap *map, unsigned bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
// im2col copy of consecutive pixels: base pixel (w, h, n), filter offset (ow, oh)
__device__ __forceinline__ void tma_load_im2col(unsigned dst, const CUtensorMap *map, unsigned bar, int c, int w, int h,
                                                int n, unsigned short ow, unsigned short oh) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.im2col.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2], {%7, %8};"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c), "r"(w), "r"(h), "r"(n), "h"(ow), "h"(oh)
      : "memory");
}
// Adds a 32 x 32 int32 tile from shared memory (rows of 128 bytes, 128-byte swizzle) into the accumulator tensor;
// elements outside the tensor are left out.
__device__ __forceinline__ void tma_reduce_add_4d(const CUtensorMap *map, unsigned src, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.reduce.async.bulk.tensor.4d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4, %5}], [%1];\n\t"
      "cp.async.bulk.commit_group;"
      ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}
// this thread's reduce copies have read their source / are complete
__device__ __forceinline__ void tma_reduce_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tma_reduce_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void st_shared_v4(unsigned addr, int a, int b, int c, int d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void st_shared_b32(unsigned addr, int a) {
  asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(a) : "memory");
}
// One lane's 32 values as row `lane` (or, TRANSPOSED, as column `lane`) of the swizzled tile at `buf`.
template <bool TRANSPOSED>
__device__ __forceinline__ void stage_tile32(unsigned buf, int lane, const int (&v)[32]) {
  if (TRANSPOSED) {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      st_shared_b32(buf + (unsigned)(j * 128 + ((((lane >> 2) ^ (j & 7)) << 4) | ((lane & 3) << 2))), v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      st_shared_v4(buf + (unsigned)(lane * 128 + ((j ^ (lane & 7)) << 4)), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
  }
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(unsigned bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Same with the two 64-bit matrix descriptors given as 32-bit halves: the issuing thread then does
// its address arithmetic in 32 bits (the high halves never change inside a kernel).
__device__ __forceinline__ void tc_mma_i8_lh(unsigned tmem_d, unsigned a_lo, unsigned a_hi, unsigned b_lo,
                                             unsigned b_hi, unsigned idesc, unsigned accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "mov.b64 da, {%1, %2};\n\t"
      "mov.b64 db, {%3, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %5, p;\n\t}"
      ::"r"(tmem_d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_ld32(unsigned taddr, int (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
        "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
        "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// ------------------------------------------------------------------------------------------
// Cluster helpers (CTAS == 2: a pair of CTAs on neighbouring SMs works on one 256-row tile with
// tcgen05 cta_group::2; the even CTA of the pair issues the MMAs and owns the barriers).
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned cluster_ctarank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned map_to_cta(unsigned local_addr, unsigned rank) {
  unsigned r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local_addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(unsigned cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void tma_load_2d_pair(unsigned dst, const CUtensorMap *map, unsigned bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d_pair(unsigned dst, const CUtensorMap *map, unsigned bar, int c0, int c1,
                                                 int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(unsigned dst, const CUtensorMap *map, unsigned bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void tma_load_im2col_pair(unsigned dst, const CUtensorMap *map, unsigned bar, int c, int w, int h,
                                                     int n, unsigned short ow, unsigned short oh) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.im2col.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2], {%7, %8};"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c), "r"(w), "r"(h), "r"(n), "h"(ow), "h"(oh)
      : "memory");
}
__device__ __forceinline__ void tc_commit_pair(unsigned bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
      ::"r"(bar), "h"((unsigned short)3)
      : "memory");
}

__device__ __forceinline__ void tc_mma_i8_pair_lh(unsigned tmem_d, unsigned a_lo, unsigned a_hi, unsigned b_lo,
                                                  unsigned b_hi, unsigned idesc, unsigned accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "mov.b64 da, {%1, %2};\n\t"
      "mov.b64 db, {%3, %4};\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %5, p;\n\t}"
      ::"r"(tmem_d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}

// One k-block of the generic loop: KS MMAs whose operands advance by the k-step strides.
template <int CTAS, int KS>
__device__ __forceinline__ void issue_kblock(unsigned tmem_d, unsigned a_lo, unsigned a_hi, unsigned b_lo, unsigned b_hi,
                                             unsigned a_kstep16, unsigned b_kstep16, unsigned idesc, unsigned first_acc) {
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    if (CTAS == 2)
      tc_mma_i8_pair_lh(tmem_d, a_lo + (unsigned)k * a_kstep16, a_hi, b_lo + (unsigned)k * b_kstep16, b_hi, idesc,
                        k > 0 ? 1u : first_acc);
    else
      tc_mma_i8_lh(tmem_d, a_lo + (unsigned)k * a_kstep16, a_hi, b_lo + (unsigned)k * b_kstep16, b_hi, idesc,
                   k > 0 ? 1u : first_acc);
  }
}

template <int CTAS>
__device__ __forceinline__ void load2(unsigned dst, const CUtensorMap *m, unsigned bar, int c0, int c1) {
  if (CTAS == 2) tma_load_2d_pair(dst, m, bar, c0, c1); else tma_load_2d(dst, m, bar, c0, c1);
}

// ------------------------------------------------------------------------------------------
// Host side: tensor maps, descriptors, eligibility
// ------------------------------------------------------------------------------------------
typedef CUresult (*EncodeIm2colFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                   const cuuint64_t *, const int *, const int *, cuuint32_t, cuuint32_t,
                                   const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

static CUtensorMapSwizzle swizzle_enum(int bytes) {
  return bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : (bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B);
}
static unsigned long long layout_bits(int swizzle_bytes) {
  // matrix-descriptor layout type: 2 = 128-byte swizzle, 4 = 64-byte, 6 = 32-byte
  unsigned long long t = swizzle_bytes == 128 ? 2 : (swizzle_bytes == 64 ? 4 : 6);
  return t << 61;
}
// Descriptor (without start address) of a K-major operand whose rows are `sw` bytes wide.
static unsigned long long desc_kmajor(int sw, int group_rows = 8) {
  unsigned long long d = 0;
  d |= (unsigned long long)1 << 16;                          // leading byte offset: unused, 1
  d |= (unsigned long long)((group_rows * sw) >> 4) << 32;   // stride between 8-row groups
  d |= (unsigned long long)1 << 46;                          // descriptor version
  return d | layout_bits(sw);
}
// Descriptor of an MN-major operand stored as sub-tiles [kdepth rows][sw bytes].
static unsigned long long desc_mnmajor(int sw, int kdepth) {
  unsigned long long d = 0;
  d |= (unsigned long long)((kdepth * sw) >> 4) << 16;       // next sw-wide chunk along M/N
  d |= (unsigned long long)((8 * sw) >> 4) << 32;            // next group of 8 k-rows
  d |= (unsigned long long)1 << 46;
  return d | layout_bits(sw);
}
// Swizzle width (= bytes of a copied row) of an operand with `extent` elements along its rows.  Copies past the
// extent are filled with zeros, so a short last chunk costs no memory traffic, and the MMAs that would only
// see zeros are left out.
static int pick_swizzle(long long extent) { return extent > 64 ? 128 : (extent > 32 ? 64 : 32); }
// Swizzle width of an MN-major operand of which a CTA stages `n` columns: the width that copies the fewest
// columns, the wider one of two equals.
static int pick_swizzle_mn(int n) {
  if (n <= 32) return 32;
  return (n + 127) / 128 * 128 <= (n + 63) / 64 * 64 ? 128 : 64;
}

struct MapSpec {
  int nd;
  cuuint64_t dims[4];
  cuuint64_t strides[3];   // bytes, dims 1..3
  cuuint32_t box[4];       // extent of the box in tensor elements (before the element stride)
  int swizzle;
  const void *base;
  cuuint32_t estr[4];      // element (traversal) stride per dimension; 0 = 1
  int im2col;              // 1: im2col map; box[0] = channels per pixel, box[1] = pixels per copy
  int lo[2], hi[2];        // its bounding box: first base pixel (W, H), last base pixel relative to the last pixel
};

static bool encode(niti_ctx *ctx, CUtensorMap *m, const MapSpec &s) {
  if (!ctx->encode_tiled) return false;
  if (((uintptr_t)s.base & 15) != 0) return false;
  for (int i = 0; i + 1 < s.nd; ++i)
    if (s.strides[i] % 16 != 0) return false;
  if (s.im2col) {
    if (!ctx->encode_im2col || s.box[1] > 256) return false;
    for (int i = 0; i < 2; ++i)
      if (s.lo[i] < -128 || s.lo[i] > 127 || s.hi[i] < -128 || s.hi[i] > 127) return false;
    const cuuint32_t es[4] = {1, s.estr[1] > 1 ? s.estr[1] : 1, s.estr[2] > 1 ? s.estr[2] : 1, 1};
    if (es[1] > 8 || es[2] > 8) return false;
    return ((EncodeIm2colFn)ctx->encode_im2col)(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void *>(s.base), s.dims,
                                                s.strides, s.lo, s.hi, s.box[0], s.box[1], es,
                                                CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle_enum(s.swizzle),
                                                CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  }
  for (int i = 0; i < s.nd; ++i)
    if (s.box[i] == 0 || s.box[i] > 256) return false;
  cuuint32_t es[4] = {1, 1, 1, 1};
  for (int i = 0; i < s.nd; ++i)
    if (s.estr[i] > 1) es[i] = s.estr[i];
  CUresult r = ((EncodeTiledFn)ctx->encode_tiled)(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, (cuuint32_t)s.nd,
                                                  const_cast<void *>(s.base), s.dims, s.strides, s.box, es,
                                                  CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle_enum(s.swizzle),
                                                  CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS;
}

}  // namespace
