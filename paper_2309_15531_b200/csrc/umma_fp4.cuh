// Instructions of the 4-bit floating-point kernels beyond those of umma.cuh: block-scaled 4-bit MMAs and their scales,
// pairs of CTAs on one tile, cluster barriers in two halves, programmatic dependent launch.  Internal header.
#pragma once

#include "umma.cuh"

namespace adadim {
namespace ptx {

// True in one lane of a converged warp.  A role whose whole warp walks its loop, with this around the
// issuing instructions, keeps their operands in uniform registers; under `if (lane == 0)` every one of
// them is moved there lane by lane first (70 to 120 cycles an instruction, measured).
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ int uniform_warp() { return __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0); }

// ---- mbarrier ---------------------------------------------------------------------------
// Without waiting at all (try_wait may suspend the thread for microseconds).
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
  return ok != 0;
}
// What other CTAs of the cluster wrote before the phase ended is visible afterwards.
__device__ __forceinline__ bool mbar_try_wait_cluster(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
  return ok != 0;
}
// mbar_wait for a converged warp, with one answer for all its lanes.
__device__ __forceinline__ bool mbar_wait_warp(uint64_t* bar, uint32_t parity, volatile int* dead, int* status_dev) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, dead, status_dev)) != 0;
}
// The same for what other CTAs of the cluster wrote: once the phase has ended, asking again takes their writes in.
__device__ __forceinline__ bool mbar_wait_warp_cluster(uint64_t* bar, uint32_t parity, volatile int* dead, int* status_dev) {
  if (__all_sync(0xffffffffu, mbar_try_wait_cluster(bar, parity))) return true;
  const bool ok = mbar_wait(bar, parity, dead, status_dev) && mbar_try_wait_cluster(bar, parity);
  return __all_sync(0xffffffffu, ok) != 0;
}

// ---- clusters -----------------------------------------------------------------------------
// A cluster barrier in two halves: every thread of every CTA arrives, does other work, and waits.  Orders
// no memory operations but the set-up of barriers (fence_mbar_init) before it; a release costs 700 ns here.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// Four words into a CTA of the cluster; 16 bytes are counted on that CTA's barrier when they are there.
__device__ __forceinline__ void st_async_v4(uint32_t addr, float a, float b, float c, float d, uint32_t bar) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
               ::"r"(addr), "f"(a), "f"(b), "f"(c), "f"(d), "r"(bar) : "memory");
}

// One arrival on a barrier of any CTA of the cluster.  Orders no writes towards the other CTA's
// threads (a release at cluster scope costs about 1000 cycles here): for handing back TMEM columns,
// whose reads tcgen05.wait::ld has completed.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar_cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster_addr) : "memory");
}

// ---- programmatic dependent launch ------------------------------------------------------------
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- TMA ----------------------------------------------------------------------------------
// tma_load_2d, signalled on the barrier of CTA `bar_cluster_addr` names (this CTA's or the pair's other one).
__device__ __forceinline__ void tma_load_2d_pair(void* dst, const CUtensorMap* m, int x, int y, uint32_t bar_cluster_addr) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(smem_addr(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(bar_cluster_addr)
      : "memory");
}
// 2-D tile store from this CTA's shared memory, as part of the issuing thread's bulk async-group.  The part of the
// tile outside the tensor is not written; the tile must start inside it.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* m, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(src) : "memory");
}
// until all but the latest committed group have finished reading shared memory
__device__ __forceinline__ void bulk_wait_read_but_one() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }

// ---- tcgen05 / TMEM -------------------------------------------------------------------------
// tmem_alloc, tmem_relinquish and tmem_dealloc for a pair of CTAs (one warp of each).
__device__ __forceinline__ void tmem_alloc_pair(uint32_t* smem_result, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(smem_result)), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tmem_relinquish_pair() {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
// D[tmem] (+)= A[smem] * B[smem]^T for packed 4-bit inputs with block scales in TMEM: one 64-deep step.
// MXFP4: two E8M0 scales per row and step (bytes picked by the descriptor's scale ids); NVFP4: four E4M3.
// PAIR: the two CTAs of a cluster on one tile, each holding half of the rows of either operand.
template <bool NV, bool PAIR>
__device__ __forceinline__ void mma_fp4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                        uint32_t sfa_tmem, uint32_t sfb_tmem, bool accumulate) {
#define ADADIM_MMA_FP4(GROUP, KIND, VEC)                                                                           \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"                                                \
               "tcgen05.mma.cta_group::" GROUP ".kind::" KIND ".block_scale.scale_vec::" VEC                       \
               " [%0], %1, %2, %3, [%4], [%5], p;\n\t}"                                                           \
               ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa_tmem), "r"(sfb_tmem),                    \
                 "r"(static_cast<uint32_t>(accumulate)) : "memory")
  if constexpr (NV && PAIR) ADADIM_MMA_FP4("2", "mxf4nvf4", "4X");
  else if constexpr (NV) ADADIM_MMA_FP4("1", "mxf4nvf4", "4X");
  else if constexpr (PAIR) ADADIM_MMA_FP4("2", "mxf4", "2X");
  else ADADIM_MMA_FP4("1", "mxf4", "2X");
#undef ADADIM_MMA_FP4
}
// 32 rows x 16 bytes of shared memory into 4 TMEM columns of lanes 0..31, repeated for the other
// three groups of 32 lanes: a tile of block scales.  Ordered with the MMAs this thread issues.  PAIR:
// in both CTAs, each from its own shared memory.
template <bool PAIR>
__device__ __forceinline__ void tmem_cp_scales(uint32_t taddr, uint64_t sdesc) {
  if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
}
// mma_commit for a pair: one arrival at this offset in both CTAs.
__device__ __forceinline__ void mma_commit_pair(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(smem_addr(bar)), "h"(static_cast<uint16_t>(3)) : "memory");
}
// 32 fp32 columns of this warp's 32 TMEM lanes in the order of matrix fragments: lane t of the warp gets, of every
// eight columns u, columns 2 (t % 4) and + 1 of rows t / 4 (lo[4 u], lo[4 u + 1]), t / 4 + 8 (lo[4 u + 2], ..), and of
// rows t / 4 + 16 and t / 4 + 24 the same in hi.
__device__ __forceinline__ void tmem_ld_fragments(uint32_t taddr, float (&lo)[16], float (&hi)[16]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=&r"(r[0]), "=&r"(r[1]), "=&r"(r[2]), "=&r"(r[3]), "=&r"(r[4]), "=&r"(r[5]), "=&r"(r[6]), "=&r"(r[7]),
        "=&r"(r[8]), "=&r"(r[9]), "=&r"(r[10]), "=&r"(r[11]), "=&r"(r[12]), "=&r"(r[13]), "=&r"(r[14]), "=&r"(r[15]),
        "=&r"(r[16]), "=&r"(r[17]), "=&r"(r[18]), "=&r"(r[19]), "=&r"(r[20]), "=&r"(r[21]), "=&r"(r[22]), "=&r"(r[23]),
        "=&r"(r[24]), "=&r"(r[25]), "=&r"(r[26]), "=&r"(r[27]), "=&r"(r[28]), "=&r"(r[29]), "=&r"(r[30]), "=&r"(r[31])
      : "r"(taddr), "r"(taddr + (16u << 16)) : "memory");
#pragma unroll
  for (int k = 0; k < 16; ++k) { lo[k] = __uint_as_float(r[k]); hi[k] = __uint_as_float(r[16 + k]); }
}
// Four 8 x 8 matrices of 16-bit elements to shared memory, transposed: lane t holds elements (2 (t % 4), t / 4) and
// (2 (t % 4) + 1, t / 4) of each; lane 8 i + j gives the address of row j (16 bytes) of matrix i.
__device__ __forceinline__ void stmatrix_trans(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
// The same, telling all of them whether `v` held for all of them.
__device__ __forceinline__ bool named_all(int id, int threads, bool v) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.and.pred p, %2, %3, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(r) : "r"(static_cast<uint32_t>(v)), "r"(id), "r"(threads) : "memory");
  return r != 0;
}

// ---- descriptors ----------------------------------------------------------------------------
// smem_desc_sw128 without a swizzle (scale tiles: 8-row groups of 16-byte rows, 128 bytes apart).
__host__ __device__ constexpr uint64_t smem_desc_plain(uint32_t lbo_bytes, uint32_t sbo_bytes) {
  return (static_cast<uint64_t>((lbo_bytes >> 4) & 0x3FFFu) << 16) |
         (static_cast<uint64_t>((sbo_bytes >> 4) & 0x3FFFu) << 32) | (1ull << 46);
}
// Instruction descriptor of the block-scaled 4-bit kinds: E2M1 operands, both K-major; scales E8M0 or
// E4M3; the byte of the 32-bit scale words at which this step's scales begin (MXFP4: 0 or 2).
__host__ __device__ constexpr uint32_t idesc_fp4(int M, int N, bool e8m0, uint32_t sf_byte) {
  return (sf_byte << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(e8m0) << 23) | (static_cast<uint32_t>(M >> 4) << 24) | (sf_byte << 29);
}

}  // namespace ptx
}  // namespace adadim
