// What the products on 4-bit matrices share: tensor maps, bounded waits, tcgen05 and cluster instructions.
#pragma once

#include <cuda.h>

#include "pvt_encode_m1.cuh"

namespace pvt {
namespace mma {

// Describes rows x cols elements of `size` bytes (1 or 2), rows pitch bytes apart, to the copy engine, in boxes of box_rows
// rows of box_bytes; rows of 128 bytes lie under the 128-byte swizzle unless they are to lie as they are.  What is outside reads
// as zero.  base and pitch: multiples of 16.
cudaError_t make_map(CUtensorMap* map, const void* base, int size, uint64_t rows, uint64_t cols, uint64_t pitch, uint32_t box_rows,
                     uint32_t box_bytes = 128, bool swizzled = true);

#ifdef __CUDACC__
using m1::mbar_arrive;
using m1::mbar_init;
using m1::mbar_try_wait;
using m1::smem_u32;

// A whole warp waits, and all of it has one answer.  Gives up after max_spins polls, or once another warp of the block has: the
// block is then abandoned.  CLUSTER: threads of other blocks of the cluster arrive there too.  (One thread that polls for
// its warp takes longer to bring it along than 32 that poll: both gradients of 2048 x 4096 by 11008 in 593 us, not 370.)
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile uint32_t* abandoned, uint32_t* status,
                                     uint32_t max_spins) {
  for (uint32_t spin = 0; spin < max_spins; ++spin) {
    uint32_t done;
    if (CLUSTER)
      asm volatile(
          "{\n\t.reg .pred p;\n\t"
          "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(done)
          : "r"(bar), "r"(parity)
          : "memory");
    else
      done = mbar_try_wait(bar, parity);
    if (__all_sync(0xffffffffu, done)) return true;
    if (spin % 16 == 15 && __any_sync(0xffffffffu, *abandoned)) return false;
    if (spin > 4096) __nanosleep(64);
  }
  if ((threadIdx.x & 31) == 0) {
    *abandoned = 1;
    if (status) atomicOr(status, PVT_DEV_WAIT_EXPIRED);
  }
  __syncwarp();
  return false;
}
// Two barriers of the same phase at a time, the second one the cluster's.
__device__ __forceinline__ bool wait_both(uint32_t bar, uint32_t cluster_bar, uint32_t parity, volatile uint32_t* abandoned,
                                          uint32_t* status, uint32_t max_spins) {
  uint32_t both;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %3;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 q, [%2], %3;\n\t"
      "and.pred p, p, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(both)
      : "r"(bar), "r"(cluster_bar), "r"(parity)
      : "memory");
  return __all_sync(0xffffffffu, both) ||
         (wait(bar, parity, abandoned, status, max_spins) && wait<true>(cluster_bar, parity, abandoned, status, max_spins));
}
// For what has been issued and does complete: copies and products in flight when a block is abandoned.
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) {
  for (uint32_t spin = 0; spin < m1::kMaxSpins; ++spin)
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return;
}

// What issues copies is called by a whole warp and elects the thread that does inside the statement, so that the warp stays
// together: these instructions take their operands from registers that its threads share.
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n\t.reg .pred one;\n\t"
      "elect.sync _|one, 0xffffffff;\n\t"
      "@one mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar),
      "r"(bytes)
      : "memory");
}
// `bytes` as they lie (a multiple of 16, from and to 16-byte boundaries)
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred one;\n\t"
      "elect.sync _|one, 0xffffffff;\n\t"
      "@one cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar)
      : "memory");
}
// One box at column x (elements; x * size is a multiple of 16 bytes) and row y.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred one;\n\t"
      "elect.sync _|one, 0xffffffff;\n\t"
      "@one cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}" ::"r"(
          dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
// The same in a pair of blocks that multiply together: the arrival may be at a barrier of either (an address of the cluster's).
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t cluster_bar) {
  asm volatile(
      "{\n\t.reg .pred one;\n\t"
      "elect.sync _|one, 0xffffffff;\n\t"
      "@one cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], "
      "[%4];\n\t}" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(cluster_bar)
      : "memory");
}

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// CTAS: 1, or 2 for a pair of blocks that multiply together (a warp of each calls)
template <int CTAS = 1>
__device__ __forceinline__ void tmem_alloc(uint32_t dst_smem, uint32_t cols) {
  if (CTAS == 1)
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(cols) : "memory");
  else
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(cols) : "memory");
}
template <int CTAS = 1>
__device__ __forceinline__ void tmem_relinquish() {
  if (CTAS == 1)
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  else
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
template <int CTAS = 1>
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t cols) {
  if (CTAS == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
// called by the whole warp: one arrival once everything its elected thread has issued so far has completed
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred one;\n\t"
      "elect.sync _|one, 0xffffffff;\n\t"
      "@one tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar)
      : "memory");
}
// the same for what the first block of a pair has issued: an arrival at the barrier of that place in both, which `blocks` names by
// a bit for each rank of the cluster
__device__ __forceinline__ void commit_pair(uint32_t bar, uint16_t blocks = 3) {
  asm volatile(
      "{\n\t.reg .pred one;\n\t"
      "elect.sync _|one, 0xffffffff;\n\t"
      "@one tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(bar),
      "h"(blocks)
      : "memory");
}

// Shared-memory operand descriptors: start, the two strides (bytes), 128-byte swizzle or none.
// Swizzled, K contiguous: rows of 128 bytes, groups of eight rows `strided` = 1024 apart.
// Swizzled, M or N contiguous: 64 elements to a row of 128 bytes, one row per k, groups of eight k `strided` = 1024
// apart, the next 64 elements `leading` further.
__device__ __forceinline__ uint64_t operand(uint32_t saddr, uint32_t leading, uint32_t strided, bool swizzled) {
  return (uint64_t)((saddr & 0x3ffffu) >> 4) | ((uint64_t)(leading >> 4) << 16) | ((uint64_t)(strided >> 4) << 32) |
         (1ull << 46) | (swizzled ? 2ull << 61 : 0ull);
}

// 32 lanes x 32 columns of 32-bit accumulators
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* v) {
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
}
// 32 lanes x 16 columns
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}
// (the registers pass through the statement: no use of them can be scheduled ahead of the wait)
template <int N>
__device__ __forceinline__ void tmem_ld_wait(uint32_t* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; i += 8)
    asm volatile("" : "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]),
                      "+r"(v[i + 7]));
}

// ---- clusters: the blocks of a cluster share a sum, one part of it each ----
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_address(uint32_t saddr, uint32_t rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(saddr), "r"(rank));
  return at;
}
// Arrives at a barrier of any block of the cluster.  What it stands for is this block's own: shared memory that the tensor core
// beside it reads once the other block says so, or tensor memory that has been read.  No thread of the other block reads what
// this one wrote, so there is nothing to release to it; .release.cluster would wait for everything the thread has in flight,
// 2000 cycles.  For shared memory this rests on what stands before every call, in this order, and none of it may move: each lane's
// own stores, its own fence.proxy.async, and a __syncwarp that brings all lanes' fences ahead of the one lane's arrival.
__device__ __forceinline__ void cluster_arrive(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ float cluster_load(uint32_t saddr, uint32_t rank) {
  const uint32_t at = cluster_address(saddr, rank);
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint64_t cluster_load64(uint32_t saddr, uint32_t rank) {
  const uint32_t at = cluster_address(saddr, rank);
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
  return v;
}

// a grid whose blocks form clusters of `cluster`, and whose start may overlap the kernel ahead (see launch_dependent)
template <typename... KArgs, typename... Args>
cudaError_t launch_clusters(void (*kernel)(KArgs...), unsigned grid, unsigned cluster, unsigned block, size_t smem,
                            cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}
#endif

}  // namespace mma
}  // namespace pvt
