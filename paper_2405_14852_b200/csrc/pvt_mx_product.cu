// Product of two matrices in 4-bit block floating point, y = x w^T, on the tensor cores' block-scaled instructions
// (tcgen05.mma kind::mxf4 / mxf4nvf4): elements and scales go in as they lie in memory, sums come out in binary32.
//
// The weights are on the instruction's side of fixed size, 128 rows, so that few tokens cost few columns, and the
// accumulator's lanes are consecutive outputs of a token.  One step is 256 columns: 128 bytes of each row, copied by TMA under the
// 128-byte swizzle, and the scales of those columns, 2 or 4 tiles per 128 rows, which lie in memory as tensor memory wants them
// (tcgen05.cp, each part of 32 lanes for all four).  Four products of 64 columns each follow.  Tensor memory holds the scales
// of every stage: a stage is refilled once the products that read it have completed, so nothing is overwritten early.
//
// Up to 16 tokens, as in generation, the product is one pass over the weights: tiles of 128 rows by 16 tokens, two blocks per SM, and
// all of a block's weights asked for at its start.  128 rows leave SMs idle in most layers, so the steps of a tile
// are shared by a cluster of up to eight blocks, whose partial sums meet in shared memory across the cluster, always in
// the order of ranks.  From 17 tokens on pairs of blocks take over (below): 4096 by 11008, 16 / 32 / 64 / 128 tokens, tiles
// of as many tokens here 9.8 / 11.8 / 16.3 / 14.9 us, pairs from 32 on 10.2 / 9.2 / 9.2.
#include "pvt_mx_mma.cuh"

namespace pvt {
namespace {

using namespace mx;
using namespace mma;

constexpr int kPThreads = 192;   // four warps read sums out, one copies, one multiplies
constexpr int kCopyWarp = 4, kMmaWarp = 5;
struct ProductParams {
  const uint8_t* w_codes;
  const uint8_t* w_scales;
  const uint8_t* x_scales;
  const float* w_ts;
  const float* x_ts;
  void* y;
  int64_t ldy, ldw;
  uint32_t* status;
  uint32_t w_rows, x_rows;
  uint32_t row_bytes;     // of w, to the last 16 that hold codes
  uint32_t strip_bytes;   // scales of a strip of 128 rows
  uint32_t steps;         // of 256 columns
  uint32_t split;         // blocks per tile
  uint32_t max_spins, withhold;
};

struct ProductShared {
  alignas(8) uint64_t full[8];
  uint64_t empty[8];
  uint64_t done, spare;
  uint32_t tmem, abandoned;
};

template <typename T, int FMT>
__global__ void __launch_bounds__(kPThreads) mx_product_kernel(const __grid_constant__ CUtensorMap w_map,
                                                               const __grid_constant__ CUtensorMap x_map, const ProductParams p) {
  using S = FewSizes<FMT>;
  constexpr uint32_t KT = S::KT, STAGES = S::kStages;
  extern __shared__ __align__(1024) unsigned char raw[];
  __shared__ ProductShared sm;
  const uint32_t tid = threadIdx.x, warp = tid >> 5;
  volatile uint32_t* abandoned = &sm.abandoned;
  const uint32_t rank = blockIdx.x % p.split, w0 = blockIdx.x / p.split * kTileW;
  const uint32_t first = p.steps * rank / p.split, last = p.steps * (rank + 1) / p.split;  // (steps < 2^20, split <= 8)
  // all of the block's weights at once, while it sets itself up and the kernel ahead ends
  const uint32_t from_byte = first * kRowBytes, to_byte = min(last * kRowBytes, p.row_bytes);
  if (tid < (uint32_t)kTileW && w0 + tid < p.w_rows)
    prefetch_l2(p.w_codes + (int64_t)(w0 + tid) * p.ldw + from_byte, to_byte - from_byte);
  if (tid == (uint32_t)kTileW)
    prefetch_l2(p.w_scales + (size_t)(w0 / kStrip) * p.strip_bytes + (size_t)first * (KT * kTileBytes), (last - first) * (KT * kTileBytes));
  if (tid == 0) {
    sm.abandoned = 0;
    for (uint32_t s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&sm.full[s]), 1);
      mbar_init(smem_u32(&sm.empty[s]), 1);
    }
    mbar_init(smem_u32(&sm.done), 1);
    mbar_init(smem_u32(&sm.spare), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(&sm.tmem), S::kTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();  // not before this block has its tensor memory: the next kernel's blocks hold theirs while they wait for this one
  pdl_wait();

  const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sm.tmem);
  const uint32_t col = w0 + tid;
  Factors alpha(1.0f, 1.0f);
  T* const y = static_cast<T*>(p.y) + col;

  if (warp == kCopyWarp) {
    const uint8_t* const ws = p.w_scales + (size_t)(w0 / kStrip) * p.strip_bytes;
    uint32_t i = 0;
    for (uint32_t step = first; step < last; ++step, ++i) {
      const uint32_t s = i % STAGES, bar = smem_u32(&sm.full[s]), to = base + s * S::kStageAligned;
      if (i >= STAGES && !wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins)) break;
      if (i == p.withhold) continue;  // test hook: never issued
      expect_bytes(bar, S::kStage);
      tma_load(to, &w_map, (int)(step * kRowBytes), (int)w0, bar);
      tma_load(to + S::kX, &x_map, (int)(step * kRowBytes), 0, bar);
      bulk_load(to + S::kWs, ws + (size_t)step * (KT * kTileBytes), KT * kTileBytes, bar);
      bulk_load(to + S::kXs, p.x_scales + (size_t)step * (KT * kTileBytes), KT * kTileBytes, bar);
    }
    if (*abandoned)  // what was issued lands before the block's memory is another's
      for (uint32_t j = i > STAGES ? i - STAGES : 0; j < i; ++j)
        if (j != p.withhold) drain(smem_u32(&sm.full[j % STAGES]), (j / STAGES) & 1);
  } else if (warp == kMmaWarp) {
    // e2m1 both, N = 16, M = 128, type of the scales
    constexpr uint32_t idesc =
        1u << 7 | 1u << 10 | (kFewTokens >> 3) << 17 | (FMT == PVT_MX_E8M0_32 ? 1u << 23 : 0u) | 1u << 27;
    uint32_t i = 0;
    bool ok = true;
    for (uint32_t step = first; step < last; ++step, ++i) {
      const uint32_t s = i % STAGES, from = base + s * S::kStageAligned;
      ok = wait(smem_u32(&sm.full[s]), (i / STAGES) & 1, abandoned, p.status, p.max_spins);
      if (!ok) break;
      tc_fence_after();
      const uint32_t sfa = tmem + 32 + s * S::kScaleCols, sfb = sfa + KT * 4;
      // a scale tile: 32 rows of 16 bytes, groups of eight rows 128 bytes apart
#pragma unroll
      for (uint32_t t = 0; t < KT; ++t) {
        scales_to_tmem(sfa + t * 4, operand(from + S::kWs + t * kTileBytes, 0, 128, false));
        scales_to_tmem(sfb + t * 4, operand(from + S::kXs + t * kTileBytes, 0, 128, false));
      }
      const uint64_t a = operand(from, 16, 1024, true), b = operand(from + S::kX, 16, 1024, true);
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {  // 64 columns, 32 bytes
        const uint32_t t = FMT == PVT_MX_E8M0_32 ? j / 2 : j, id = FMT == PVT_MX_E8M0_32 ? (j & 1) * 2 : 0;
        multiply<FMT>(tmem, a + 2 * j, b + 2 * j, idesc | id << 4 | id << 29, sfa + t * 4, sfb + t * 4, (uint32_t)(i > 0 || j > 0));
      }
      commit(smem_u32(&sm.empty[s]));
    }
    if (ok) {
      commit(smem_u32(&sm.done));
    } else if (i > 0) {
      commit(smem_u32(&sm.spare));
      drain(smem_u32(&sm.spare), 0);
    }
  } else {
    // lanes are consecutive outputs of a token
    if (p.w_ts || p.x_ts) alpha = Factors(p.w_ts ? *p.w_ts : 1.0f, p.x_ts ? *p.x_ts : 1.0f);
    float* const part = reinterpret_cast<float*>(raw + (base - smem_u32(raw)));
    if (wait(smem_u32(&sm.done), 0, abandoned, p.status, p.max_spins)) {
      tc_fence_after();
      uint32_t v[kFewTokens];
      tmem_ld16(tmem + (warp << 21), v);
      tmem_ld_wait<kFewTokens>(v);
#pragma unroll
      for (uint32_t j = 0; j < kFewTokens; ++j) {
        if (j >= p.x_rows) break;
        if (p.split > 1)
          part[j * kTileW + tid] = __uint_as_float(v[j]);
        else if (col < p.w_rows)
          y[(int64_t)j * p.ldy] = narrow<T>(alpha(__uint_as_float(v[j])));
      }
      tc_fence_before();
    }
  }
  if (p.split > 1) {
    cluster_sync();
    // every block adds up the tokens that are its share
    if (tid < (uint32_t)kTileW && col < p.w_rows && !*abandoned)
      for (uint32_t j = rank; j < p.x_rows; j += p.split) {
        float v[8], sum = 0.0f;
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r) v[r] = r < p.split ? cluster_load(base + (j * kTileW + tid) * 4, r) : 0.0f;
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r) sum += v[r];
        y[(int64_t)j * p.ldy] = narrow<T>(alpha(sum));
      }
    cluster_sync();
  }
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kTmem);
  }
}

// ---- pairs of blocks -------------------------------------------------------------------------------------------
// With many rows of x a pair of blocks on neighbouring SMs multiplies 256 rows of w by 256 of x (tcgen05.mma cta_group::2): each block
// holds 128 rows of either, so a step brings 32 KB of codes into an SM instead of 48 KB for the same 128 x 256 sums.  The four
// products of a step are 512 cycles, the bound: the tensor pipe is active in 85 % of all cycles (4096 x 8192 by 28672: 318 us
// and 6.0 PFLOP/s where the clock holds, 390 under the power cap).  The blocks stay and take tile after tile; copies for the
// next one are under way while eight warps empty the sums into registers, and those are stored while it is multiplied.
struct PairShared {
  alignas(8) uint64_t full[kPairStages];  // of the first block: bytes of both
  uint64_t empty[kPairStages];            // of each
  uint64_t sums_full;                     // of each
  uint64_t sums_empty;                    // of the first: an arrival per reading warp of both
  uint64_t spare;
  uint32_t tmem, abandoned;
};

struct PairParams {
  const float* w_ts;
  const float* x_ts;
  void* y;
  int64_t ldy;
  uint32_t* status;
  uint32_t w_rows, x_rows;
  uint32_t strip_rows;   // rows of 128 bytes that a strip's scales are
  uint32_t steps;        // of 256 columns
  uint32_t x_tiles, tiles;
  uint32_t split;        // pairs per tile
  uint32_t max_spins, withhold;
};

template <typename T, int FMT, uint32_t N>
__global__ void __launch_bounds__(kPairThreads, 1)
    mx_product_pair_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map,
                           const __grid_constant__ CUtensorMap ws_map, const __grid_constant__ CUtensorMap xs_map, const PairParams p) {
  using S = PairSizes<FMT, N>;
  constexpr uint32_t KT = S::KT, STAGES = S::kStages;
  extern __shared__ __align__(1024) unsigned char raw[];
  __shared__ PairShared sm;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile uint32_t* abandoned = &sm.abandoned;
  if (tid == 0) {
    sm.abandoned = 0;
    for (uint32_t s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&sm.full[s]), 1);
      mbar_init(smem_u32(&sm.empty[s]), 1);
    }
    mbar_init(smem_u32(&sm.sums_full), 1);
    mbar_init(smem_u32(&sm.sums_empty), 2 * kPairReaders);
    mbar_init(smem_u32(&sm.spare), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kPairMmaWarp) {
    tmem_alloc<2>(smem_u32(&sm.tmem), 512);
    tmem_relinquish<2>();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();  // not before this block has its tensor memory: the next kernel's blocks hold theirs while they wait for this one
  pdl_wait();
  cluster_sync();  // the barriers of both blocks are set up

  const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sm.tmem);
  // Pairs by themselves take tile after tile; those of a cluster share one tile's steps.
  const uint32_t in_cluster = cluster_rank(), rank = in_cluster & 1, lead = in_cluster & ~1u, share = in_cluster / 2;
  const uint32_t tile0 = blockIdx.x / 2 / p.split, stride = p.split > 1 ? p.tiles : gridDim.x / 2;
  const uint32_t first = p.steps * share / p.split, steps = p.steps * (share + 1) / p.split - first;  // (steps < 2^24, share < 4)

  if (warp >= kPairCopyWarp && warp < kPairMmaWarp) {
    const bool of_w = warp == kPairCopyWarp;  // one warp for w's codes and scales, one for x's
    uint32_t i = 0;
    bool ok = true;
    for (uint32_t tile = tile0; tile < p.tiles && ok; tile += stride) {
      const uint32_t tile0 = of_w ? tile / p.x_tiles * kPairRows : tile % p.x_tiles * N;
      const int row = (int)(tile0 + rank * (of_w ? kTileW : N / 2));
      const int strip = (int)((of_w ? (uint32_t)row : tile0) / kStrip * p.strip_rows);
      for (uint32_t step = first; step < first + steps; ++step, ++i) {
        const uint32_t s = i % STAGES, to = base + s * S::kStageAligned;
        if (i >= STAGES && !(ok = wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins))) break;
        if (i == p.withhold) continue;  // test hook: never issued
        const uint32_t bar = cluster_address(smem_u32(&sm.full[s]), lead);
        const int col = (int)(step * kRowBytes), scales = strip + (int)(step * (KT * 4));
        if (of_w) {
          if (rank == 0) expect_bytes(smem_u32(&sm.full[s]), 2 * S::kStage);
          tma_load_pair(to, &w_map, col, row, bar);
          tma_load_pair(to + S::kWs, &ws_map, 0, scales, bar);
        } else {  // both blocks multiply by all of the tile's rows of x
          tma_load_pair(to + S::kX, &x_map, col, row, bar);
          tma_load_pair(to + S::kXs, &xs_map, 0, scales, bar);
          if (S::kStrips == 2) tma_load_pair(to + S::kXs + KT * kTileBytes, &xs_map, 0, scales + (int)p.strip_rows, bar);
        }
      }
    }
    if (*abandoned && rank == 0)  // what was issued lands before the blocks' memory is another's
      for (uint32_t j = i > STAGES ? i - STAGES : 0; j < i; ++j)
        if (j != p.withhold) drain(smem_u32(&sm.full[j % STAGES]), (j / STAGES) & 1);
  } else if (warp == kPairMmaWarp) {
    if (rank == 0) {
      // e2m1 both, N, M = 256, type of the scales
      constexpr uint32_t idesc =
          1u << 7 | 1u << 10 | (N >> 3) << 17 | (FMT == PVT_MX_E8M0_32 ? 1u << 23 : 0u) | (kPairRows >> 7) << 27;
      const uint16_t both = (uint16_t)(3u << lead);
      uint32_t i = 0, n = 0;
      bool ok = true;
      for (uint32_t tile = tile0; tile < p.tiles && ok; tile += stride, ++n) {
        if (n > 0) ok = wait<true>(smem_u32(&sm.sums_empty), (n - 1) & 1, abandoned, p.status, p.max_spins);
        tc_fence_after();
        for (uint32_t step = 0; step < steps && ok; ++step) {
          const uint32_t s = i % STAGES, from = base + s * S::kStageAligned;
          ok = wait(smem_u32(&sm.full[s]), (i / STAGES) & 1, abandoned, p.status, p.max_spins);
          if (!ok) break;
          tc_fence_after();
          const uint32_t sfa = tmem + N + s * S::kScaleCols, sfb = sfa + KT * 4;
          // (a scale tile: 32 rows of 16 bytes, groups of eight rows 128 bytes apart)
          multiply_step<FMT, S::kStrips>(tmem, operand(from, 16, 1024, true), operand(from + S::kX, 16, 1024, true), idesc, sfa, sfb,
                             operand(from + S::kWs, 0, 128, false), operand(from + S::kXs, 0, 128, false), (uint32_t)(step > 0));
          commit_pair(smem_u32(&sm.empty[s]), both);
          ++i;
        }
        if (ok) commit_pair(smem_u32(&sm.sums_full), both);
      }
      if (!ok && i > 0) {
        commit_pair(smem_u32(&sm.spare), both);
        drain(smem_u32(&sm.spare), 0);
      }
    }
  } else {
    const Factors alpha(p.w_ts ? *p.w_ts : 1.0f, p.x_ts ? *p.x_ts : 1.0f);
    const uint32_t quarter = warp % 4, half = warp / 4;
    const uint32_t sums_empty = cluster_address(smem_u32(&sm.sums_empty), lead);
    uint32_t n = 0;
    for (uint32_t tile = tile0; tile < p.tiles; tile += stride, ++n) {
      bool ok = wait(smem_u32(&sm.sums_full), n & 1, abandoned, p.status, p.max_spins);
      if (!ok) break;
      tc_fence_after();
      uint32_t v[N / 2];
#pragma unroll
      for (uint32_t j = 0; j < N / 2; j += 32) tmem_ld32(tmem + (quarter << 21) + half * (N / 2) + j, v + j);
      tmem_ld_wait<(int)N / 2>(v);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) cluster_arrive(sums_empty);
      __syncwarp();
      if (p.split > 1) {  // the products are done: the stages hold the partial sums
        float* const part = reinterpret_cast<float*>(raw + (base - smem_u32(raw))) + half * (N / 2) * kTileW + quarter * 32 + lane;
#pragma unroll
        for (uint32_t j = 0; j < N / 2; ++j) part[j * kTileW] = __uint_as_float(v[j]);
        break;
      }
      // lanes are consecutive outputs of a token
      const uint32_t col = tile / p.x_tiles * kPairRows + rank * kTileW + quarter * 32 + lane;
      const uint32_t row = tile % p.x_tiles * N + half * (N / 2);
      if (col < p.w_rows && row < p.x_rows) {
        T* y = static_cast<T*>(p.y) + (int64_t)row * p.ldy + col;
        const uint32_t rows = p.x_rows - row;
#pragma unroll
        for (uint32_t j = 0; j < N / 2; ++j) {
          if (j < rows) *y = narrow<T>(alpha(__uint_as_float(v[j])));
          y += p.ldy;
        }
      }
    }
  }
  __syncthreads();
  cluster_sync();  // neither block leaves while the other's copies or products reach it
  if (p.split > 1) {
    // every pair adds up the tokens that are its share, one to a warp, always in the order of pairs
    if (!*abandoned) {
      const Factors alpha(p.w_ts ? *p.w_ts : 1.0f, p.x_ts ? *p.x_ts : 1.0f);
      const uint32_t col0 = tile0 / p.x_tiles * kPairRows + rank * kTileW, row0 = tile0 % p.x_tiles * N;
      const uint32_t tokens = min(N, p.x_rows - row0);
      for (uint32_t j = share + warp * p.split; j < tokens; j += kPairThreads / 32 * p.split) {
        float v[4][4];  // (all under way at once: a load from another block takes a thousand cycles)
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
          for (uint32_t q = 0; q < 4; ++q)
            v[i][q] = q < p.split ? cluster_load(base + (j * kTileW + i * 32 + lane) * 4, 2 * q + rank) : 0.0f;
        T* const y = static_cast<T*>(p.y) + (int64_t)(row0 + j) * p.ldy + col0 + lane;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
          if (col0 + i * 32 + lane < p.w_rows) y[i * 32] = narrow<T>(alpha(v[i][0] + v[i][1] + v[i][2] + v[i][3]));
      }
    }
    cluster_sync();  // nor while another reads its partial sums
  }
  if (warp == kPairMmaWarp) {
    tc_fence_after();
    tmem_dealloc<2>(tmem, 512);
  }
}

template <typename T, int FMT, uint32_t N>
cudaError_t product_pairs(const pvt_mx& x, const pvt_mx& w, T* y, int64_t ldy, uint32_t* status, int sm_count, cudaStream_t stream) {
  using S = PairSizes<FMT, N>;
  PairParams p = {};
  p.w_ts = w.tensor_scale, p.x_ts = x.tensor_scale, p.y = y, p.ldy = ldy, p.status = status;
  p.w_rows = (uint32_t)w.rows, p.x_rows = (uint32_t)x.rows;
  p.strip_rows = strip_tiles(w.cols, block_of(FMT)) * (kTileBytes / 128);
  p.steps = ((uint32_t)w.cols + kSpan - 1) / kSpan;
  p.x_tiles = (p.x_rows + N - 1) / N;
  p.tiles = (p.w_rows + kPairRows - 1) / kPairRows * p.x_tiles;
  const m1::WaitTestHook hook = m1::wait_test_hook();
  p.max_spins = hook.max_spins, p.withhold = hook.withhold_copy;
  CUtensorMap maps[4];
  cudaError_t e = make_map(&maps[0], w.codes, 1, (uint64_t)w.rows, ((uint64_t)w.cols + 1) / 2, (uint64_t)w.ld, kTileW);
  if (e == cudaSuccess) e = make_map(&maps[1], x.codes, 1, (uint64_t)x.rows, ((uint64_t)x.cols + 1) / 2, (uint64_t)x.ld, N / 2);
  if (e == cudaSuccess) e = make_map(&maps[2], w.scales, 1, scale_bytes(w.rows, w.cols, FMT) / 128, 128, 128, S::KT * 4, 128, false);
  if (e == cudaSuccess) e = make_map(&maps[3], x.scales, 1, scale_bytes(x.rows, x.cols, FMT) / 128, 128, 128, S::KT * 4, 128, false);
  if (e == cudaSuccess) e = allow_smem<mx_product_pair_kernel<T, FMT, N>>();
  if (e != cudaSuccess) return e;
  uint32_t pairs = (uint32_t)sm_count / 2;
  if (pairs > p.tiles) pairs = p.tiles;
  p.split = pairs_per_tile(p.tiles, p.steps, sm_count);
  return launch_clusters(mx_product_pair_kernel<T, FMT, N>, 2 * (p.split > 1 ? p.tiles * p.split : pairs), 2 * p.split, kPairThreads,
                         S::kBytes, stream, maps[0], maps[1], maps[2], maps[3], p);
}

template <typename T, int FMT>
cudaError_t product(const pvt_mx& x, const pvt_mx& w, T* y, int64_t ldy, uint32_t* status, int sm_count, cudaStream_t stream) {
  using S = FewSizes<FMT>;
  if (x.rows > (int32_t)kFewTokens)
    return narrow_tiles(x.rows, ((uint64_t)w.rows + kPairRows - 1) / kPairRows, sm_count) ? product_pairs<T, FMT, 128>(x, w, y, ldy, status, sm_count, stream)
                                                  : product_pairs<T, FMT, 256>(x, w, y, ldy, status, sm_count, stream);
  ProductParams p = {};
  p.w_codes = w.codes, p.w_scales = w.scales, p.x_scales = x.scales, p.w_ts = w.tensor_scale, p.x_ts = x.tensor_scale;
  p.y = y, p.ldy = ldy, p.ldw = w.ld, p.status = status;
  p.w_rows = (uint32_t)w.rows, p.x_rows = (uint32_t)x.rows, p.row_bytes = ((uint32_t)w.cols + 31) / 32 * 16;
  p.strip_bytes = strip_tiles(w.cols, block_of(FMT)) * kTileBytes;
  p.steps = ((uint32_t)w.cols + kSpan - 1) / kSpan;
  const uint64_t tiles = (uint64_t)((w.rows + kTileW - 1) / kTileW);
  p.split = 1;
  while (p.split < 8 && tiles * p.split * 2 <= (uint64_t)sm_count * 2 && p.split * 2 <= p.steps) p.split *= 2;
  const m1::WaitTestHook hook = m1::wait_test_hook();
  p.max_spins = hook.max_spins, p.withhold = hook.withhold_copy;
  CUtensorMap w_map, x_map;
  cudaError_t e = make_map(&w_map, w.codes, 1, (uint64_t)w.rows, ((uint64_t)w.cols + 1) / 2, (uint64_t)w.ld, kTileW);
  if (e == cudaSuccess) e = make_map(&x_map, x.codes, 1, (uint64_t)x.rows, ((uint64_t)x.cols + 1) / 2, (uint64_t)x.ld, kFewTokens);
  if (e == cudaSuccess) e = allow_smem<mx_product_kernel<T, FMT>>();
  if (e != cudaSuccess) return e;
  return launch_clusters(mx_product_kernel<T, FMT>, (unsigned)(tiles * p.split), p.split, kPThreads, S::kBytes, stream, w_map, x_map, p);
}

template <typename T>
cudaError_t product(const pvt_mx& x, const pvt_mx& w, void* y, int64_t ldy, uint32_t* status, int sm_count, cudaStream_t stream) {
  return w.format == PVT_MX_E8M0_32 ? product<T, PVT_MX_E8M0_32>(x, w, static_cast<T*>(y), ldy, status, sm_count, stream)
                                    : product<T, PVT_MX_E4M3_16>(x, w, static_cast<T*>(y), ldy, status, sm_count, stream);
}

}  // namespace

namespace mma {
cudaError_t make_map(CUtensorMap* map, const void* base, int size, uint64_t rows, uint64_t cols, uint64_t pitch,
                     uint32_t box_rows, uint32_t box_bytes, bool swizzled) {
  static std::atomic<void*> known{nullptr};
  void* f = known.load(std::memory_order_relaxed);
  if (!f) {
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (found != cudaDriverEntryPointSuccess || !f) return cudaErrorSymbolNotFound;
    known.store(f, std::memory_order_relaxed);
  }
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {pitch};
  const cuuint32_t box[2] = {(cuuint32_t)(box_bytes / size), box_rows}, steps[2] = {1, 1};
  const CUresult r = reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(f)(
      map, size == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides,
      box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}
}  // namespace mma

cudaError_t launch_mx_product(const pvt_mx& x, const pvt_mx& w, void* y, int32_t dtype, int64_t ldy, uint32_t* status,
                              int sm_count, cudaStream_t stream) {
  timing_begin(kKernMx, stream);
  const cudaError_t e = dtype == PVT_F32   ? product<float>(x, w, y, ldy, status, sm_count, stream)
                        : dtype == PVT_F16 ? product<__half>(x, w, y, ldy, status, sm_count, stream)
                                           : product<__nv_bfloat16>(x, w, y, ldy, status, sm_count, stream);
  timing_end(kKernMx, stream);
  count_launches(1);
  return e;
}

}  // namespace pvt
