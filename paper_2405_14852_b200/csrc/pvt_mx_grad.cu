// Gradients of the product on 4-bit matrices: D[p, c] = sum over r of A(p, r) Q[r, c], Q held in 4 bits with its blocks along
// c, A the bfloat16 gradient of the product's result: as it lies in memory for dx (p a token, r an output), its
// transpose for dw (p an output, r a token).
//
// The blocks of Q run across the sum, so the block-scaled instructions do not apply.  Eight warps widen Q to
// bfloat16 on its way into shared memory (an element times its scale is exact there, with at most six significant
// bits) and tcgen05.mma multiplies 16-bit operands.  A step is 64 rows of Q by 256 columns, stored with the columns contiguous (128
// bytes = 64 columns to a row, under the 128-byte swizzle: eight threads that write 16 bytes each for eight rows meet no
// bank twice); A's tiles arrive by TMA, contiguous along r or along p as they lie.  Few tiles leave most SMs idle, so the
// steps of a tile are then shared by a cluster of up to eight blocks, whose partial sums meet in shared memory across the
// cluster, always in the order of ranks.
#include "pvt_mma.cuh"
#include "pvt_mx.cuh"

namespace pvt {
namespace {

using namespace mx;
using namespace mma;

constexpr int kWideners = 256;   // threads; they read the sums out afterwards
constexpr int kGThreads = kWideners + 64;
constexpr int kCopyWarp = 8, kMmaWarp = 9;
constexpr int kTileA = 128, kTileC = 256, kStepR = 64;
constexpr uint32_t kABytes = kTileA * kStepR * 2, kBBytes = kTileC * kStepR * 2;
constexpr int kStages = 4;
constexpr uint32_t kPartPitch = kTileC + 1;  // floats, of a row of partial sums

struct GradParams {
  const uint8_t* codes;
  const uint8_t* scales;
  const float* ts;
  int64_t ld;
  void* out;
  int64_t ldo;
  uint32_t* status;
  uint32_t a_rows, r_rows, cols;  // of A, of Q, columns of Q
  uint32_t tiles;                 // scale tiles of a strip
  uint32_t steps;
  uint32_t c_tiles;
  uint32_t split;
  uint32_t accumulate;
  uint32_t max_spins, withhold;
};

struct GradShared {
  alignas(8) uint64_t full_a[kStages];
  uint64_t full_b[kStages];
  uint64_t empty[kStages];
  uint64_t done, spare;
  uint32_t tmem, abandoned;
};

__device__ __forceinline__ void multiply16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t onto) {
  asm volatile(
      "{\n\t.reg .pred one, p;\n\t"
      "elect.sync _|one, 0xffffffff;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "@one tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(onto)
      : "memory");
}

// Eight elements times their scale, as bfloat16.  The three bits of a magnitude become the low two exponent bits and the
// first fraction bit of a bfloat16, whose bias is 126 more, the sign goes to the top; one product with 2^126 times the scale
// gives the value, that of 0.5 (a number without its leading one) included.  Where 2^126 times the scale is
// beyond bfloat16 it takes two products (e8m0, scales above 2), or the value is 2^-8 of itself and the sums are
// multiplied by 2^8 (e4m3, always: kWidened).
template <bool TWICE>
__device__ __forceinline__ uint4 widen8(uint32_t w, uint32_t factor) {
  const uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
  const uint32_t big = 0x7e807e80u;  // 2^126 twice
  auto times = [](uint32_t a, uint32_t b) {
    const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
  };
  uint32_t out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // byte i of both, a zero byte above each (the selector's fourth bit repeats the byte's top bit, which is 0)
    uint32_t pair;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(pair) : "r"(even), "r"(odd), "r"(0xc480 + 0x1111 * i));
    const uint32_t bits = (pair * 0x1040u) & 0x81c081c0u;  // shifted by 6 and by 12
    out[i] = TWICE ? times(times(bits, big), factor) : times(bits, factor);
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

template <int FMT>
constexpr float kWidened = FMT == PVT_MX_E4M3_16 ? 256.0f : 1.0f;
template <int FMT>
__device__ __forceinline__ bool takes_two(uint32_t byte) { return FMT == PVT_MX_E8M0_32 && byte > 128; }
// the (second) factor of a scale byte, twice
template <int FMT>
__device__ __forceinline__ uint32_t factor_of(uint32_t byte, bool twice) {
  uint32_t b;
  if (FMT == PVT_MX_E4M3_16)
    b = __float_as_uint(e4m3_value(byte) * 3.32306998946229e35f) >> 16;  // 2^118: at most five significant bits
  else if (twice)
    b = byte == 255 ? 0x7fc0u : byte ? byte << 7 : 0x0040u;
  else
    b = (byte + 126) << 7;  // 2^126 2^(byte - 127)
  return b | b << 16;
}

// 32 elements of a row: 16 bytes of codes and one or two scale bytes, to four pieces of 16 bytes, `put`'s
template <int FMT, typename Put>
__device__ __forceinline__ void widen32(const uint4& codes, uint32_t scales, Put put) {
  const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
  const uint32_t b0 = FMT == PVT_MX_E8M0_32 ? scales : scales & 255u, b1 = FMT == PVT_MX_E8M0_32 ? scales : scales >> 8;
  if (FMT == PVT_MX_E8M0_32 && __any_sync(0xffffffffu, takes_two<FMT>(b0))) {
    const uint32_t f = factor_of<FMT>(b0, true);
#pragma unroll
    for (int q = 0; q < 4; ++q) put(q, widen8<true>(w[q], f));
  } else {
    const uint32_t f0 = factor_of<FMT>(b0, false), f1 = FMT == PVT_MX_E8M0_32 ? f0 : factor_of<FMT>(b1, false);
#pragma unroll
    for (int q = 0; q < 4; ++q) put(q, widen8<false>(w[q], q < 2 ? f0 : f1));
  }
}

// What a thread fetches of a step: 32 columns of two rows.
struct Fetched {
  uint4 codes[2];
  uint32_t scales[2];
};
template <int FMT>
__device__ __forceinline__ void fetch(Fetched& f, const GradParams& p, uint32_t r0, uint32_t c) {
#pragma unroll
  for (int it = 0; it < 2; ++it) {
    const uint32_t r = r0 + 32 * it;
    f.codes[it] = make_uint4(0, 0, 0, 0);
    f.scales[it] = 0;
    if (r < p.r_rows && c < p.cols) {
      f.codes[it] = *reinterpret_cast<const uint4*>(p.codes + (int64_t)r * p.ld + c / 2);
      f.scales[it] = FMT == PVT_MX_E8M0_32 ? p.scales[scale_at(r, c / 32, p.tiles)]
                                           : *reinterpret_cast<const uint16_t*>(p.scales + scale_at(r, c / 16, p.tiles));
    }
  }
}

template <typename T, int FMT, bool TRANS>
__global__ void __launch_bounds__(kGThreads) mx_grad_kernel(const __grid_constant__ CUtensorMap a_map, const GradParams p) {
  constexpr uint32_t kStageBytes = kABytes + kBBytes, STAGES = kStages;
  extern __shared__ __align__(1024) unsigned char raw[];
  __shared__ GradShared sm;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile uint32_t* abandoned = &sm.abandoned;
  if (tid == 0) {
    sm.abandoned = 0;
    for (uint32_t s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&sm.full_a[s]), 1);
      mbar_init(smem_u32(&sm.full_b[s]), kWideners / 32);
      mbar_init(smem_u32(&sm.empty[s]), 1);
    }
    mbar_init(smem_u32(&sm.done), 1);
    mbar_init(smem_u32(&sm.spare), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(&sm.tmem), kTileC);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();  // not before this block has its tensor memory: the next kernel's blocks hold theirs while they wait for this one
  pdl_wait();

  const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
  unsigned char* const mem = raw + (base - smem_u32(raw));
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sm.tmem);
  const uint32_t rank = blockIdx.x % p.split, tile = blockIdx.x / p.split;
  const uint32_t a0 = tile / p.c_tiles * kTileA, c0 = tile % p.c_tiles * kTileC;
  const uint32_t first = (uint32_t)((uint64_t)p.steps * rank / p.split), last = (uint32_t)((uint64_t)p.steps * (rank + 1) / p.split);

  if (warp == kCopyWarp) {
    uint32_t i = 0;
    for (uint32_t step = first; step < last; ++step, ++i) {
      const uint32_t s = i % STAGES, bar = smem_u32(&sm.full_a[s]), to = base + s * kStageBytes;
      if (i >= STAGES && !wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins)) break;
      if (i == p.withhold) continue;  // test hook: never issued
      expect_bytes(bar, kABytes);
      if (TRANS) {
        tma_load(to, &a_map, (int)a0, (int)(step * kStepR), bar);
        tma_load(to + kABytes / 2, &a_map, (int)(a0 + 64), (int)(step * kStepR), bar);
      } else {
        tma_load(to, &a_map, (int)(step * kStepR), (int)a0, bar);
      }
    }
    if (*abandoned)  // what was issued lands before the block's memory is another's
      for (uint32_t j = i > STAGES ? i - STAGES : 0; j < i; ++j)
        if (j != p.withhold) drain(smem_u32(&sm.full_a[j % STAGES]), (j / STAGES) & 1);
  } else if (warp == kMmaWarp) {
    // binary32 sums, bfloat16 both, A contiguous along r or p, Q along c, N = 256, M = 128
    const uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | (TRANS ? 1u << 15 : 0u) | 1u << 16 | (uint32_t)(kTileC >> 3) << 17 |
                           (uint32_t)(kTileA >> 4) << 24;
    uint32_t i = 0;
    bool ok = true;
    for (uint32_t step = first; step < last; ++step, ++i) {
      const uint32_t s = i % STAGES, from = base + s * kStageBytes, parity = (i / STAGES) & 1;
      ok = wait(smem_u32(&sm.full_a[s]), parity, abandoned, p.status, p.max_spins) &&
           wait(smem_u32(&sm.full_b[s]), parity, abandoned, p.status, p.max_spins);
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (uint32_t k = 0; k < kStepR / 16; ++k) {
        const uint64_t a = TRANS ? operand(from + k * 2048, kABytes / 2, 1024, true) : operand(from + k * 32, 16, 1024, true);
        const uint64_t b = operand(from + kABytes + k * 2048, kBBytes / 4, 1024, true);
        multiply16(tmem, a, b, idesc, (uint32_t)(i > 0 || k > 0));
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
    const uint32_t in_row = tid % 8, chunk = tid / 8 % 8, group = tid / 64;
    const uint32_t row = group * 8 + in_row, c = c0 + chunk * 32;
    Fetched now;
    fetch<FMT>(now, p, first * kStepR + row, c);
    uint32_t i = 0;
    bool ok = true;
    for (uint32_t step = first; step < last; ++step, ++i) {
      Fetched next;
      if (step + 1 < last) fetch<FMT>(next, p, (step + 1) * kStepR + row, c);
      const uint32_t s = i % STAGES;
      if (i >= STAGES) ok = wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins);
      if (!ok) break;
      unsigned char* const to = mem + s * kStageBytes + kABytes + chunk / 2 * (kBBytes / 4) + row * 128;
#pragma unroll
      for (int it = 0; it < 2; ++it) {
        widen32<FMT>(now.codes[it], now.scales[it], [&](uint32_t q, uint4 v) {
          *reinterpret_cast<uint4*>(to + it * (32 * 128) + ((((chunk & 1) * 4 + q) ^ in_row) << 4)) = v;
        });
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // generic-proxy writes -> visible to the products
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.full_b[s]));
      now = next;
    }
    ok = wait(smem_u32(&sm.done), 0, abandoned, p.status, p.max_spins);
    tc_fence_after();
    if (ok) {
      const float alpha = kWidened<FMT> * (p.ts ? *p.ts : 1.0f);
      const uint32_t quarter = warp % 4, half = warp / 4;
      if (p.split == 1) {
        // 32 rows by 32 columns at a time, turned in shared memory so that a warp stores along a row; the upper four warps
        // have the second half of the columns
        float* const turn = reinterpret_cast<float*>(mem) + warp * (32 * 33);
        const uint32_t row0 = a0 + quarter * 32, j_lo = half * (kTileC / 2), j_hi = j_lo + kTileC / 2;
        const uint32_t n_rows = row0 < p.a_rows ? min(32u, p.a_rows - row0) : 0;
        for (uint32_t j0 = j_lo; j0 < j_hi && c0 + j0 < p.cols && n_rows; j0 += 32) {
          uint32_t v[32];
          tmem_ld32(tmem + (quarter << 21) + j0, v);
          tmem_ld_wait<32>(v);
#pragma unroll
          for (int j = 0; j < 32; ++j) turn[lane * 33 + j] = __uint_as_float(v[j]);
          __syncwarp();
          const uint32_t col = c0 + j0 + lane;
          if (col < p.cols) {
            T* out = static_cast<T*>(p.out) + (int64_t)row0 * p.ldo + col;
            if (sizeof(T) == 4 && p.accumulate) {
#pragma unroll 8
              for (uint32_t r = 0; r < n_rows; ++r) out[(int64_t)r * p.ldo] = narrow<T>(widen<T>(out[(int64_t)r * p.ldo]) + turn[r * 33 + lane] * alpha);
            } else {
#pragma unroll 8
              for (uint32_t r = 0; r < n_rows; ++r) out[(int64_t)r * p.ldo] = narrow<T>(turn[r * 33 + lane] * alpha);
            }
          }
          __syncwarp();
        }
      } else {
        float* const part = reinterpret_cast<float*>(mem) + (quarter * 32 + lane) * kPartPitch;
        for (uint32_t j0 = half * (kTileC / 2); j0 < (half + 1) * (kTileC / 2); j0 += 32) {
          uint32_t v[32];
          tmem_ld32(tmem + (quarter << 21) + j0, v);
          tmem_ld_wait<32>(v);
#pragma unroll
          for (int j = 0; j < 32; ++j) part[j0 + j] = __uint_as_float(v[j]);
        }
      }
    }
    tc_fence_before();
  }
  if (p.split > 1) {
    cluster_sync();
    // every block adds up the rows that are its share, always in the order of ranks
    if (warp < kWideners / 32 && !*abandoned) {
      const float alpha = kWidened<FMT> * (p.ts ? *p.ts : 1.0f);
      for (uint32_t r = rank + warp * p.split; r < kTileA && a0 + r < p.a_rows; r += kWideners / 32 * p.split) {
        T* out = static_cast<T*>(p.out) + (int64_t)(a0 + r) * p.ldo + c0;
        for (uint32_t j = lane; j < kTileC && c0 + j < p.cols; j += 32) {
          float sum = 0.0f;
          for (uint32_t q = 0; q < p.split; ++q) sum += cluster_load(base + (r * kPartPitch + j) * 4, q);
          sum *= alpha;
          if (sizeof(T) == 4 && p.accumulate) sum += widen<T>(out[j]);
          out[j] = narrow<T>(sum);
        }
      }
    }
    cluster_sync();
  }
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, kTileC);
  }
}

template <typename T, int FMT, bool TRANS>
cudaError_t start(const CUtensorMap& a_map, const GradParams& p, uint64_t tiles, cudaStream_t stream) {
  constexpr size_t smem = kStages * (kABytes + kBBytes) + 1024;
  static_assert(smem + sizeof(GradShared) + 1024 <= 227 * 1024, "a block's shared memory");
  static_assert(kTileA * kPartPitch * 4 <= kStages * (kABytes + kBBytes), "the partial sums fit the stages");
  if (tiles * p.split > 0x7fffffffull) return cudaErrorInvalidConfiguration;
  const cudaError_t e = allow_smem<mx_grad_kernel<T, FMT, TRANS>>();
  if (e != cudaSuccess) return e;
  return launch_clusters(mx_grad_kernel<T, FMT, TRANS>, (unsigned)(tiles * p.split), p.split, kGThreads, smem, stream, a_map, p);
}

// ---- pairs of blocks -------------------------------------------------------------------------------------------
// Where there are tiles for all SMs a pair of blocks on neighbouring ones multiplies 512 rows of A by 128 columns of Q (two of
// tcgen05.mma cta_group::2 with M = 256; where A has no more rows than that, 256 by 256).  Each block widens half the columns:
// 64 rows cost it 4096 elements, about 100 cycles of its issue slots, beside products of 512 cycles; with 256 x 256 it
// is twice that, and the warps that widen set the pace (2048 x 4096 by 11008: both gradients 414 us).  Codes and scales
// come by TMA like A's tiles, a few steps ahead.  What a step takes from codes to operands is several times its share
// (a wait, loads, products, stores, the fence that shows them to the tensor cores), so four groups of four warps take
// every fourth step each.  The blocks stay and take tile after tile: there are two sets of sums, four warps read one
// out while the other is added to.
constexpr int kPairGroups = 4, kPairGroupWarps = 4, kPairReaders = 4;  // warps
constexpr int kPairWideners = kPairGroups * kPairGroupWarps;
// (beside that many other warps one that copies takes 100 cycles and more for each instruction it issues: codes and A's tiles
// have one each, or two)
constexpr int kPairHeldWarp = kPairWideners + kPairReaders, kPairCopyWarp = kPairHeldWarp + 1, kPairMmaWarp = kPairCopyWarp + 2;
constexpr int kPairThreads = (kPairMmaWarp + 1) * 32;
constexpr uint32_t kPairStages = 5, kPairHeld = 8;    // steps of operands (at most), of codes and scales
constexpr uint32_t kPairSums = 256;                   // columns of tensor memory of a set

// MT: products of 256 rows per step
template <int FMT, int MT>
struct PairSizes {
  static constexpr uint32_t kRows = 256 * MT, kCols = 256 / MT, kHalf = kCols / 2;  // of a tile, columns of a block
  static constexpr uint32_t kBBytes = kHalf * kStepR * 2, kStage = MT * kABytes + kBBytes, kStages = MT == 2 ? 4 : 5;
  static constexpr uint32_t kCodeBytes = kHalf / 2 * kStepR;
  // scale tiles of 128 rows: those of kHalf columns, or the one they are half of
  static constexpr uint32_t kScaleCols = FMT == PVT_MX_E8M0_32 ? 128 : 64;
  static constexpr uint32_t kScaleBytes = (kHalf > kScaleCols ? kHalf / kScaleCols : 1) * kTileBytes;
  static constexpr uint32_t kHeldBytes = kCodeBytes + kScaleBytes;
  static constexpr uint32_t kHeldAt = kStages * kStage, kTurnAt = kHeldAt + kPairHeld * kHeldBytes;
  static constexpr size_t kBytes = kTurnAt + kPairReaders * 32 * 33 * 4 + 1024;
  static_assert(kBytes + 1024 <= 227 * 1024 && kStage % 1024 == 0 && kHeldBytes % 128 == 0, "a block's shared memory");
};

struct PairShared {
  alignas(8) uint64_t held[kPairHeld];     // of each block: codes and scales
  uint64_t held_empty[kPairHeld];          // of each: an arrival per warp of the group
  uint64_t full_a[kPairStages];            // of the first: A's tiles of both
  uint64_t full_b[kPairStages];            // of the first: an arrival per warp of both blocks' groups
  uint64_t empty[kPairStages];             // of each
  uint64_t sums_full[2];                   // of each
  uint64_t sums_empty[2];                  // of the first: an arrival per reading warp of both
  uint64_t spare;
  uint32_t tmem, abandoned;
};

struct PairParams {
  const uint8_t* scales;
  const float* ts;
  void* out;
  int64_t ldo;
  uint32_t* status;
  uint32_t a_rows, cols;
  uint32_t strip_bytes;
  uint32_t steps, a_tiles, tiles;
  uint32_t accumulate;
  uint32_t max_spins, withhold;
};

// The products of a step: four times 16 of its 64 rows, for one or two tiles of A.  One thread is elected for all of them,
// and the operands' descriptors are counted on inside (a statement for each took 46 cycles an instruction).
// a_k, b_k, a_m: from 16 rows to the next and from A's first tile to its second, in 16 bytes; d_m: columns between their sums.
template <int MT, uint32_t A_K, uint32_t B_K, uint32_t A_M, uint32_t D_M>
__device__ __forceinline__ void multiply16_step(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t onto) {
  if (MT == 1)
    asm volatile(
        "{\n\t.reg .pred one, p, t;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %4, 0;\n\tsetp.eq.u32 t, 0, 0;\n\t"
        "add.s64 a1, %1, %5;\n\tadd.s64 a2, a1, %5;\n\tadd.s64 a3, a2, %5;\n\t"
        "add.s64 b1, %2, %6;\n\tadd.s64 b2, b1, %6;\n\tadd.s64 b3, b2, %6;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a1, b1, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a2, b2, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a3, b3, %3, t;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(onto), "n"(A_K), "n"(B_K)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred one, p, t;\n\t.reg .b32 e;\n\t.reg .b64 a1, a2, a3, c0, c1, c2, c3, b1, b2, b3;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %4, 0;\n\tsetp.eq.u32 t, 0, 0;\n\tadd.u32 e, %0, %8;\n\t"
        "add.s64 a1, %1, %5;\n\tadd.s64 a2, a1, %5;\n\tadd.s64 a3, a2, %5;\n\t"
        "add.s64 c0, %1, %7;\n\tadd.s64 c1, c0, %5;\n\tadd.s64 c2, c1, %5;\n\tadd.s64 c3, c2, %5;\n\t"
        "add.s64 b1, %2, %6;\n\tadd.s64 b2, b1, %6;\n\tadd.s64 b3, b2, %6;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [e], c0, %2, %3, p;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a1, b1, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [e], c1, b1, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a2, b2, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [e], c2, b2, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a3, b3, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [e], c3, b3, %3, t;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(onto), "n"(A_K), "n"(B_K), "n"(A_M), "n"(D_M)
        : "memory");
}

template <typename T, int FMT, bool TRANS, int MT>
__global__ void __launch_bounds__(kPairThreads, 1)
    mx_grad_pair_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap q_map, const PairParams p) {
  using S = PairSizes<FMT, MT>;
  constexpr uint32_t STAGES = S::kStages;
  extern __shared__ __align__(1024) unsigned char raw[];
  __shared__ PairShared sm;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile uint32_t* abandoned = &sm.abandoned;
  if (tid == 0) {
    sm.abandoned = 0;
    for (uint32_t s = 0; s < kPairHeld; ++s) {
      mbar_init(smem_u32(&sm.held[s]), 1);
      mbar_init(smem_u32(&sm.held_empty[s]), kPairGroupWarps);
    }
    for (uint32_t s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&sm.full_a[s]), 1);
      mbar_init(smem_u32(&sm.full_b[s]), 2 * kPairGroupWarps);
      mbar_init(smem_u32(&sm.empty[s]), 1);
    }
    for (uint32_t s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&sm.sums_full[s]), 1);
      mbar_init(smem_u32(&sm.sums_empty[s]), 2 * kPairReaders);
    }
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
  unsigned char* const mem = raw + (base - smem_u32(raw));
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sm.tmem);
  const uint32_t rank = cluster_rank(), pairs = gridDim.x / 2;

  if (warp == kPairHeldWarp) {
    uint32_t i = 0;
    bool ok = true;
    for (uint32_t tile = blockIdx.x / 2; tile < p.tiles && ok; tile += pairs) {
      const uint32_t c0 = tile / p.a_tiles * S::kCols + rank * S::kHalf;
      const uint8_t* const scales = p.scales + (size_t)(c0 / S::kScaleCols) * kTileBytes;
      for (uint32_t step = 0; step < p.steps; ++step, ++i) {
        const uint32_t s = i % kPairHeld, to = base + S::kHeldAt + s * S::kHeldBytes, bar = smem_u32(&sm.held[s]);
        if (i >= kPairHeld && !(ok = wait(smem_u32(&sm.held_empty[s]), (i / kPairHeld - 1) & 1, abandoned, p.status, p.max_spins))) break;
        if (i == p.withhold) continue;  // test hook: never issued
        expect_bytes(bar, S::kHeldBytes);
        tma_load(to, &q_map, (int)(c0 / 2), (int)(step * kStepR), bar);
        bulk_load(to + S::kCodeBytes, scales + (size_t)(step * kStepR / kStrip) * p.strip_bytes, S::kScaleBytes, bar);
      }
    }
    if (*abandoned)  // what was issued lands before the block's memory is another's
      for (uint32_t j = i > kPairHeld ? i - kPairHeld : 0; j < i; ++j)
        if (j != p.withhold) drain(smem_u32(&sm.held[j % kPairHeld]), (j / kPairHeld) & 1);
  } else if (warp >= kPairCopyWarp && warp < kPairCopyWarp + 2) {
    // the second of two tiles of A has a warp of its own; where there is one, the first warp has it
    const uint32_t m = warp - kPairCopyWarp;
    if (m < (uint32_t)MT) {
      uint32_t i = 0;
      bool ok = true;
      for (uint32_t tile = blockIdx.x / 2; tile < p.tiles && ok; tile += pairs) {
        const int a0 = (int)(tile % p.a_tiles * S::kRows + rank * kTileA + m * 256);
        for (uint32_t step = 0; step < p.steps; ++step, ++i) {
          const uint32_t s = i % STAGES, to = base + s * S::kStage + m * kABytes;
          if (i >= STAGES && !(ok = wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins))) break;
          if (rank == 0 && m == 0) expect_bytes(smem_u32(&sm.full_a[s]), 2 * MT * kABytes);
          const uint32_t bar = cluster_address(smem_u32(&sm.full_a[s]), 0);
          if (TRANS) {
            tma_load_pair(to, &a_map, a0, (int)(step * kStepR), bar);
            tma_load_pair(to + kABytes / 2, &a_map, a0 + 64, (int)(step * kStepR), bar);
          } else {
            tma_load_pair(to, &a_map, (int)(step * kStepR), a0, bar);
          }
        }
      }
      if (*abandoned && rank == 0)  // (the last of them is in before this block's barrier completes)
        for (uint32_t j = i > STAGES ? i - STAGES : 0; j < i; ++j) drain(smem_u32(&sm.full_a[j % STAGES]), (j / STAGES) & 1);
    }
  } else if (warp == kPairMmaWarp) {
    if (rank == 0) {
      // binary32 sums, bfloat16 both, A contiguous along r or p, Q along c, N, M = 256
      constexpr uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | (TRANS ? 1u << 15 : 0u) | 1u << 16 |
                                 (S::kCols >> 3) << 17 | (256u >> 4) << 24;
      uint32_t i = 0, n = 0;
      bool ok = true;
      for (uint32_t tile = blockIdx.x / 2; tile < p.tiles && ok; tile += pairs, ++n) {
        const uint32_t set = n & 1;
        if (n > 1) ok = wait<true>(smem_u32(&sm.sums_empty[set]), (n / 2 - 1) & 1, abandoned, p.status, p.max_spins);
        tc_fence_after();
        for (uint32_t step = 0; step < p.steps && ok; ++step) {
          const uint32_t s = i % STAGES, from = base + s * S::kStage;
          ok = wait_both(smem_u32(&sm.full_a[s]), smem_u32(&sm.full_b[s]), (i / STAGES) & 1, abandoned, p.status, p.max_spins);
          if (!ok) break;
          tc_fence_after();
          const uint64_t a = TRANS ? operand(from, kABytes / 2, 1024, true) : operand(from, 16, 1024, true);
          multiply16_step<MT, (TRANS ? 2048 : 32) / 16, 2048 / 16, kABytes / 16, S::kCols>(
              tmem + set * kPairSums, a, operand(from + MT * kABytes, 8192, 1024, true), idesc, (uint32_t)(step > 0));
          commit_pair(smem_u32(&sm.empty[s]));
          ++i;
        }
        if (ok) commit_pair(smem_u32(&sm.sums_full[set]));
      }
      if (!ok && i > 0) {
        commit_pair(smem_u32(&sm.spare));
        drain(smem_u32(&sm.spare), 0);
      }
    }
  } else if (warp < kPairWideners) {
    const uint32_t group = warp / kPairGroupWarps, in_group = tid % (kPairGroupWarps * 32);
    // 32 columns of one or two of the 64 rows, 32 apart
    constexpr uint32_t kChunks = S::kHalf / 32, kItems = kStepR * kChunks / (kPairGroupWarps * 32);
    const uint32_t row = in_group / kChunks, chunk = in_group % kChunks, atom = chunk / 2;
    uint64_t left = 0;  // steps of all this block's tiles
    if (blockIdx.x / 2 < p.tiles) left = (uint64_t)((p.tiles - blockIdx.x / 2 + pairs - 1) / pairs) * p.steps;
    uint32_t step = group % p.steps;
    for (uint64_t i64 = group; i64 < left; i64 += kPairGroups) {
      const uint32_t i = (uint32_t)i64, hs = i % kPairHeld, s = i % STAGES;
      const unsigned char* const held = mem + S::kHeldAt + hs * S::kHeldBytes;
      bool ok = wait(smem_u32(&sm.held[hs]), (i / kPairHeld) & 1, abandoned, p.status, p.max_spins);
      if (!ok) break;
      uint4 codes[kItems];
      uint32_t scales[kItems];
#pragma unroll
      for (uint32_t it = 0; it < kItems; ++it) {
        codes[it] = *reinterpret_cast<const uint4*>(held + (in_group + it * (kPairGroupWarps * 32)) * 16);
        const uint32_t r = (step * kStepR + row + it * 32) % kStrip, at = S::kCodeBytes + r % 32 * 16 + r / 32 * 4;
        // (of 64 columns every other block has the upper half of a tile of four e8m0 scales)
        if (FMT == PVT_MX_E8M0_32)
          scales[it] = held[at + (MT == 2 ? rank * 2 : 0) + chunk];
        else
          scales[it] = *reinterpret_cast<const uint16_t*>(held + at + atom * kTileBytes + (chunk & 1) * 2);
      }
      if (i >= STAGES) ok = wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins);
      if (!ok) break;
      unsigned char* const to = mem + s * S::kStage + MT * kABytes + atom * 8192 + row * 128;
#pragma unroll
      for (uint32_t it = 0; it < kItems; ++it)
        widen32<FMT>(codes[it], scales[it], [&](uint32_t q, uint4 v) {
          *reinterpret_cast<uint4*>(to + it * (32 * 128) + ((((chunk & 1) * 4 + q) ^ (row & 7)) << 4)) = v;
        });
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // generic-proxy writes -> visible to the products
      __syncwarp();
      if (lane == 0) {
        cluster_arrive(cluster_address(smem_u32(&sm.full_b[s]), 0));
        // (only now: the stores above have taken the codes out of registers that their loads have filled)
        mbar_arrive(smem_u32(&sm.held_empty[hs]));
      }
      step = (step + kPairGroups) % p.steps;
    }
  } else {
    const float alpha = kWidened<FMT> * (p.ts ? *p.ts : 1.0f);
    const uint32_t quarter = warp % 4;
    float* const turn = reinterpret_cast<float*>(mem + S::kTurnAt) + quarter * (32 * 33);
    uint32_t n = 0;
    for (uint32_t tile = blockIdx.x / 2; tile < p.tiles; tile += pairs, ++n) {
      const uint32_t set = n & 1;
      bool ok = wait(smem_u32(&sm.sums_full[set]), (n / 2) & 1, abandoned, p.status, p.max_spins);
      if (!ok) break;
      tc_fence_after();
      const uint32_t c0 = tile / p.a_tiles * S::kCols;
      // 32 rows by 32 columns at a time, turned in shared memory so that a warp stores along a row
      for (uint32_t j0 = 0; j0 < kPairSums; j0 += 32) {
        const uint32_t row0 = tile % p.a_tiles * S::kRows + j0 / S::kCols * 256 + rank * kTileA + quarter * 32, col0 = c0 + j0 % S::kCols;
        if (row0 >= p.a_rows || col0 >= p.cols) continue;
        const uint32_t n_rows = min(32u, p.a_rows - row0);
        uint32_t v[32];
        tmem_ld32(tmem + (quarter << 21) + set * kPairSums + j0, v);
        tmem_ld_wait<32>(v);
#pragma unroll
        for (int j = 0; j < 32; ++j) turn[lane * 33 + j] = __uint_as_float(v[j]);
        __syncwarp();
        const uint32_t col = col0 + lane;
        if (col < p.cols) {
          T* out = static_cast<T*>(p.out) + (int64_t)row0 * p.ldo + col;
          if (sizeof(T) == 4 && p.accumulate) {
#pragma unroll 8
            for (uint32_t r = 0; r < n_rows; ++r) out[(int64_t)r * p.ldo] = narrow<T>(widen<T>(out[(int64_t)r * p.ldo]) + turn[r * 33 + lane] * alpha);
          } else {
#pragma unroll 8
            for (uint32_t r = 0; r < n_rows; ++r) out[(int64_t)r * p.ldo] = narrow<T>(turn[r * 33 + lane] * alpha);
          }
        }
        __syncwarp();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) cluster_arrive(cluster_address(smem_u32(&sm.sums_empty[set]), 0));
      __syncwarp();
    }
  }
  __syncthreads();
  cluster_sync();  // neither block leaves while the other's copies, arrivals or products reach it
  if (warp == kPairMmaWarp) {
    tc_fence_after();
    tmem_dealloc<2>(tmem, 512);
  }
}

template <typename T, int FMT, bool TRANS, int MT>
cudaError_t start_pairs(const CUtensorMap& a_map, const GradParams& g, const pvt_mx& q, int sm_count, cudaStream_t stream) {
  using S = PairSizes<FMT, MT>;
  PairParams p = {};
  p.scales = g.scales, p.ts = g.ts, p.out = g.out, p.ldo = g.ldo, p.status = g.status;
  p.a_rows = g.a_rows, p.cols = g.cols, p.accumulate = g.accumulate, p.max_spins = g.max_spins, p.withhold = g.withhold;
  p.strip_bytes = g.tiles * kTileBytes, p.steps = g.steps;
  p.a_tiles = (g.a_rows + S::kRows - 1) / S::kRows, p.tiles = p.a_tiles * ((g.cols + S::kCols - 1) / S::kCols);
  CUtensorMap q_map;
  cudaError_t e = make_map(&q_map, q.codes, 1, (uint64_t)q.rows, (uint64_t)(q.cols + 1) / 2, (uint64_t)q.ld, kStepR, S::kHalf / 2, false);
  if (e == cudaSuccess) e = allow_smem<mx_grad_pair_kernel<T, FMT, TRANS, MT>>();
  if (e != cudaSuccess) return e;
  uint32_t pairs = (uint32_t)sm_count / 2;
  if (pairs > p.tiles) pairs = p.tiles;
  return launch_clusters(mx_grad_pair_kernel<T, FMT, TRANS, MT>, 2 * pairs, 2, kPairThreads, S::kBytes, stream, a_map, q_map, p);
}

template <typename T, int FMT, bool TRANS>
cudaError_t grad(const void* dy, int64_t lddy, uint32_t a_rows, const pvt_mx& q, T* out, int64_t ldo, bool accumulate,
                 uint32_t* status, int sm_count, cudaStream_t stream) {
  GradParams p = {};
  p.codes = q.codes, p.scales = q.scales, p.ts = q.tensor_scale, p.ld = q.ld;
  p.out = out, p.ldo = ldo, p.status = status, p.accumulate = accumulate;
  p.a_rows = a_rows, p.r_rows = (uint32_t)q.rows, p.cols = (uint32_t)q.cols;
  p.tiles = strip_tiles(q.cols, block_of(FMT));
  p.steps = (p.r_rows + kStepR - 1) / kStepR;
  p.c_tiles = (p.cols + kTileC - 1) / kTileC;
  const m1::WaitTestHook hook = m1::wait_test_hook();
  p.max_spins = hook.max_spins, p.withhold = hook.withhold_copy;
  const uint64_t tokens = TRANS ? p.r_rows : a_rows, features = TRANS ? a_rows : p.r_rows;
  CUtensorMap a_map;
  const cudaError_t e = make_map(&a_map, dy, 2, tokens, features, (uint64_t)lddy * 2, TRANS ? kStepR : kTileA);
  if (e != cudaSuccess) return e;
  p.split = 1;
  const uint64_t pair_tiles = (uint64_t)((a_rows + 255) / 256) * p.c_tiles;
  if (a_rows > (uint32_t)kTileA && pair_tiles >= (uint64_t)sm_count / 4)
    return a_rows > 256 ? start_pairs<T, FMT, TRANS, 2>(a_map, p, q, sm_count, stream)
                        : start_pairs<T, FMT, TRANS, 1>(a_map, p, q, sm_count, stream);
  const uint64_t one = (uint64_t)((a_rows + kTileA - 1) / kTileA) * p.c_tiles;
  while (p.split < 8 && one * p.split * 2 <= (uint64_t)sm_count && p.split * 2 <= p.steps) p.split *= 2;
  return start<T, FMT, TRANS>(a_map, p, one, stream);
}

}  // namespace

cudaError_t launch_mx_grad_input(const void* dy, int64_t lddy, int32_t tokens, const pvt_mx& w, void* dx, int32_t dtype,
                                 int64_t lddx, uint32_t* status, int sm_count, cudaStream_t stream) {
  const uint32_t n = (uint32_t)tokens;
  const bool fine = w.format == PVT_MX_E4M3_16;
  timing_begin(kKernMx, stream);
  cudaError_t e;
  auto call = [&](auto* out) {
    using T = std::remove_pointer_t<decltype(out)>;
    return fine ? grad<T, PVT_MX_E4M3_16, false>(dy, lddy, n, w, out, lddx, false, status, sm_count, stream)
                : grad<T, PVT_MX_E8M0_32, false>(dy, lddy, n, w, out, lddx, false, status, sm_count, stream);
  };
  if (dtype == PVT_F32)
    e = call(static_cast<float*>(dx));
  else if (dtype == PVT_F16)
    e = call(static_cast<__half*>(dx));
  else
    e = call(static_cast<__nv_bfloat16*>(dx));
  timing_end(kKernMx, stream);
  count_launches(1);
  return e;
}

cudaError_t launch_mx_grad_weight(const void* dy, int64_t lddy, int32_t n, const pvt_mx& x, float* dw, int64_t lddw,
                                  bool accumulate, uint32_t* status, int sm_count, cudaStream_t stream) {
  timing_begin(kKernMx, stream);
  const cudaError_t e =
      x.format == PVT_MX_E4M3_16
          ? grad<float, PVT_MX_E4M3_16, true>(dy, lddy, (uint32_t)n, x, dw, lddw, accumulate, status, sm_count, stream)
          : grad<float, PVT_MX_E8M0_32, true>(dy, lddy, (uint32_t)n, x, dw, lddw, accumulate, status, sm_count, stream);
  timing_end(kKernMx, stream);
  count_launches(1);
  return e;
}

}  // namespace pvt
