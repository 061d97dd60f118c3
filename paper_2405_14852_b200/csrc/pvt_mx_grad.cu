// Gradients of the product on 4-bit matrices: D[p, c] = sum over r of A(p, r) Q[r, c], Q held in 4 bits with its blocks along
// c, A the bfloat16 gradient of the product's result: as it lies in memory for dx (p a token, r an output), its
// transpose for dw (p an output, r a token).
//
// The blocks of Q run across the sum, so the block-scaled instructions do not apply.  Sixteen warps widen Q to
// bfloat16 on its way into shared memory (an element times its scale is exact there, with at most six significant
// bits) and tcgen05.mma multiplies 16-bit operands.  A step is 64 rows of Q, stored with the columns contiguous (128 bytes = 64
// columns to a row, under the 128-byte swizzle: eight threads that write 16 bytes each for different rows meet no bank
// twice); A's tiles arrive by TMA, contiguous along r or along p as they lie.
//
// Where there are tiles for all SMs a pair of blocks on neighbouring ones multiplies 512 rows of A by 128 columns of Q (two of
// tcgen05.mma cta_group::2 with M = 256; for dw, and where A has no more rows than that, 256 by 256).  Each block widens half
// the columns: 64 rows cost it 4096 elements, about 100 cycles of its issue slots, beside products of 512 cycles.  The blocks
// stay and take tile after tile: there are two sets of sums, eight warps read one out while the other is added to.  The tensor
// pipe is active in 84 % of all cycles for dx, in 73 % for dw with its 180 MB of sums (2048 x 4096 by 11008: 125 and 142 us; 112
// at the rate of a library's 16-bit product).
// Few tiles (few tokens, small layers) leave most SMs idle: then blocks by themselves multiply 128 rows by 128 columns, and
// the steps of a tile are shared by a cluster of up to eight of them, whose partial sums meet in shared memory across the
// cluster, always in the order of ranks.
//
// The gradient by the common input of two matrices is one such sum over both, twice as many steps to a tile; pairs may share them, too.
//
// Codes and scales come by TMA like A's tiles, a few steps ahead.  What a step takes from codes to operands is several
// times its share (a wait, loads, products, stores, the fence that shows them to the tensor cores), so four groups
// of four warps take every fourth step each.
#include "pvt_mma.cuh"
#include "pvt_mx.cuh"

namespace pvt {
namespace {

using namespace mx;
using namespace mma;

constexpr int kTileA = 128, kStepR = 64;
constexpr uint32_t kABytes = kTileA * kStepR * 2;

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

constexpr int kGroups = 4, kGroupWarps = 4, kReaders = 8;  // warps
constexpr int kWideners = kGroups * kGroupWarps;
// (beside that many other warps one that copies takes 100 cycles and more for each instruction it issues: codes and A's tiles
// have one each, or two)
constexpr int kHeldWarp = kWideners + kReaders, kCopyWarp = kHeldWarp + 1, kMmaWarp = kCopyWarp + 2;
constexpr int kThreads = (kMmaWarp + 1) * 32;
constexpr uint32_t kStages = 4, kMostHeld = 8;  // steps of operands, of codes and scales
constexpr uint32_t kSums = 256;                 // columns of tensor memory of a pair's set

// CTAS: blocks that multiply together, MT: products of 128 CTAS rows per step, TWO: the sum over two pairs of operands
template <int FMT, int MT, int CTAS, bool TWO>
struct GradSizes {
  static constexpr bool kShares = CTAS == 1 || (TWO && MT == 1);  // a cluster may share a tile's steps
  static constexpr uint32_t kRows = 128 * CTAS * MT, kCols = CTAS == 2 ? 256 / MT : 128, kHalf = kCols / CTAS;  // of a tile, of a block
  static constexpr uint32_t kBBytes = kHalf * kStepR * 2, kStage = MT * kABytes + kBBytes;
  static constexpr uint32_t kCodeBytes = kHalf / 2 * kStepR;
  // scale tiles of 128 rows: those of kHalf columns, or the one they are half of
  static constexpr uint32_t kScaleCols = FMT == PVT_MX_E8M0_32 ? 128 : 64;
  static constexpr uint32_t kScaleBytes = (kHalf > kScaleCols ? kHalf / kScaleCols : 1) * kTileBytes;
  static constexpr uint32_t kHeldBytes = kCodeBytes + kScaleBytes;
  // columns that a reading warp turns at a time, and what is left for codes and scales
  static constexpr uint32_t kTurn = CTAS == 2 && MT == 1 && !TWO ? 64 : 32, kHeld = kTurn == 64 ? 6 : kMostHeld;
  static constexpr uint32_t kHeldAt = kStages * kStage, kTurnAt = kHeldAt + kHeld * kHeldBytes;
  static constexpr size_t kBytes = kTurnAt + kReaders * 32 * (kTurn + 1) * 4 + 1024;
  static_assert(kBytes + 1024 <= 227 * 1024 && kStage % 1024 == 0 && kHeldBytes % 128 == 0, "a block's shared memory");
  static constexpr uint32_t kTmem = CTAS == 2 ? 512 : 128;
  static constexpr uint32_t kPartPitch = kCols + 1;  // floats, of a row of partial sums
  static_assert(!kShares || kTileA * kPartPitch * 4 <= kTurnAt, "the partial sums fit what the steps were in");
};

struct GradShared {
  alignas(8) uint64_t held[kMostHeld];     // of each block: codes and scales
  uint64_t held_empty[kMostHeld];          // of each: an arrival per warp of the group
  uint64_t full_a[kStages];            // of the first: A's tiles of both
  uint64_t full_b[kStages];            // of the first: an arrival per warp of both blocks' groups
  uint64_t empty[kStages];             // of each
  uint64_t sums_full[2];                   // of each
  uint64_t sums_empty[2];                  // of the first: an arrival per reading warp of both
  uint64_t spare;
  uint32_t tmem, abandoned;
};

struct GradParams {
  const uint8_t* scales;
  const uint8_t* scales2;         // of the second pair of operands, which has the steps from `half` on
  const float* ts;
  void* out;
  int64_t ldo;
  uint32_t* status;
  uint32_t a_rows, cols;
  uint32_t strip_bytes;
  uint32_t steps, half, a_tiles, tiles;
  uint32_t split;                 // blocks per tile, where they multiply by themselves, or pairs
  uint32_t accumulate;
  uint32_t max_spins, withhold;
};

template <int CTAS>
__device__ __forceinline__ void load_a(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if (CTAS == 2)
    tma_load_pair(dst, map, x, y, bar);
  else
    tma_load(dst, map, x, y, bar);
}
template <int CTAS>
__device__ __forceinline__ void commit_to(uint32_t bar, uint32_t lead) {
  if (CTAS == 2)
    commit_pair(bar, (uint16_t)(3u << lead));
  else
    commit(bar);
}
// at a barrier of the first block of a pair, or of this block
template <int CTAS>
__device__ __forceinline__ void arrive_at_first(uint32_t bar, uint32_t lead) {
  if (CTAS == 2)
    cluster_arrive(cluster_address(bar, lead));
  else
    mbar_arrive(bar);
}

// The products of a step: four times 16 of its 64 rows, for one or two tiles of A.  One thread is elected for all of them,
// and the operands' descriptors are counted on inside (a statement for each took 46 cycles an instruction).
// A_K, B_K, A_M: from 16 rows to the next and from A's first tile to its second, in 16 bytes; D_M: columns between their sums.
template <int CTAS, int MT, uint32_t A_K, uint32_t B_K, uint32_t A_M, uint32_t D_M>
__device__ __forceinline__ void multiply_step(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t onto) {
  static_assert(MT == 1 || CTAS == 2, "a block by itself has one tile of A");
  if (CTAS == 1)
    asm volatile(
        "{\n\t"
        ".reg .pred one, p, t;\n\t"
        ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "setp.eq.u32 t, 0, 0;\n\t"
        "add.s64 a1, %1, %5;\n\t"
        "add.s64 a2, a1, %5;\n\t"
        "add.s64 a3, a2, %5;\n\t"
        "add.s64 b1, %2, %6;\n\t"
        "add.s64 b2, b1, %6;\n\t"
        "add.s64 b3, b2, %6;\n\t"
        "@one tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "@one tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, t;\n\t"
        "}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(onto), "n"(A_K), "n"(B_K)
        : "memory");
  else if (MT == 1)
    asm volatile(
        "{\n\t"
        ".reg .pred one, p, t;\n\t"
        ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "setp.eq.u32 t, 0, 0;\n\t"
        "add.s64 a1, %1, %5;\n\t"
        "add.s64 a2, a1, %5;\n\t"
        "add.s64 a3, a2, %5;\n\t"
        "add.s64 b1, %2, %6;\n\t"
        "add.s64 b2, b1, %6;\n\t"
        "add.s64 b3, b2, %6;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a1, b1, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a2, b2, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a3, b3, %3, t;\n\t"
        "}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(onto), "n"(A_K), "n"(B_K)
        : "memory");
  else
    asm volatile(
        "{\n\t"
        ".reg .pred one, p, t;\n\t"
        ".reg .b32 e;\n\t"
        ".reg .b64 a1, a2, a3, c0, c1, c2, c3, b1, b2, b3;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "setp.eq.u32 t, 0, 0;\n\t"
        "add.s64 a1, %1, %5;\n\t"
        "add.s64 a2, a1, %5;\n\t"
        "add.s64 a3, a2, %5;\n\t"
        "add.s64 b1, %2, %6;\n\t"
        "add.s64 b2, b1, %6;\n\t"
        "add.s64 b3, b2, %6;\n\t"
        "add.u32 e, %0, %8;\n\t"
        "add.s64 c0, %1, %7;\n\t"
        "add.s64 c1, c0, %5;\n\t"
        "add.s64 c2, c1, %5;\n\t"
        "add.s64 c3, c2, %5;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [e], c0, %2, %3, p;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a1, b1, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [e], c1, b1, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a2, b2, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [e], c2, b2, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [%0], a3, b3, %3, t;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::f16 [e], c3, b3, %3, t;\n\t"
        "}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(onto), "n"(A_K), "n"(B_K), "n"(A_M), "n"(D_M)
        : "memory");
}

// TWO: the sum goes on over the rows of a second pair of operands, D += A2(p, r) Q2[r, c]: its maps and scales take the place of the
// first one's from step `half` on, and nothing else changes.
template <typename T, int FMT, bool TRANS, int MT, int CTAS, bool TWO>
__global__ void __launch_bounds__(kThreads, 1)
    mx_grad_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap q_map,
                   const __grid_constant__ CUtensorMap a2_map, const __grid_constant__ CUtensorMap q2_map, const GradParams p) {
  using S = GradSizes<FMT, MT, CTAS, TWO>;
  constexpr uint32_t STAGES = kStages, kHeld = S::kHeld, TURN = S::kTurn;
  extern __shared__ __align__(1024) unsigned char raw[];
  __shared__ GradShared sm;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile uint32_t* abandoned = &sm.abandoned;
  if (tid == 0) {
    sm.abandoned = 0;
    for (uint32_t s = 0; s < kHeld; ++s) {
      mbar_init(smem_u32(&sm.held[s]), 1);
      mbar_init(smem_u32(&sm.held_empty[s]), kGroupWarps);
    }
    for (uint32_t s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&sm.full_a[s]), 1);
      mbar_init(smem_u32(&sm.full_b[s]), CTAS * kGroupWarps);
      mbar_init(smem_u32(&sm.empty[s]), 1);
    }
    for (uint32_t s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&sm.sums_full[s]), 1);
      mbar_init(smem_u32(&sm.sums_empty[s]), CTAS * kReaders);
    }
    mbar_init(smem_u32(&sm.spare), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    tmem_alloc<CTAS>(smem_u32(&sm.tmem), S::kTmem);
    tmem_relinquish<CTAS>();
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
  // A pair's blocks take tile after tile; a block by itself, or a pair where a cluster has several, has some steps of one.
  const uint32_t in_cluster = cluster_rank(), rank = CTAS == 2 ? in_cluster % 2 : 0, lead = S::kShares ? in_cluster - rank : 0;
  const uint32_t split = S::kShares ? p.split : 1, share = in_cluster / CTAS;
  const uint32_t tile0 = blockIdx.x / (CTAS * split), stride = CTAS == 2 && split == 1 ? gridDim.x / 2 : p.tiles;
  const uint32_t first = S::kShares ? (uint32_t)((uint64_t)p.steps * share / split) : 0;
  const uint32_t steps = S::kShares ? (uint32_t)((uint64_t)p.steps * (share + 1) / split) - first : p.steps;

  if (warp == kHeldWarp) {
    uint32_t i = 0;
    bool ok = true;
    for (uint32_t tile = tile0; tile < p.tiles && ok; tile += stride) {
      const uint32_t c0 = tile / p.a_tiles * S::kCols + rank * S::kHalf;
      const size_t scales_at = (size_t)(c0 / S::kScaleCols) * kTileBytes;
      for (uint32_t step = 0; step < steps; ++step, ++i) {
        const uint32_t s = i % kHeld, to = base + S::kHeldAt + s * S::kHeldBytes, bar = smem_u32(&sm.held[s]);
        if (i >= kHeld && !(ok = wait(smem_u32(&sm.held_empty[s]), (i / kHeld - 1) & 1, abandoned, p.status, p.max_spins))) break;
        if (i == p.withhold) continue;  // test hook: never issued
        const bool second = TWO && first + step >= p.half;
        const uint32_t r0 = (first + step - (second ? p.half : 0)) * kStepR;
        expect_bytes(bar, S::kHeldBytes);
        tma_load(to, second ? &q2_map : &q_map, (int)(c0 / 2), (int)r0, bar);
        bulk_load(to + S::kCodeBytes, (second ? p.scales2 : p.scales) + scales_at + (size_t)(r0 / kStrip) * p.strip_bytes, S::kScaleBytes, bar);
      }
    }
    if (*abandoned)  // what was issued lands before the block's memory is another's
      for (uint32_t j = i > kHeld ? i - kHeld : 0; j < i; ++j)
        if (j != p.withhold) drain(smem_u32(&sm.held[j % kHeld]), (j / kHeld) & 1);
  } else if (warp >= kCopyWarp && warp < kCopyWarp + 2) {
    // the second of two tiles of A has a warp of its own; where there is one, the first warp has it
    const uint32_t m = warp - kCopyWarp;
    if (m < (uint32_t)MT) {
      uint32_t i = 0;
      bool ok = true;
      for (uint32_t tile = tile0; tile < p.tiles && ok; tile += stride) {
        const int a0 = (int)(tile % p.a_tiles * S::kRows + rank * kTileA + m * 256);
        for (uint32_t step = 0; step < steps; ++step, ++i) {
          const uint32_t s = i % STAGES, to = base + s * S::kStage + m * kABytes;
          if (i >= STAGES && !(ok = wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins))) break;
          if (rank == 0 && m == 0) expect_bytes(smem_u32(&sm.full_a[s]), CTAS * MT * kABytes);
          const uint32_t bar = CTAS == 2 ? cluster_address(smem_u32(&sm.full_a[s]), lead) : smem_u32(&sm.full_a[s]);
          const bool second = TWO && first + step >= p.half;
          const int r0 = (int)((first + step - (second ? p.half : 0)) * kStepR);
          if (TRANS) {
            load_a<CTAS>(to, &a_map, a0, r0, bar);
            load_a<CTAS>(to + kABytes / 2, &a_map, a0 + 64, r0, bar);
          } else {
            load_a<CTAS>(to, second ? &a2_map : &a_map, r0, a0, bar);
          }
        }
      }
      if (*abandoned && rank == 0)  // (the last of them is in before this block's barrier completes)
        for (uint32_t j = i > STAGES ? i - STAGES : 0; j < i; ++j) drain(smem_u32(&sm.full_a[j % STAGES]), (j / STAGES) & 1);
    }
  } else if (warp == kMmaWarp) {
    if (rank == 0) {
      // binary32 sums, bfloat16 both, A contiguous along r or p, Q along c, N, M
      constexpr uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | (TRANS ? 1u << 15 : 0u) | 1u << 16 |
                                 (S::kCols >> 3) << 17 | (128u * CTAS >> 4) << 24;
      uint32_t i = 0, n = 0;
      bool ok = true;
      for (uint32_t tile = tile0; tile < p.tiles && ok; tile += stride, ++n) {
        const uint32_t set = n & 1;
        if (n > 1) ok = wait<true>(smem_u32(&sm.sums_empty[set]), (n / 2 - 1) & 1, abandoned, p.status, p.max_spins);
        tc_fence_after();
        for (uint32_t step = 0; step < steps && ok; ++step) {
          const uint32_t s = i % STAGES, from = base + s * S::kStage;
          ok = wait_both(smem_u32(&sm.full_a[s]), smem_u32(&sm.full_b[s]), (i / STAGES) & 1, abandoned, p.status, p.max_spins);
          if (!ok) break;
          tc_fence_after();
          const uint64_t a = TRANS ? operand(from, kABytes / 2, 1024, true) : operand(from, 16, 1024, true);
          multiply_step<CTAS, MT, (TRANS ? 2048 : 32) / 16, 2048 / 16, kABytes / 16, S::kCols>(
              tmem + set * kSums, a, operand(from + MT * kABytes, 8192, 1024, true), idesc, (uint32_t)(step > 0));
          commit_to<CTAS>(smem_u32(&sm.empty[s]), lead);
          ++i;
        }
        if (ok) commit_to<CTAS>(smem_u32(&sm.sums_full[set]), lead);
      }
      if (!ok && i > 0) {
        commit_to<CTAS>(smem_u32(&sm.spare), lead);
        drain(smem_u32(&sm.spare), 0);
      }
    }
  } else if (warp < kWideners) {
    const uint32_t group = warp / kGroupWarps, in_group = tid % (kGroupWarps * 32);
    // 32 columns of one or two of the 64 rows, 32 apart
    constexpr uint32_t kChunks = S::kHalf / 32, kItems = kStepR * kChunks / (kGroupWarps * 32);
    // (eight neighbouring lanes have four rows of one 128-byte column of B: their stores meet no bank twice)
    const uint32_t row = in_group / (8 * kChunks) * 8 + in_group / 2 % 4 + in_group / (4 * kChunks) % 2 * 4;
    const uint32_t chunk = in_group % 2 + (kChunks == 4 ? in_group / 8 % 2 * 2 : 0), atom = chunk / 2;
    // steps of all this block's tiles
    const uint64_t left = tile0 < p.tiles ? (uint64_t)((p.tiles - tile0 + stride - 1) / stride) * steps : 0;
    uint32_t step = group % steps;
    for (uint64_t i64 = group; i64 < left; i64 += kGroups) {
      const uint32_t i = (uint32_t)i64, hs = i % kHeld, s = i % STAGES;
      const unsigned char* const held = mem + S::kHeldAt + hs * S::kHeldBytes;
      // A parity tells two rounds of a slot apart, not three: a group may wait for its codes only once those of kHeld steps ago are in, and
      // they may come later than younger ones.  Where the slots are a multiple of the groups it has seen to them itself; elsewhere
      // it waits for its stage first, whose products come behind those of all steps ahead of them.
      constexpr bool kStageFirst = kHeld % kGroups != 0;
      static_assert(kHeld >= STAGES, "codes of kHeld steps ago were taken before the products of STAGES steps ago");
      auto stage_free = [&] { return i < STAGES || wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins); };
      bool ok = !kStageFirst || stage_free();
      if (ok) ok = wait(smem_u32(&sm.held[hs]), (i / kHeld) & 1, abandoned, p.status, p.max_spins);
      if (!ok) break;
      uint4 codes[kItems];
      uint32_t scales[kItems];
#pragma unroll
      for (uint32_t it = 0; it < kItems; ++it) {
        codes[it] = *reinterpret_cast<const uint4*>(held + (row * kChunks + chunk + it * (kGroupWarps * 32)) * 16);
        const uint32_t of_q = first + step - (TWO && first + step >= p.half ? p.half : 0);
        const uint32_t r = (of_q * kStepR + row + it * 32) % kStrip, at = S::kCodeBytes + r % 32 * 16 + r / 32 * 4;
        // (of 64 columns every other block has the upper half of a tile of four e8m0 scales)
        if (FMT == PVT_MX_E8M0_32)
          scales[it] = held[at + (MT == 2 ? rank * 2 : 0) + chunk];
        else
          scales[it] = *reinterpret_cast<const uint16_t*>(held + at + atom * kTileBytes + (chunk & 1) * 2);
      }
      if (!kStageFirst && !stage_free()) break;
      unsigned char* const to = mem + s * S::kStage + MT * kABytes + atom * 8192 + row * 128;
#pragma unroll
      for (uint32_t it = 0; it < kItems; ++it)
        widen32<FMT>(codes[it], scales[it], [&](uint32_t q, uint4 v) {
          *reinterpret_cast<uint4*>(to + it * (32 * 128) + ((((chunk & 1) * 4 + q) ^ (row & 7)) << 4)) = v;
        });
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // generic-proxy writes -> visible to the products
      __syncwarp();
      if (lane == 0) {
        arrive_at_first<CTAS>(smem_u32(&sm.full_b[s]), lead);
        // (only now: the stores above have taken the codes out of registers that their loads have filled)
        mbar_arrive(smem_u32(&sm.held_empty[hs]));
      }
      step = (step + kGroups) % steps;
    }
  } else {
    const Factors alpha(kWidened<FMT>, p.ts ? *p.ts : 1.0f);
    // (a warp reads the quarter of the lanes that its number gives it; the upper four have the second half of the columns)
    const uint32_t quarter = warp % 4, half = (warp - kWideners) / 4;
    float* const turn = reinterpret_cast<float*>(mem + S::kTurnAt) + (warp - kWideners) * (32 * (TURN + 1));
    uint32_t n = 0;
    for (uint32_t tile = tile0; tile < p.tiles; tile += stride, ++n) {
      const uint32_t set = n & 1;
      bool ok = wait(smem_u32(&sm.sums_full[set]), (n / 2) & 1, abandoned, p.status, p.max_spins);
      if (!ok) break;
      tc_fence_after();
      const uint32_t c0 = tile / p.a_tiles * S::kCols;
      if (S::kShares && split > 1) {  // the products are done: the partial sums lie where their operands and codes were
        float* const part = reinterpret_cast<float*>(mem) + (quarter * 32 + lane) * S::kPartPitch;
        for (uint32_t j0 = half * (S::kCols / 2); j0 < (half + 1) * (S::kCols / 2); j0 += 32) {
          uint32_t v[32];
          tmem_ld32(tmem + (quarter << 21) + j0, v);
          tmem_ld_wait<32>(v);
#pragma unroll
          for (int j = 0; j < 32; ++j) part[j0 + j] = __uint_as_float(v[j]);
        }
        tc_fence_before();
        break;
      }
      // 32 rows by 32 or 64 columns at a time, turned in shared memory so that a warp stores along a row.  (Where rows begin
      // inside of 32 bytes, what two stores share of these costs least if the second one comes at once: dw of 77 tokens 5119 by
      // 4095, 32 and 64 columns: 36 and 28 us.)
      for (uint32_t j0 = half * (S::kCols * MT / 2); j0 < (half + 1) * (S::kCols * MT / 2); j0 += TURN) {
        const uint32_t row0 = tile % p.a_tiles * S::kRows + j0 / S::kCols * 256 + rank * kTileA + quarter * 32, col0 = c0 + j0 % S::kCols;
        if (row0 >= p.a_rows || col0 >= p.cols) continue;
        const uint32_t n_rows = min(32u, p.a_rows - row0);
#pragma unroll
        for (uint32_t h = 0; h < TURN; h += 32) {
          uint32_t v[32];
          tmem_ld32(tmem + (quarter << 21) + set * kSums + j0 + h, v);
          tmem_ld_wait<32>(v);
#pragma unroll
          for (uint32_t j = 0; j < 32; ++j) turn[lane * (TURN + 1) + h + j] = __uint_as_float(v[j]);
        }
        __syncwarp();
        T* const out = static_cast<T*>(p.out) + (int64_t)row0 * p.ldo + col0 + lane;
        auto rows = [&](auto add, auto both) {
#pragma unroll 8
          for (uint32_t r = 0; r < n_rows; ++r)
#pragma unroll
            for (uint32_t h = 0; h < (decltype(both)::value ? TURN : 32); h += 32) {
              T* const to = out + (int64_t)r * p.ldo + h;
              const float sum = alpha(turn[r * (TURN + 1) + h + lane]);
              *to = narrow<T>(decltype(add)::value ? widen<T>(*to) + sum : sum);
            }
        };
        using Yes = std::true_type;
        using No = std::false_type;
        const bool second = TURN == 64 && col0 + 32 + lane < p.cols;
        if (sizeof(T) == 4 && p.accumulate) {
          if (second)
            rows(Yes{}, Yes{});
          else if (col0 + lane < p.cols)
            rows(Yes{}, No{});
        } else {
          if (second)
            rows(No{}, Yes{});
          else if (col0 + lane < p.cols)
            rows(No{}, No{});
        }
        __syncwarp();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_at_first<CTAS>(smem_u32(&sm.sums_empty[set]), lead);
      __syncwarp();
    }
  }
  __syncthreads();
  cluster_sync();  // no block leaves while another's copies, arrivals or products reach it
  if (S::kShares && split > 1) {
    // every block adds up the rows that are its share, always in the order of ranks
    if (warp < kWideners && !*abandoned) {
      const Factors alpha(kWidened<FMT>, p.ts ? *p.ts : 1.0f);
      const uint32_t a0 = tile0 % p.a_tiles * S::kRows + rank * kTileA, c0 = tile0 / p.a_tiles * S::kCols;
      for (uint32_t r = share + warp * split; r < kTileA && a0 + r < p.a_rows; r += kWideners * split) {
        T* const out = static_cast<T*>(p.out) + (int64_t)(a0 + r) * p.ldo + c0;
#pragma unroll
        for (uint32_t j = lane; j < S::kCols; j += 32) {
          float v[8 / CTAS], sum = 0.0f;
#pragma unroll
          for (uint32_t q = 0; q < 8 / CTAS; ++q)
            v[q] = q < split ? cluster_load(base + (r * S::kPartPitch + j) * 4, CTAS * q + rank) : 0.0f;
#pragma unroll
          for (uint32_t q = 0; q < 8 / CTAS; ++q) sum += v[q];
          sum = alpha(sum);
          if (c0 + j < p.cols) {
            if (sizeof(T) == 4 && p.accumulate) sum += widen<T>(out[j]);
            out[j] = narrow<T>(sum);
          }
        }
      }
    }
    cluster_sync();  // nor while another reads its partial sums
  }
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc<CTAS>(tmem, S::kTmem);
  }
}

// Blocks or pairs that share a tile's steps, at most 8 / CTAS of them: the number that leaves each the fewest steps while all clusters
// run at once.  time: what that takes, in units of 10 ns, by what a step and the rest of a tile took for sums over 2 x 11008 and 2 x 6144
// (a step waits for its elements to be widened, whatever multiplies them, unless both tiles of A are there).
template <typename T, int FMT, int MT, int CTAS>
uint32_t shares_of(uint32_t a_rows, uint32_t cols, uint32_t steps, int sm_count, uint64_t* time) {
  using S = GradSizes<FMT, MT, CTAS, true>;
  constexpr uint32_t kStep = CTAS == 1 ? 40 : MT == 1 ? 43 : 38, kTile = CTAS == 1 ? 450 : 600;
  const uint64_t tiles = (uint64_t)((a_rows + S::kRows - 1) / S::kRows) * ((cols + S::kCols - 1) / S::kCols), all = (uint32_t)sm_count / CTAS;
  *time = (tiles + all - 1) / all * steps * kStep + kTile;
  uint32_t shares = 1;
  if (S::kShares)
    for (uint32_t n = 2; n <= 8 / CTAS && 4 * n <= steps && n * tiles <= all; ++n)
      if (tiles <= clusters_at_once<mx_grad_kernel<T, FMT, false, MT, CTAS, true>>(CTAS * n, kThreads, S::kBytes))
        shares = n, *time = (uint64_t)((steps + n - 1) / n) * kStep + kTile + (CTAS == 2 ? 150 : 0);
  return shares;
}

// split: blocks or pairs that share a tile's steps (TWO)
template <typename T, int FMT, bool TRANS, int MT, int CTAS, bool TWO>
cudaError_t start(const CUtensorMap& a_map, const CUtensorMap& a2_map, GradParams p, const pvt_mx& q, const pvt_mx& q2, int sm_count,
                  cudaStream_t stream, uint32_t split = 1) {
  using S = GradSizes<FMT, MT, CTAS, TWO>;
  p.a_tiles = (p.a_rows + S::kRows - 1) / S::kRows, p.tiles = p.a_tiles * ((p.cols + S::kCols - 1) / S::kCols);
  CUtensorMap q_map, q2_map;
  cudaError_t e = make_map(&q_map, q.codes, 1, (uint64_t)q.rows, ((uint64_t)q.cols + 1) / 2, (uint64_t)q.ld, kStepR, S::kHalf / 2, false);
  if (TWO && e == cudaSuccess)
    e = make_map(&q2_map, q2.codes, 1, (uint64_t)q2.rows, ((uint64_t)q2.cols + 1) / 2, (uint64_t)q2.ld, kStepR, S::kHalf / 2, false);
  if (e == cudaSuccess) e = allow_smem<mx_grad_kernel<T, FMT, TRANS, MT, CTAS, TWO>>();
  if (e != cudaSuccess) return e;
  uint32_t grid = 2 * (p.tiles < (uint32_t)sm_count / 2 ? p.tiles : (uint32_t)sm_count / 2), cluster = 2;
  p.split = split;
  if (CTAS == 1 && !TWO)
    while (p.split < 8 && (uint64_t)p.tiles * p.split * 2 <= (uint64_t)sm_count && p.split * 2 <= p.steps) p.split *= 2;
  if (CTAS == 1 || p.split > 1) cluster = CTAS * p.split, grid = p.tiles * cluster;
  return launch_clusters(mx_grad_kernel<T, FMT, TRANS, MT, CTAS, TWO>, grid, cluster, kThreads, S::kBytes, stream, a_map, q_map,
                         TWO ? a2_map : a_map, TWO ? q2_map : q_map, p);
}

// dy2, q2: the second pair, of the same sizes (TWO)
template <typename T, int FMT, bool TRANS, bool TWO = false>
cudaError_t grad(const void* dy, int64_t lddy, uint32_t a_rows, const pvt_mx& q, T* out, int64_t ldo, bool accumulate,
                 uint32_t* status, int sm_count, cudaStream_t stream, const void* dy2 = nullptr, const pvt_mx* other = nullptr) {
  const pvt_mx& q2 = TWO ? *other : q;
  GradParams p = {};
  p.scales = q.scales, p.scales2 = q2.scales, p.ts = q.tensor_scale, p.out = out, p.ldo = ldo, p.status = status;
  p.a_rows = a_rows, p.cols = (uint32_t)q.cols, p.accumulate = accumulate;
  p.strip_bytes = strip_tiles(q.cols, block_of(FMT)) * kTileBytes;
  p.half = ((uint32_t)q.rows + kStepR - 1) / kStepR, p.steps = TWO ? 2 * p.half : p.half;
  const m1::WaitTestHook hook = m1::wait_test_hook();
  p.max_spins = hook.max_spins, p.withhold = hook.withhold_copy;
  const uint64_t tokens = TRANS ? (uint64_t)q.rows : a_rows, features = TRANS ? a_rows : (uint64_t)q.rows;
  CUtensorMap a_map, a2_map;
  cudaError_t e = make_map(&a_map, dy, 2, tokens, features, (uint64_t)lddy * 2, TRANS ? kStepR : kTileA);
  if (TWO && e == cudaSuccess) e = make_map(&a2_map, dy2, 2, tokens, features, (uint64_t)lddy * 2, kTileA);
  if (e != cudaSuccess) return e;
  if constexpr (TWO) {
    // What takes least.  11008 by 4096, 256 tokens: 64 tiles by two blocks each 66 us, 16 tiles by three pairs each 50; 512 tokens: 128
    // tiles by blocks 120, 32 tiles by two pairs each 70.  77 tokens 4095 by 5119: 40 tiles by two and by three blocks 31 and 24.
    uint64_t by_blocks, by_pairs, by_tall;
    const uint32_t blocks = shares_of<T, FMT, 1, 1>(a_rows, p.cols, p.steps, sm_count, &by_blocks);
    const uint32_t pairs = shares_of<T, FMT, 1, 2>(a_rows, p.cols, p.steps, sm_count, &by_pairs);
    shares_of<T, FMT, 2, 2>(a_rows, p.cols, p.steps, sm_count, &by_tall);
    if (by_blocks <= by_pairs && by_blocks <= by_tall)
      return start<T, FMT, TRANS, 1, 1, TWO>(a_map, a2_map, p, q, q2, sm_count, stream, blocks);
    if (by_pairs <= by_tall) return start<T, FMT, TRANS, 1, 2, TWO>(a_map, a2_map, p, q, q2, sm_count, stream, pairs);
    return start<T, FMT, TRANS, 2, 2, TWO>(a_map, a2_map, p, q, q2, sm_count, stream);
  }
  // Blocks by themselves where they have the rows, or pairs would leave three quarters of the SMs idle: dx by blocks and by pairs,
  // 256 tokens 4096 by 4096 18.5 and 28.2 us, 600 tokens 2048 by 2048 15.3 and 16.9.
  const uint64_t pair_tiles = (uint64_t)((a_rows + 255) / 256) * ((p.cols + 255) / 256);
  if (a_rows <= (uint32_t)kTileA || pair_tiles < (uint64_t)sm_count / 4)
    return start<T, FMT, TRANS, 1, 1, TWO>(a_map, a2_map, p, q, q2, sm_count, stream);
  // (512 by 128 and 256 by 256, 2048 x 4096 by 11008: dx 125 and 128 us, dw 150 and 142: A's transpose takes two copies a tile)
  if (TRANS || a_rows <= 256) return start<T, FMT, TRANS, 1, 2, TWO>(a_map, a2_map, p, q, q2, sm_count, stream);
  return start<T, FMT, TRANS, TRANS ? 1 : 2, 2, TWO>(a_map, a2_map, p, q, q2, sm_count, stream);
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

cudaError_t launch_mx_gated_grad_input(const void* dgate, const void* dup, int64_t ldd, int32_t tokens, const pvt_mx& wg, const pvt_mx& wu,
                                       void* dx, int32_t dtype, int64_t lddx, uint32_t* status, int sm_count, cudaStream_t stream) {
  const uint32_t n = (uint32_t)tokens;
  timing_begin(kKernMx, stream);
  cudaError_t e;
  auto call = [&](auto* out) {
    using T = std::remove_pointer_t<decltype(out)>;
    return wg.format == PVT_MX_E4M3_16
               ? grad<T, PVT_MX_E4M3_16, false, true>(dgate, ldd, n, wg, out, lddx, false, status, sm_count, stream, dup, &wu)
               : grad<T, PVT_MX_E8M0_32, false, true>(dgate, ldd, n, wg, out, lddx, false, status, sm_count, stream, dup, &wu);
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

}  // namespace pvt
