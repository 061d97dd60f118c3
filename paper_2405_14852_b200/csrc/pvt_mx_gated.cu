// Two products on 4-bit matrices with the activation between them, h = f(x wg^T) (x wu^T), and its gradients by both products,
// dgate = dh b f'(a) and dup = dh f(a), from the 4-bit matrices again (a, b: the products; they are a ninth of a backward pass's
// operations, where keeping them would take four bytes an element and two more passes over memory).
//
// Up to 16 tokens: the product's kernel for few tokens, by clusters whose even blocks multiply by 128 rows of wg and whose odd ones by
// the same rows of wu, each pair its share of the steps.  A token's partial sums go to the block that finishes it, where they are added
// up in the order of ranks; behind the one barrier of the cluster no block needs another.
//
// From 17 tokens on: the product's pairs of blocks, 256 rows of weights by 256 (or 128) of x to a tile; but a block's 128 rows are 64
// of wg and the same 64 of wu.  The main loop, its traffic (32 KB of codes a step and SM) and its rate are the product's; only scales
// do not lie so in memory: a warp puts the tiles of 128 rows together, eight bytes of wg's and eight of wu's to sixteen, which the copy to
// tensor memory takes as one.  A tile's sums are read out of tensor memory, which is free for the next tile at once, turned in shared
// memory, where a thread finds a and b of the same eight outputs of a token, and finished beside the next tile's products.
// (128 rows of wg in one block and of wu in the other need no such scales, but every second sum has to go from one SM to the other: their
// exchange, in the same order as here, took 6000 cycles a tile of the 8192 that 4096 inputs multiply, gradients of 2048 x 4096 by 11008 93 us.)
//
// What bounds it.  4096 x 8192 by 28672 under e8m0: 640 us (6.0 PFLOP/s; 755 where the power limit holds the clock down), the tensor pipe 82 %
// active, the rest shared memory's bandwidth.  2048 x 4096 by 11008: 73 us, gradients 80: 16 steps a tile leave more to its end.  One token 4096 by 11008:
// 12 us (4.0 TB/s), of which 5 stream weights; 8.5 are behind the kernel ahead's end.
#include "pvt_mx_block.cuh"
#include "pvt_mx_mma.cuh"
#include "pvt_norm.cuh"

namespace pvt {
namespace {

using namespace mx;
using namespace mma;
using norm::with_type;

constexpr int kFewThreads = 192;  // four warps finish, one copies, one multiplies
constexpr int kFewCopyWarp = 4, kFewMmaWarp = 5;

// What becomes of a and b.  GRAD: dgate and dup, otherwise h, as floats, in 4 bits, or both.
struct Finish {
  int32_t activation, dtype;  // dtype: of h or dh
  void* h;                    // or null
  const void* dh;
  __nv_bfloat16 *dgate, *dup;
  int64_t ldh, ldd;
  bool wide;                  // eight neighbouring elements of h or dh begin on 16 bytes
  Held q;
  const float* x_ts;
  const float* gate_ts;
  const float* up_ts;
  uint32_t n, tokens;  // outputs, rows
  uint32_t padded;     // rows that have scales
};

// exp(-z) as a power of two (the product's rounding counts |z| times 2^-24), and 1 / v: the approximations, 2 units each
__device__ __forceinline__ float exp_minus(float z) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(z * -1.44269504088896f));
  return r;
}
__device__ __forceinline__ float inverse(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// f(a), and f'(a) if it is asked for.  (ACT is a constant: a branch for each element kept the elements of a thread from being worked at
// side by side, 2048 x 4096 by 11008: gradients 297 us, of which the products are 60.)
template <int ACT, bool SLOPE>
__device__ __forceinline__ float activate(float a, float* slope) {
  if (ACT == PVT_ACT_GELU) {  // f = a phi, phi the normal distribution's function
    // phi(-|a|) = exp(-a^2 / 2) g(t): a polynomial in t = 1 / (1 + 0.3 |a|), fitted to the least largest relative error for |a| up to 14,
    // beyond which the exponential is 0: 2^-24, and 2^-21.2 as binary32 works it out.  The slope takes the same exponential.  (erfcf and a
    // second exponential: 2048 x 4096 by 11008 92 us, gradients with dx 374, with this 77 and 355, with the other activations 73 and 345.)
    const float e = exp_minus(0.5f * a * a), t = inverse(fmaf(0.3f, fabsf(a), 1.0f));
    float g = fmaf(0.0383782895f, t, -0.169166111f);
    g = fmaf(g, t, 0.228660081f), g = fmaf(g, t, -0.0765064771f), g = fmaf(g, t, 0.142535524f), g = fmaf(g, t, 0.094683523f);
    g = fmaf(g, t, 0.121920342f), g = fmaf(g, t, 0.119487689f), g = fmaf(g, t, 7.16887583e-06f);
    const float phi = a > 0.0f ? fmaf(-e, g, 1.0f) : e * g;
    if (SLOPE) *slope = fmaf(a * 0.39894228040143268f, e, phi);
    return a * phi;
  }
  // f = a s(z), s the logistic function; z = a, or twice sqrt(2 / pi) (a + 0.044715 a^3): (1 + tanh(y)) / 2 = s(2 y)
  float z = a, dz = 1.0f;
  if (ACT == PVT_ACT_GELU_TANH) {
    const float sq = a * a;
    z = a * fmaf(sq, 0.07135481282942f, 1.59576912160573f);
    if (SLOPE) dz = fmaf(sq, 0.21406443848826f, 1.59576912160573f);
  }
  const float s = inverse(1.0f + exp_minus(z));  // (0 where the exponential is infinite)
  if (SLOPE) {
    const float rest = s * (1.0f - s);
    *slope = ACT == PVT_ACT_GELU_TANH && rest == 0.0f ? s : fmaf(a * dz, rest, s);  // (a dz / da is infinite from 1e13 on)
  }
  return a * s;
}
// calls f with the activation as a constant
template <typename F>
__device__ __forceinline__ void with_activation(int32_t which, F f) {
  if (which == PVT_ACT_SILU)
    f(std::integral_constant<int, PVT_ACT_SILU>{});
  else if (which == PVT_ACT_GELU)
    f(std::integral_constant<int, PVT_ACT_GELU>{});
  else
    f(std::integral_constant<int, PVT_ACT_GELU_TANH>{});
}

// dgate and dup of one element
template <int ACT>
__device__ __forceinline__ void gradients(float a, float b, float dh, float* gate, float* up) {
  float slope;
  const float f = activate<ACT, true>(a, &slope);
  *gate = dh * b * slope, *up = dh * f;
}

// A token of 128 outputs, lane, 32 + lane, ... of them to a lane; scratch: 128 floats of the warp's own.
template <int FMT, bool GRAD>
__device__ __forceinline__ void finish_token(const Finish& p, const TensorScale& t, uint32_t token, uint32_t col0, const float* a, const float* b,
                                             float* scratch) {
  const uint32_t lane = threadIdx.x & 31;
  if (GRAD) {
    with_type(p.dtype, [&](auto* type) {
      using T = std::remove_pointer_t<decltype(type)>;
      const T* const dh = static_cast<const T*>(p.dh) + (int64_t)token * p.ldh + col0 + lane;
      const int64_t at = (int64_t)token * p.ldd + col0 + lane;
      float v[4];
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) v[i] = col0 + i * 32 + lane < p.n ? widen<T>(dh[i * 32]) : 0.0f;
      float gate[4], up[4];
      with_activation(p.activation, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 4; ++i) gradients<decltype(act)::value>(a[i], b[i], v[i], &gate[i], &up[i]);
      });
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (col0 + i * 32 + lane < p.n)
          p.dgate[at + i * 32] = __float2bfloat16_rn(gate[i]), p.dup[at + i * 32] = __float2bfloat16_rn(up[i]);
    });
  } else {
    float h[4];
    with_activation(p.activation, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = activate<decltype(act)::value, false>(a[i], nullptr) * b[i];
    });
    if (p.h)
      with_type(p.dtype, [&](auto* type) {
        using T = std::remove_pointer_t<decltype(type)>;
        T* const to = static_cast<T*>(p.h) + (int64_t)token * p.ldh + col0 + lane;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
          if (col0 + i * 32 + lane < p.n) to[i * 32] = narrow<T>(h[i]);
      });
    if (p.q.codes) {
      __syncwarp();
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) scratch[i * 32 + lane] = h[i];
      __syncwarp();
      float v[8];
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) v[i] = lane < 16 ? scratch[8 * lane + i] : 0.0f;
      // (the upper lanes: the next 128 columns, which are another block's, or of which there are scales but no outputs)
      const bool own = lane < 16 || col0 + 128 >= p.n;
      put_eight<FMT>(p.q, token, col0 + 8 * lane, own, own, t, v);
    }
  }
}
// scales of rows that do not exist, of the 128 outputs from col0 on and of what is behind the last output; thread `i` of `count`
template <int FMT>
__device__ __forceinline__ void clear_scales(const Finish& p, uint32_t from, uint32_t to, uint32_t col0, uint32_t i, uint32_t count) {
  constexpr uint32_t BLOCK = FMT == PVT_MX_E8M0_32 ? 32 : 16, WORDS = 128 / (4 * BLOCK);
  const uint32_t words = col0 + 128 < p.n ? WORDS : 2 * WORDS;
  for (uint32_t at = from * words + i; at < to * words; at += count) {
    const uint32_t block = col0 / BLOCK + at % words * 4;
    if (block / 4 < p.q.tiles) *reinterpret_cast<uint32_t*>(p.q.scales + scale_at(at / words, block, p.q.tiles)) = 0;
  }
}

// ---- few tokens ------------------------------------------------------------------------------------------------
struct FewParams {
  const uint8_t *gate_codes, *up_codes, *gate_scales, *up_scales, *x_scales;
  int64_t gate_ld, up_ld;
  Finish f;
  uint32_t* status;
  uint32_t row_bytes;    // of weights, to the last 16 that hold codes
  uint32_t strip_bytes;  // scales of a strip of 128 rows
  uint32_t steps;        // of 256 columns
  uint32_t split;        // pairs per tile
  uint32_t max_spins, withhold;
};

struct FewShared {
  alignas(8) uint64_t full[8];
  uint64_t empty[8];
  uint64_t done, spare;
  uint32_t tmem, abandoned;
};

// the product's, but for shared memory that the cluster's sums have to themselves: other blocks write there while this one multiplies
template <int FMT>
struct GatedFewSizes : FewSizes<FMT> {
  using F = FewSizes<FMT>;
  static constexpr uint32_t kStages = 104 * 1024 / F::kStageAligned;  // of two blocks per SM
  static constexpr uint32_t kSumsAt = kStages * F::kStageAligned;
  static constexpr size_t kBytes = kSumsAt + kFewTokens * kTileW * 4 + 1024;
};

template <int FMT, bool GRAD>
__global__ void __launch_bounds__(kFewThreads)
    mx_gated_few_kernel(const __grid_constant__ CUtensorMap gate_map, const __grid_constant__ CUtensorMap up_map,
                        const __grid_constant__ CUtensorMap x_map, const __grid_constant__ FewParams p) {
  using S = GatedFewSizes<FMT>;
  constexpr uint32_t KT = S::KT, STAGES = S::kStages;
  extern __shared__ __align__(1024) unsigned char raw[];
  __shared__ FewShared sm;
  __shared__ float scratch[4][128];
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile uint32_t* abandoned = &sm.abandoned;
  const uint32_t blocks = 2 * p.split, rank = blockIdx.x % blocks, w0 = blockIdx.x / blocks * kTileW;
  const bool of_up = rank & 1;
  const uint32_t first = p.steps * (rank / 2) / p.split, last = p.steps * (rank / 2 + 1) / p.split;  // (steps < 2^20, split <= 4)
  const uint8_t* const w_scales = (of_up ? p.up_scales : p.gate_scales) + (size_t)(w0 / kStrip) * p.strip_bytes;
  // all of the block's weights at once, while it sets itself up and the kernel ahead ends
  const uint32_t from_byte = first * kRowBytes, to_byte = min(last * kRowBytes, p.row_bytes);
  if (tid < (uint32_t)kTileW && w0 + tid < p.f.n)
    prefetch_l2((of_up ? p.up_codes : p.gate_codes) + (int64_t)(w0 + tid) * (of_up ? p.up_ld : p.gate_ld) + from_byte, to_byte - from_byte);
  if (tid == (uint32_t)kTileW) prefetch_l2(w_scales + (size_t)first * (KT * kTileBytes), (last - first) * (KT * kTileBytes));
  if (tid == kTileW + 1) {  // (descriptors, which the launch has brought along)
    asm volatile("prefetch.tensormap [%0];" ::"l"(of_up ? &up_map : &gate_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&x_map) : "memory");
  }
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
  if (warp == kFewMmaWarp) {
    tmem_alloc(smem_u32(&sm.tmem), S::kTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();  // not before this block has its tensor memory: the next kernel's blocks hold theirs while they wait for this one
  pdl_wait();
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // that this block has started; awaited where others' memory is written

  const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sm.tmem);
  const Finish& f = p.f;
  const float* const sums = reinterpret_cast<const float*>(raw + (base - smem_u32(raw)) + S::kSumsAt);
  const uint32_t log = 31 - __clz((int)blocks), slots = kFewTokens >> log;  // tokens of a block (of two, four or eight)
  auto all_started = [] {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  };
  Factors gate(1.0f, 1.0f), up(1.0f, 1.0f);
  TensorScale t(nullptr);

  if (warp == kFewCopyWarp) {
    const CUtensorMap* const w_map = of_up ? &up_map : &gate_map;
    uint32_t i = 0;
    for (uint32_t step = first; step < last; ++step, ++i) {
      const uint32_t s = i % STAGES, bar = smem_u32(&sm.full[s]), to = base + s * S::kStageAligned;
      if (i >= STAGES && !wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins)) break;
      if (i == p.withhold) continue;  // test hook: never issued
      expect_bytes(bar, S::kStage);
      tma_load(to, w_map, (int)(step * kRowBytes), (int)w0, bar);
      tma_load(to + S::kX, &x_map, (int)(step * kRowBytes), 0, bar);
      bulk_load(to + S::kWs, w_scales + (size_t)step * (KT * kTileBytes), KT * kTileBytes, bar);
      bulk_load(to + S::kXs, p.x_scales + (size_t)step * (KT * kTileBytes), KT * kTileBytes, bar);
    }
    if (*abandoned)  // what was issued lands before the block's memory is another's
      for (uint32_t j = i > STAGES ? i - STAGES : 0; j < i; ++j)
        if (j != p.withhold) drain(smem_u32(&sm.full[j % STAGES]), (j / STAGES) & 1);
    all_started();
  } else if (warp == kFewMmaWarp) {
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
    all_started();
  } else {
    const float x_ts = f.x_ts ? *f.x_ts : 1.0f;
    gate = Factors(f.gate_ts ? *f.gate_ts : 1.0f, x_ts), up = Factors(f.up_ts ? *f.up_ts : 1.0f, x_ts);
    t = TensorScale(f.q.tensor_scale);
    all_started();
    if (wait(smem_u32(&sm.done), 0, abandoned, p.status, p.max_spins)) {
      tc_fence_after();
      uint32_t v[kFewTokens];
      tmem_ld16(tmem + (warp << 21), v);
      tmem_ld_wait<kFewTokens>(v);
      const uint32_t to = base + S::kSumsAt + (rank * slots * kTileW + tid) * 4;
#pragma unroll
      for (uint32_t j = 0; j < kFewTokens; ++j)
        if (j < f.tokens)
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_address(to + (j >> log) * (kTileW * 4), j & (blocks - 1))), "r"(v[j])
                       : "memory");
      tc_fence_before();
    }
    if (!GRAD && f.q.codes && rank == 0) clear_scales<FMT>(f, f.tokens, f.padded, w0, tid, 128);
  }
  cluster_sync();  // a block's sums are there, from all of its cluster
  if (warp < 4 && !*abandoned)
    for (uint32_t k = warp; rank + k * blocks < f.tokens; k += 4) {  // a token to a warp
      float a[4] = {0.0f, 0.0f, 0.0f, 0.0f}, b[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      for (uint32_t q = 0; q < p.split; ++q)
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
          a[i] += sums[(2 * q * slots + k) * kTileW + i * 32 + lane];
          b[i] += sums[((2 * q + 1) * slots + k) * kTileW + i * 32 + lane];
        }
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) a[i] = gate(a[i]), b[i] = up(b[i]);
      finish_token<FMT, GRAD>(f, t, rank + k * blocks, w0, a, b, scratch[warp]);
    }
  __syncthreads();
  if (warp == kFewMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kTmem);
  }
}

// ---- pairs of blocks -------------------------------------------------------------------------------------------
// Sixteen warps finish: with eight there were two to a scheduler, and most of the time neither could go on.
constexpr int kReaders = 16, kCopyWarp = kReaders, kMmaWarp = kCopyWarp + kPairCopyWarps, kScaleWarp = kMmaWarp + 1;
constexpr int kThreads = (kScaleWarp + 1) * 32;
constexpr uint32_t kOutputs = 64;               // of a block
constexpr uint32_t kRound = 16;                 // tokens that two warps, one with a and one with b, turn at a time
constexpr uint32_t kSums = kRound * 32 * 4;     // bytes of either

struct PairShared {
  alignas(8) uint64_t full[kPairStages];  // of the first block: bytes of both
  uint64_t raw[kPairStages];              // of each: the weights' scales as they lie in memory
  uint64_t scaled[kPairStages];           // of the first: these have been put together in both
  uint64_t empty[kPairStages];            // of each
  uint64_t sums_full;                     // of each
  uint64_t sums_empty;                    // of the first: an arrival per reading warp of both
  uint64_t spare;
  uint32_t tmem, abandoned;
};

struct PairParams {
  Finish f;
  uint32_t* status;
  uint32_t strip_rows;  // rows of 128 bytes that a strip's scales are
  uint32_t steps;       // of 256 columns
  uint32_t x_tiles, tiles;
  uint32_t split;       // pairs per tile
  uint32_t max_spins, withhold;
};

template <int FMT, uint32_t N>
struct GatedSizes {
  static constexpr uint32_t KT = FMT == PVT_MX_E8M0_32 ? 2 : 4, kStrips = N / kStrip;
  // a stage: rows of weights, rows of x, scales of x, scales of the weights put together, and of either as they lie in memory
  static constexpr uint32_t kX = kTileW * kRowBytes, kXs = kX + N / 2 * kRowBytes, kWs = kXs + kStrips * KT * kTileBytes;
  static constexpr uint32_t kRaw = kWs + KT * kTileBytes, kStage = kRaw + 2 * KT * kTileBytes, kStageAligned = (kStage + 1023) / 1024 * 1024;
  static constexpr uint32_t kScaleCols = KT * 4 * (1 + kStrips);  // of a stage
  static constexpr uint32_t kRoom = (225 * 1024 - kReaders * kSums) / kStageAligned, kMost = N == 256 ? 5 : 7;
  static constexpr uint32_t kStages = kRoom < kMost ? kRoom : kMost;
  static_assert(N + kStages * kScaleCols <= 512 && kStages <= kPairStages, "sums and scales fit tensor memory");
  static constexpr uint32_t kTurnAt = kStages * kStageAligned;
  static constexpr size_t kBytes = kTurnAt + kReaders * kSums + 1024;
  static_assert(kBytes + 1024 <= 227 * 1024, "a block's shared memory");
  static_assert(N * kTileW * 4 <= kTurnAt, "the partial sums fit the stages");
};

// asks for the line of an address to be brought into the L2
__device__ __forceinline__ void ask_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p) : "memory"); }

// two warps of a block, `id` of their own; with `ok` of both if both have it
__device__ __forceinline__ void pair_sync(uint32_t id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool pair_agrees(uint32_t id, bool ok) {
  uint32_t both;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %2, 0;\n\t"
      "barrier.cta.red.and.pred q, %1, 64, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(both)
      : "r"(id), "r"((uint32_t)ok)
      : "memory");
  return both != 0;
}

// Where sums of a round lie: 32 outputs of a token to 128 bytes, in pieces of four whose places in it are exchanged by the token, so that
// no bank is met twice either by lanes that have an output each or by four lanes to a token with eight outputs each.
__device__ __forceinline__ uint32_t place(uint32_t token, uint32_t output) { return token * 32 + (output ^ (token & 7) * 4); }

// Where partial sums of a tile lie: 64 of a and 64 of b to a token, in pieces of four, the even ones ahead of the odd ones, these exchanged by
// fours: no bank is met twice either by lanes that have an output each or by eight that have two pieces each.
__device__ __forceinline__ uint32_t piece_at(uint32_t piece) { return piece % 2 ? 8 + (piece / 2 ^ 4) : piece / 2; }

// eight neighbouring elements, rounded; `left` of them exist
template <typename T>
__device__ __forceinline__ void put8(T* to, const float* v, bool wide, uint32_t left) {
  if (wide && left >= 8) {
    if constexpr (sizeof(T) == 4) {
      reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      Eight<T> e;
#pragma unroll
      for (int i = 0; i < 8; i += 2) norm::narrow_pair(v[i], v[i + 1], &e.v[i]);
      *reinterpret_cast<Eight<T>*>(to) = e;
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < left) to[i] = narrow<T>(v[i]);
  }
}

// Eight outputs of a token, from column c on, into 4 bits: four lanes have 32 of them.  (here: the token exists.)
template <int FMT>
__device__ __forceinline__ void put_four_bits(const Finish& p, const TensorScale& t, uint32_t token, uint32_t c, bool here, float* v) {
  constexpr uint32_t BLOCK = FMT == PVT_MX_E8M0_32 ? 32 : 16;
  uint32_t word;
  if (c + 8 > p.n) {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (c + i >= p.n) v[i] = 0.0f;
  }
  uint32_t top = top_of8(v);
#pragma unroll
  for (uint32_t d = 1; d < BLOCK / 8; d *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
  uint32_t bytes = quantize_block<FMT, 8>(v, top, t, &word);
  if (!here || c >= p.n) bytes = 0;  // scales of what does not exist
  if (FMT == PVT_MX_E4M3_16) bytes |= __shfl_down_sync(0xffffffffu, bytes, 2) << 8;
  if (threadIdx.x % 4 == 0 && token < p.padded) {
    auto put_scales = [&](uint32_t col, uint32_t value) {
      if (col / BLOCK / 4 >= p.q.tiles) return;
      uint8_t* const to = p.q.scales + scale_at(token, col / BLOCK, p.q.tiles);
      if (FMT == PVT_MX_E8M0_32)
        *to = (uint8_t)value;
      else
        *reinterpret_cast<uint16_t*>(to) = (uint16_t)value;
    };
    put_scales(c, bytes);
    if (c / 128 == (p.n - 1) / 128) put_scales(c + 128, 0);  // (blocks of no outputs at all)
  }
  if (!here || c >= p.n) return;
  uint8_t* const to = p.q.codes + (int64_t)token * p.q.ld + c / 2;
  if (c + 8 <= p.n) {
    *reinterpret_cast<uint32_t*>(to) = word;
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      if (2 * i < p.n - c) to[i] = (uint8_t)(word >> (8 * i));
  }
}

// eight elements of dh as they lie in memory
struct EightOfDh {
  uint32_t w[8];
  __device__ __forceinline__ void ask(const Finish& p, uint32_t token, uint32_t c, uint32_t left) {
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = 0;
    if (token >= p.tokens || left == 0) return;
    const int64_t at = (int64_t)token * p.ldh + c;
    if (p.dtype == PVT_F32) {
      const uint32_t* const from = static_cast<const uint32_t*>(p.dh) + at;
      if (p.wide && left >= 8) {
        const uint4 a = reinterpret_cast<const uint4*>(from)[0], b = reinterpret_cast<const uint4*>(from)[1];
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
      } else {
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
          if (k < left) w[k] = from[k];
      }
    } else {
      const uint16_t* const from = static_cast<const uint16_t*>(p.dh) + at;
      if (p.wide && left >= 8) {
        const uint4 a = *reinterpret_cast<const uint4*>(from);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
      } else {
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
          if (k < left) w[k / 2] |= (uint32_t)from[k] << (k % 2 * 16);
      }
    }
  }
  __device__ __forceinline__ void values(int32_t dtype, float* d) const {
    if (dtype == PVT_F32) {
#pragma unroll
      for (int k = 0; k < 8; ++k) d[k] = __uint_as_float(w[k]);
    } else if (dtype == PVT_BF16) {
#pragma unroll
      for (int k = 0; k < 8; ++k) d[k] = __uint_as_float(k % 2 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) d[k] = __half2float(__ushort_as_half((unsigned short)(w[k / 2] >> (k % 2 * 16))));
    }
  }
};

// Eight outputs of a token, from column c on; all lanes of a warp call.  turn: shared memory for eight tokens of 32 outputs (place()) that
// is this warp's for now, or null: where rows of h have no alignment they go out by way of it, so that a warp stores along them.
template <int FMT, bool GRAD, int ACT>
__device__ __forceinline__ void finish8(const Finish& p, const TensorScale& t, uint32_t token, uint32_t c, const float* a, const float* b,
                                        const EightOfDh& dh, float* turn = nullptr) {
  const uint32_t left = c < p.n ? p.n - c : 0;  // outputs that exist
  const bool here = token < p.tokens;
  if (GRAD) {
    float d[8], gate[8], up[8];
    dh.values(p.dtype, d);
#pragma unroll
    for (int k = 0; k < 8; ++k) gradients<ACT>(a[k], b[k], d[k], &gate[k], &up[k]);
    if (here) {
      const int64_t at = (int64_t)token * p.ldd + c;
      put8(p.dgate + at, gate, true, left);
      put8(p.dup + at, up, true, left);
    }
  } else {
    float h[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = activate<ACT, false>(a[k], nullptr) * b[k];
    if (turn) {
      const uint32_t lane = threadIdx.x & 31, token0 = token - lane / 4, col = c - lane % 4 * 8 + lane;
      __syncwarp();
#pragma unroll
      for (uint32_t k = 0; k < 8; k += 4)
        *reinterpret_cast<float4*>(turn + place(lane / 4, lane % 4 * 8 + k)) = make_float4(h[k], h[k + 1], h[k + 2], h[k + 3]);
      __syncwarp();
      with_type(p.dtype, [&](auto* type) {
        using T = std::remove_pointer_t<decltype(type)>;
        T* const to = static_cast<T*>(p.h) + (int64_t)token0 * p.ldh + col;
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
          if (token0 + k < p.tokens && col < p.n) to[k * p.ldh] = narrow<T>(turn[place(k, lane)]);
      });
    } else if (p.h && here) {
      with_type(p.dtype, [&](auto* type) {
        using T = std::remove_pointer_t<decltype(type)>;
        put8(static_cast<T*>(p.h) + (int64_t)token * p.ldh + c, h, p.wide, left);
      });
    }
    if (p.q.codes) put_four_bits<FMT>(p, t, token, c, here, h);
  }
}

template <int FMT, uint32_t N, bool GRAD>
__global__ void __launch_bounds__(kThreads, 1)
    mx_gated_pair_kernel(const __grid_constant__ CUtensorMap gate_map, const __grid_constant__ CUtensorMap up_map,
                         const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap gate_s_map,
                         const __grid_constant__ CUtensorMap up_s_map, const __grid_constant__ CUtensorMap x_s_map,
                         const __grid_constant__ PairParams p) {
  using S = GatedSizes<FMT, N>;
  constexpr uint32_t KT = S::KT, STAGES = S::kStages, PART = N / 4;
  extern __shared__ __align__(1024) unsigned char raw[];
  __shared__ PairShared sm;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile uint32_t* abandoned = &sm.abandoned;
  if (tid == 0) {
    sm.abandoned = 0;
    for (uint32_t s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&sm.full[s]), 1);
      mbar_init(smem_u32(&sm.raw[s]), 1);
      mbar_init(smem_u32(&sm.scaled[s]), 2);
      mbar_init(smem_u32(&sm.empty[s]), 1);
    }
    mbar_init(smem_u32(&sm.sums_full), 1);
    mbar_init(smem_u32(&sm.sums_empty), 2 * kReaders);
    mbar_init(smem_u32(&sm.spare), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
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
  // Pairs by themselves take tile after tile; those of a cluster share one tile's steps.
  const uint32_t in_cluster = cluster_rank(), rank = in_cluster & 1, lead = in_cluster & ~1u, share = in_cluster / 2;
  const uint32_t tile0 = blockIdx.x / 2 / p.split, stride = p.split > 1 ? p.tiles : gridDim.x / 2;
  const uint32_t first = p.steps * share / p.split, steps = p.steps * (share + 1) / p.split - first;  // (steps < 2^24, share < 4)
  const Finish& f = p.f;

  if (warp >= kCopyWarp && warp < kMmaWarp) {
    const bool of_w = warp == kCopyWarp;  // one warp for the weights' codes and scales, one for x's
    uint32_t i = 0;
    bool ok = true;
    for (uint32_t tile = tile0; tile < p.tiles && ok; tile += stride) {
      const uint32_t row0 = of_w ? tile / p.x_tiles * kTileW : tile % p.x_tiles * N;
      const int row = (int)(row0 + rank * (of_w ? kOutputs : N / 2));
      const int strip = (int)(row0 / kStrip * p.strip_rows);
      for (uint32_t step = first; step < first + steps; ++step, ++i) {
        const uint32_t s = i % STAGES, to = base + s * S::kStageAligned;
        if (i >= STAGES && !(ok = wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins))) break;
        if (i == p.withhold) continue;  // test hook: never issued
        const uint32_t bar = cluster_address(smem_u32(&sm.full[s]), lead);
        const int col = (int)(step * kRowBytes), scales = strip + (int)(step * (KT * 4));
        if (of_w) {
          if (rank == 0) expect_bytes(smem_u32(&sm.full[s]), 2 * S::kWs);
          expect_bytes(smem_u32(&sm.raw[s]), 2 * KT * kTileBytes);
          tma_load(to + S::kRaw, &gate_s_map, 0, scales, smem_u32(&sm.raw[s]));
          tma_load(to + S::kRaw + KT * kTileBytes, &up_s_map, 0, scales, smem_u32(&sm.raw[s]));
          tma_load_pair(to, &gate_map, col, row, bar);
          tma_load_pair(to + kOutputs * kRowBytes, &up_map, col, row, bar);
        } else {  // both blocks multiply by all of the tile's rows of x
          tma_load_pair(to + S::kX, &x_map, col, row, bar);
          tma_load_pair(to + S::kXs, &x_s_map, 0, scales, bar);
          if (S::kStrips == 2) tma_load_pair(to + S::kXs + KT * kTileBytes, &x_s_map, 0, scales + (int)p.strip_rows, bar);
        }
      }
    }
    if (*abandoned)  // what was issued lands before the blocks' memory is another's
      for (uint32_t j = i > STAGES ? i - STAGES : 0; j < i; ++j)
        if (j != p.withhold) {
          if (rank == 0) drain(smem_u32(&sm.full[j % STAGES]), (j / STAGES) & 1);
          if (of_w) drain(smem_u32(&sm.raw[j % STAGES]), (j / STAGES) & 1);
        }
  } else if (warp == kMmaWarp) {
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
          ok = wait_both(smem_u32(&sm.full[s]), smem_u32(&sm.scaled[s]), (i / STAGES) & 1, abandoned, p.status, p.max_spins);
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
  } else if (warp == kScaleWarp) {
    // Scales of row r lie in 16 bytes of r % 32, four to each of four rows 32 apart: of the strip's 128 rows this block has the first or the
    // last 64 of either matrix, eight bytes.
    const uint32_t left = tile0 < p.tiles ? (p.tiles - tile0 + stride - 1) / stride : 0;
    const uint32_t scaled0 = cluster_address(smem_u32(&sm.scaled[0]), lead);
    uint32_t i = 0;
    bool ok = true;
    for (uint32_t n = 0; n < left && ok; ++n)
      for (uint32_t step = 0; step < steps; ++step, ++i) {
        const uint32_t s = i % STAGES;
        if (!(ok = wait(smem_u32(&sm.raw[s]), (i / STAGES) & 1, abandoned, p.status, p.max_spins))) break;
        unsigned char* const stage = mem + s * S::kStageAligned;
#pragma unroll
        for (uint32_t t = 0; t < KT; ++t) {
          const uint2 g = *reinterpret_cast<const uint2*>(stage + S::kRaw + t * kTileBytes + lane * 16 + rank * 8);
          const uint2 u = *reinterpret_cast<const uint2*>(stage + S::kRaw + (KT + t) * kTileBytes + lane * 16 + rank * 8);
          *reinterpret_cast<uint4*>(stage + S::kWs + t * kTileBytes + lane * 16) = make_uint4(g.x, g.y, u.x, u.y);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // generic-proxy writes -> visible to the products
        __syncwarp();
        if (lane == 0) cluster_arrive(scaled0 + s * 8);
        __syncwarp();
      }
  } else {
    const float x_ts = f.x_ts ? *f.x_ts : 1.0f;
    const Factors gate(f.gate_ts ? *f.gate_ts : 1.0f, x_ts), up(f.up_ts ? *f.up_ts : 1.0f, x_ts);
    const bool scaled = !(gate.first == 1.0f && gate.second == 1.0f && up.first == 1.0f && up.second == 1.0f);
    const TensorScale t(f.q.tensor_scale);
    // A quarter of tensor memory's lanes, which have a (the lower two) or b of 32 outputs, and a quarter of the tokens.  The warp with b of the
    // same outputs and tokens, or a, is its partner: both turn 16 tokens at a time, and each finishes eight of them.
    const uint32_t quarter = warp % 4, part = warp / 4, of_b = quarter / 2, pair = part * 2 + quarter % 2;
    const uint32_t sums_empty = cluster_address(smem_u32(&sm.sums_empty), lead);
    float* const a_sums = reinterpret_cast<float*>(mem + S::kTurnAt + pair * (2 * kSums));
    float* const b_sums = a_sums + kSums / 4;
    float* const own = of_b ? b_sums : a_sums;
    const uint32_t j = of_b * 8 + lane / 4;  // token of a round
    const bool turned = !GRAD && f.h && !f.wide;
    uint32_t n = 0;
    bool ok = true;
    for (uint32_t tile = tile0; tile < p.tiles && ok; tile += stride, ++n) {
      const uint32_t c = tile / p.x_tiles * kTileW + rank * kOutputs + quarter % 2 * 32 + lane % 4 * 8;
      const uint32_t row = tile % p.x_tiles * N + part * PART, left = c < f.n ? f.n - c : 0;
      if (GRAD && p.split == 1 && left > 0)  // what will be needed of dh, on its way to the L2 beside the products
        for (uint32_t r = 0; r < PART; r += kRound)
          if (row + r + j < f.tokens)
            ask_l2(static_cast<const char*>(f.dh) + ((int64_t)(row + r + j) * f.ldh + c) * (f.dtype == PVT_F32 ? 4 : 2));
      ok = pair_agrees(pair + 1, wait(smem_u32(&sm.sums_full), n & 1, abandoned, p.status, p.max_spins));
      if (!ok) break;
      tc_fence_after();
      uint32_t v[PART];
#pragma unroll
      for (uint32_t k = 0; k < PART; k += 32) tmem_ld32(tmem + (quarter << 21) + part * PART + k, v + k);
      tmem_ld_wait<(int)PART>(v);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) cluster_arrive(sums_empty);
      __syncwarp();
      if (p.split > 1) {  // the products are done: the stages hold the partial sums
        const uint32_t at = piece_at(quarter % 2 * 8 + lane / 4) * 4 + lane % 4;
#pragma unroll
        for (uint32_t k = 0; k < PART; ++k)
          reinterpret_cast<float*>(mem)[(part * PART + k) * kTileW + of_b * kOutputs + at] = __uint_as_float(v[k]);
        break;
      }
      with_activation(f.activation, [&](auto act) {
        EightOfDh dh;
        if (GRAD) dh.ask(f, row + j, c, left);
#pragma unroll
        for (uint32_t r = 0; r < PART; r += kRound) {
#pragma unroll
          for (uint32_t k = 0; k < kRound; ++k) own[place(k, lane)] = __uint_as_float(v[r + k]);
          pair_sync(pair + 1);
          float a[8], b[8];
#pragma unroll
          for (uint32_t k = 0; k < 8; k += 4) {
            const float4 x = *reinterpret_cast<const float4*>(a_sums + place(j, lane % 4 * 8 + k));
            const float4 y = *reinterpret_cast<const float4*>(b_sums + place(j, lane % 4 * 8 + k));
            a[k] = x.x, a[k + 1] = x.y, a[k + 2] = x.z, a[k + 3] = x.w, b[k] = y.x, b[k + 1] = y.y, b[k + 2] = y.z, b[k + 3] = y.w;
          }
          if (!turned) pair_sync(pair + 1);  // (the next round's sums may come)
          if (scaled) {
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
              set2(a + k, mul2(mul2(two(a + k), both(gate.first)), both(gate.second)));
              set2(b + k, mul2(mul2(two(b + k), both(up.first)), both(up.second)));
            }
          }
          EightOfDh now = dh;
          if (GRAD && r + kRound < PART) dh.ask(f, row + r + kRound + j, c, left);
          finish8<FMT, GRAD, decltype(act)::value>(f, t, row + r + j, c, a, b, now, turned ? a_sums + of_b * 256 : nullptr);
          if (turned) pair_sync(pair + 1);
        }
      });
      __syncwarp();
    }
  }
  __syncthreads();
  cluster_sync();  // neither block leaves while the other's copies, products or arrivals reach it
  if (p.split > 1) {
    // every pair adds up and finishes the tokens that are its share, four to a warp, always in the order of pairs; a lane has eight outputs
    const uint32_t col0 = tile0 / p.x_tiles * kTileW + rank * kOutputs, row0 = tile0 % p.x_tiles * N;
    if (!*abandoned) {
      const float x_ts = f.x_ts ? *f.x_ts : 1.0f;
      const Factors gate(f.gate_ts ? *f.gate_ts : 1.0f, x_ts), up(f.up_ts ? *f.up_ts : 1.0f, x_ts);
      const TensorScale t(f.q.tensor_scale);
      const uint32_t c = col0 + lane % 8 * 8, left = c < f.n ? f.n - c : 0;
      for (uint32_t j0 = (share + warp * p.split) * 4; j0 < N; j0 += kThreads / 32 * p.split * 4) {
        const uint32_t j = j0 + lane / 8, token = row0 + j;
        EightOfDh dh;
        if (GRAD) dh.ask(f, token, c, left);
        float a[8], b[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) a[k] = b[k] = 0.0f;
        if (row0 + j0 < f.tokens)
          for (uint32_t q = 0; q < p.split; ++q) {
            float4 x[2], y[2];  // (all under way at once: a load from another block takes a thousand cycles)
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k) {
              const uint32_t at = base + (j * kTileW + piece_at(lane % 8 * 2 + k) * 4) * 4;
              x[k] = cluster_load4(at, 2 * q + rank), y[k] = cluster_load4(at + kOutputs * 4, 2 * q + rank);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              a[4 * k] += x[k].x, a[4 * k + 1] += x[k].y, a[4 * k + 2] += x[k].z, a[4 * k + 3] += x[k].w;
              b[4 * k] += y[k].x, b[4 * k + 1] += y[k].y, b[4 * k + 2] += y[k].z, b[4 * k + 3] += y[k].w;
            }
          }
#pragma unroll
        for (int k = 0; k < 8; ++k) a[k] = gate(a[k]), b[k] = up(b[k]);
        with_activation(f.activation, [&](auto act) { finish8<FMT, GRAD, decltype(act)::value>(f, t, token, c, a, b, dh); });
      }
    }
    cluster_sync();  // nor while another reads its partial sums
  }
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc<2>(tmem, 512);
  }
}

template <int FMT, uint32_t N, bool GRAD>
cudaError_t gated_pairs(const pvt_mx& x, const pvt_mx& wg, const pvt_mx& wu, const Finish& f, uint32_t* status, int sm_count,
                        cudaStream_t stream) {
  using S = GatedSizes<FMT, N>;
  PairParams p = {};
  p.f = f, p.status = status;
  p.strip_rows = strip_tiles(x.cols, block_of(FMT)) * (kTileBytes / 128);
  p.steps = ((uint32_t)x.cols + kSpan - 1) / kSpan;
  p.x_tiles = (f.tokens + N - 1) / N;
  p.tiles = (f.n + kTileW - 1) / kTileW * p.x_tiles;
  const m1::WaitTestHook hook = m1::wait_test_hook();
  p.max_spins = hook.max_spins, p.withhold = hook.withhold_copy;
  CUtensorMap maps[6];
  const pvt_mx* const of[3] = {&wg, &wu, &x};
  for (int i = 0; i < 3; ++i) {
    cudaError_t e = make_map(&maps[i], of[i]->codes, 1, (uint64_t)of[i]->rows, ((uint64_t)of[i]->cols + 1) / 2, (uint64_t)of[i]->ld,
                             i < 2 ? kOutputs : N / 2);
    if (e == cudaSuccess)
      e = make_map(&maps[3 + i], of[i]->scales, 1, scale_bytes(of[i]->rows, of[i]->cols, FMT) / 128, 128, 128, S::KT * 4, 128, false);
    if (e != cudaSuccess) return e;
  }
  const cudaError_t e = allow_smem<mx_gated_pair_kernel<FMT, N, GRAD>>();
  if (e != cudaSuccess) return e;
  // Few tiles: up to four pairs to each, as long as all clusters run at once and a pair keeps eight steps.  By one, two and four pairs, 100
  // tokens 8192 by 1024 14.5, 10.9 and 9.1 us; by one and two, 64 tokens 11008 by 4096 18.9 and 13.8, 77 tokens 4096 by 4096 9.7 and 8.9, 128
  // tokens 2048 by 4096 (four steps each) 7.3 and 8.3.
  p.split = 1;
  for (uint32_t n = 2; n <= 4 && 8 * n <= p.steps && (uint64_t)p.tiles * 2 * n <= (uint64_t)sm_count; ++n)
    if (p.tiles <= clusters_at_once<mx_gated_pair_kernel<FMT, N, GRAD>>(2 * n, kThreads, S::kBytes)) p.split = n;
  const uint32_t pairs = p.split > 1 ? p.tiles * p.split : p.tiles < (uint32_t)sm_count / 2 ? p.tiles : (uint32_t)sm_count / 2;
  return launch_clusters(mx_gated_pair_kernel<FMT, N, GRAD>, 2 * pairs, 2 * p.split, kThreads, S::kBytes, stream, maps[0], maps[1],
                         maps[2], maps[3], maps[4], maps[5], p);
}

template <int FMT, bool GRAD>
cudaError_t gated(const pvt_mx& x, const pvt_mx& wg, const pvt_mx& wu, const Finish& f, uint32_t* status, int sm_count, cudaStream_t stream) {
  using S = GatedFewSizes<FMT>;
  const uint64_t tiles = ((uint64_t)f.n + kTileW - 1) / kTileW;
  if (f.tokens > kFewTokens)
    return narrow_tiles((int32_t)f.tokens, tiles, sm_count) ? gated_pairs<FMT, 128, GRAD>(x, wg, wu, f, status, sm_count, stream)
                                                            : gated_pairs<FMT, 256, GRAD>(x, wg, wu, f, status, sm_count, stream);
  FewParams p = {};
  p.gate_codes = wg.codes, p.gate_scales = wg.scales, p.gate_ld = wg.ld, p.up_codes = wu.codes, p.up_scales = wu.scales, p.up_ld = wu.ld;
  p.x_scales = x.scales, p.f = f, p.status = status;
  p.row_bytes = ((uint32_t)x.cols + 31) / 32 * 16;
  p.strip_bytes = strip_tiles(x.cols, block_of(FMT)) * kTileBytes;
  p.steps = ((uint32_t)x.cols + kSpan - 1) / kSpan;
  p.split = 1;
  while (p.split < 4 && tiles * p.split * 4 <= (uint64_t)sm_count * 2 && p.split * 2 <= p.steps) p.split *= 2;
  const m1::WaitTestHook hook = m1::wait_test_hook();
  p.max_spins = hook.max_spins, p.withhold = hook.withhold_copy;
  CUtensorMap maps[3];
  const pvt_mx* const of[3] = {&wg, &wu, &x};
  for (int i = 0; i < 3; ++i) {
    const cudaError_t e = make_map(&maps[i], of[i]->codes, 1, (uint64_t)of[i]->rows, ((uint64_t)of[i]->cols + 1) / 2, (uint64_t)of[i]->ld,
                                   i < 2 ? kTileW : kFewTokens);
    if (e != cudaSuccess) return e;
  }
  const cudaError_t e = allow_smem<mx_gated_few_kernel<FMT, GRAD>>();
  if (e != cudaSuccess) return e;
  return launch_clusters(mx_gated_few_kernel<FMT, GRAD>, (unsigned)(tiles * p.split * 2), 2 * p.split, kFewThreads, S::kBytes, stream, maps[0],
                         maps[1], maps[2], p);
}

template <bool GRAD>
cudaError_t gated(const pvt_mx& x, const pvt_mx& wg, const pvt_mx& wu, Finish f, uint32_t* status, int sm_count, cudaStream_t stream) {
  f.x_ts = x.tensor_scale, f.gate_ts = wg.tensor_scale, f.up_ts = wu.tensor_scale;
  f.n = (uint32_t)wg.rows, f.tokens = (uint32_t)x.rows, f.padded = (f.tokens + kStrip - 1) / kStrip * kStrip;
  timing_begin(kKernMx, stream);
  const cudaError_t e = x.format == PVT_MX_E8M0_32 ? gated<PVT_MX_E8M0_32, GRAD>(x, wg, wu, f, status, sm_count, stream)
                                                   : gated<PVT_MX_E4M3_16, GRAD>(x, wg, wu, f, status, sm_count, stream);
  timing_end(kKernMx, stream);
  count_launches(1);
  return e;
}

}  // namespace

cudaError_t launch_mx_gated(const pvt_mx& x, const pvt_mx& wg, const pvt_mx& wu, int32_t activation, void* h, int32_t dtype, int64_t ldh,
                            const pvt_mx* hq, uint32_t* status, int sm_count, cudaStream_t stream) {
  Finish f = {};
  f.activation = activation, f.h = h, f.dtype = dtype, f.ldh = ldh;
  f.wide = reinterpret_cast<uintptr_t>(h) % 16 == 0 && ldh % 8 == 0;
  if (hq) f.q = held(*hq);
  return gated<false>(x, wg, wu, f, status, sm_count, stream);
}

cudaError_t launch_mx_gated_grad(const pvt_mx& x, const pvt_mx& wg, const pvt_mx& wu, int32_t activation, const void* dh, int32_t dtype,
                                 int64_t lddh, void* dgate, void* dup, int64_t ldd, uint32_t* status, int sm_count, cudaStream_t stream) {
  Finish f = {};
  f.activation = activation, f.dh = dh, f.dtype = dtype, f.ldh = lddh;
  f.wide = reinterpret_cast<uintptr_t>(dh) % 16 == 0 && lddh % 8 == 0;
  f.dgate = static_cast<__nv_bfloat16*>(dgate), f.dup = static_cast<__nv_bfloat16*>(dup), f.ldd = ldd;
  return gated<true>(x, wg, wu, f, status, sm_count, stream);
}

}  // namespace pvt
