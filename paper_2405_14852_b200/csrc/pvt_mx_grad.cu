// Gradients of the product on 4-bit matrices: D[p, c] = sum over r of A(p, r) Q[r, c], Q held in 4 bits with its blocks along
// c, A the bfloat16 gradient of the product's result: as it lies in memory for dx (p a token, r an output), its
// transpose for dw (p an output, r a token).
//
// The blocks of Q run across the sum, so the block-scaled instructions do not apply.  Eight warps widen Q to
// bfloat16 on its way into shared memory (an element times its scale is exact there, with at most six significant
// bits) and tcgen05.mma multiplies 16-bit operands.  A step is 64 rows of Q by 256 columns, stored with the columns contiguous (128
// bytes = 64 columns to a row, under the 128-byte swizzle: eight threads that write 16 bytes each for eight rows meet no
// bank twice); A's tiles arrive by TMA, contiguous along r or along p as they lie.  One widened step serves two tiles
// of 128 rows of A where there are as many, so that the tensor cores and not the widening set the pace: 16384 elements
// at 2.75 instructions each are 350 cycles of the SM's issue slots, 16 products of 128 x 256 x 16 take 1050.
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
constexpr int kMaxStages = 4;
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
  alignas(8) uint64_t full_a[kMaxStages];
  uint64_t full_b[kMaxStages];
  uint64_t empty[kMaxStages];
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
// first fraction bit of a bfloat16, whose bias is 126 more, the sign goes to the top: one product with 2^126 gives the
// element, 0.5 (a number without its leading one) included, a second the value.
__device__ __forceinline__ uint4 widen8(uint32_t w, __nv_bfloat162 scale) {
  const uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
  const uint32_t big = 0x7e807e80u;  // 2^126 twice
  uint32_t out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // byte i of both, a zero byte above each (the selector's fourth bit repeats the byte's top bit, which is 0)
    uint32_t pair;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(pair) : "r"(even), "r"(odd), "r"(0xc480 + 0x1111 * i));
    const uint32_t bits = (pair * 0x1040u) & 0x81c081c0u;  // shifted by 6 and by 12
    const __nv_bfloat162 el = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&bits), *reinterpret_cast<const __nv_bfloat162*>(&big));
    const __nv_bfloat162 v = __hmul2(el, scale);
    out[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

template <int FMT>
__device__ __forceinline__ __nv_bfloat162 scale16(uint32_t byte) {
  if (FMT == PVT_MX_E4M3_16) return __float2bfloat162_rn(e4m3_value(byte));
  const uint32_t b = byte == 255 ? 0x7fc0u : byte ? byte << 7 : 0x0040u, two = b | b << 16;
  return *reinterpret_cast<const __nv_bfloat162*>(&two);
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

template <typename T, int FMT, bool TRANS, int MT>
__global__ void __launch_bounds__(kGThreads) mx_grad_kernel(const __grid_constant__ CUtensorMap a_map, const GradParams p) {
  constexpr uint32_t kStageBytes = MT * kABytes + kBBytes;
  constexpr uint32_t STAGES = MT == 2 ? 3 : 4;
  constexpr uint32_t TMEM = MT * kTileC;
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
    tmem_alloc(smem_u32(&sm.tmem), TMEM);
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
  const uint32_t a0 = tile / p.c_tiles * (MT * kTileA), c0 = tile % p.c_tiles * kTileC;
  const uint32_t first = (uint32_t)((uint64_t)p.steps * rank / p.split), last = (uint32_t)((uint64_t)p.steps * (rank + 1) / p.split);

  if (warp == kCopyWarp) {
    if (elect_one()) {
      uint32_t i = 0;
      for (uint32_t step = first; step < last; ++step, ++i) {
        const uint32_t s = i % STAGES, bar = smem_u32(&sm.full_a[s]), to = base + s * kStageBytes;
        if (i >= STAGES && !wait(smem_u32(&sm.empty[s]), (i / STAGES - 1) & 1, abandoned, p.status, p.max_spins)) break;
        if (i == p.withhold) continue;  // test hook: never issued
        mbar_expect_tx(bar, MT * kABytes);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          if (TRANS) {
            tma_load(to + m * kABytes, &a_map, (int)(a0 + m * kTileA), (int)(step * kStepR), bar);
            tma_load(to + m * kABytes + kABytes / 2, &a_map, (int)(a0 + m * kTileA + 64), (int)(step * kStepR), bar);
          } else {
            tma_load(to + m * kABytes, &a_map, (int)(step * kStepR), (int)(a0 + m * kTileA), bar);
          }
        }
      }
      if (*abandoned)  // what was issued lands before the block's memory is another's
        for (uint32_t j = i > STAGES ? i - STAGES : 0; j < i; ++j)
          if (j != p.withhold) drain(smem_u32(&sm.full_a[j % STAGES]), (j / STAGES) & 1);
    }
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
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (uint32_t k = 0; k < kStepR / 16; ++k) {
        const uint64_t b = operand(from + MT * kABytes + k * 2048, kBBytes / 4, 1024, true);
#pragma unroll
        for (uint32_t m = 0; m < (uint32_t)MT; ++m) {
          const uint64_t a = TRANS ? operand(from + m * kABytes + k * 2048, kABytes / 2, 1024, true)
                                   : operand(from + m * kABytes + k * 32, 16, 1024, true);
          multiply16(tmem + m * kTileC, a, b, idesc, (uint32_t)(i > 0 || k > 0));
        }
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
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      unsigned char* const to = mem + s * kStageBytes + MT * kABytes + chunk / 2 * (kBBytes / 4) + row * 128;
#pragma unroll
      for (int it = 0; it < 2; ++it) {
        const uint32_t w[4] = {now.codes[it].x, now.codes[it].y, now.codes[it].z, now.codes[it].w};
        const __nv_bfloat162 s0 = scale16<FMT>(FMT == PVT_MX_E8M0_32 ? now.scales[it] : now.scales[it] & 255u);
        const __nv_bfloat162 s1 = FMT == PVT_MX_E8M0_32 ? s0 : scale16<FMT>(now.scales[it] >> 8);
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
          *reinterpret_cast<uint4*>(to + it * (32 * 128) + ((((chunk & 1) * 4 + q) ^ in_row) << 4)) = widen8(w[q], q < 2 ? s0 : s1);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // generic-proxy writes -> visible to the products
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.full_b[s]));
      now = next;
    }
    ok = wait(smem_u32(&sm.done), 0, abandoned, p.status, p.max_spins);
    ok = __all_sync(0xffffffffu, ok);
    tc_fence_after();
    if (ok) {
      const float alpha = p.ts ? *p.ts : 1.0f;
      const uint32_t quarter = warp % 4, half = warp / 4;
      if (p.split == 1) {
        // 32 rows by 32 columns at a time, turned in shared memory so that a warp stores along a row; the upper four warps
        // have the second tile of rows, or the second half of the columns
        float* const turn = reinterpret_cast<float*>(mem) + warp * (32 * 33);
        const uint32_t m = MT == 2 ? half : 0, row0 = a0 + m * kTileA + quarter * 32;
        const uint32_t j_lo = MT == 2 ? 0 : half * (kTileC / 2), j_hi = MT == 2 ? kTileC : j_lo + kTileC / 2;
        const uint32_t n_rows = row0 < p.a_rows ? min(32u, p.a_rows - row0) : 0;
        for (uint32_t j0 = j_lo; j0 < j_hi && c0 + j0 < p.cols && n_rows; j0 += 32) {
          uint32_t v[32];
          tmem_ld32(tmem + (quarter << 21) + m * kTileC + j0, v);
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
      const float alpha = p.ts ? *p.ts : 1.0f;
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
    tmem_dealloc(tmem, TMEM);
  }
}

template <typename T, int FMT, bool TRANS, int MT>
cudaError_t start(const CUtensorMap& a_map, GradParams& p, uint64_t tiles, cudaStream_t stream) {
  constexpr size_t stages = MT == 2 ? 3 : 4, smem = stages * (MT * kABytes + kBBytes) + 1024;
  static_assert(smem + sizeof(GradShared) + 1024 <= 227 * 1024, "a block's shared memory");
  static_assert(MT == 2 || kTileA * kPartPitch * 4 <= stages * (MT * kABytes + kBBytes), "the partial sums fit the stages");
  if (tiles * p.split > 0x7fffffffull) return cudaErrorInvalidConfiguration;
  const cudaError_t e = allow_smem<mx_grad_kernel<T, FMT, TRANS, MT>>();
  if (e != cudaSuccess) return e;
  return launch_clusters(mx_grad_kernel<T, FMT, TRANS, MT>, (unsigned)(tiles * p.split), p.split, kGThreads, smem, stream, a_map, p);
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
  const uint64_t two = (uint64_t)((a_rows + 2 * kTileA - 1) / (2 * kTileA)) * p.c_tiles;
  p.split = 1;
  if (two >= (uint64_t)sm_count) return start<T, FMT, TRANS, 2>(a_map, p, two, stream);
  const uint64_t one = (uint64_t)((a_rows + kTileA - 1) / kTileA) * p.c_tiles;
  while (p.split < 8 && one * p.split * 2 <= (uint64_t)sm_count && p.split * 2 <= p.steps) p.split *= 2;
  return start<T, FMT, TRANS, 1>(a_map, p, one, stream);
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
