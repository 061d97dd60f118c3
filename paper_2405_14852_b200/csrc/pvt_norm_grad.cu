// Gradients of the norm: by its rows and by its weights.
//
//   xh = (x - mean) rstd,  u = w dy,  dx = rstd (u - mean(u) - xh mean(u xh)) + dresidual   (without the mean: no mean(u))
//   dw = sum over rows of dy xh,  db = sum over rows of dy
//
// One reading of x and dy does both.  A thread keeps the sums for dw and db of its columns in registers, in binary32.  What the blocks
// have summed goes to the workspace, and a second kernel adds it up column by column in binary64, always in the order of blocks: which
// rows a block has depends on the shapes and the device only.  One barrier a row, for its two means: behind it row n - 1 is finished and
// row n's sums are taken, each in the other's waits (one after the other, two barriers a row: 57 to 66 us, so 56).
//
// What bounds it: 4096 x 8192 in bfloat16 with the residual's gradient, 268 MB, 56 us for both kernels, 75 % of a copy's rate, the issue slots
// 52 to 62 % taken.  333 x 5119 in float32: 14 us of 3.2, two kernels' latency, three rounds of 1400 cycles (257 instructions of a warp, one
// behind the other) and 6 MB of sums.  Rows asked for four rounds ahead instead of two changed nothing; two rows at least to each block: 592
// x 2445 14.2 -> 12.7 us, but 1184 x 1024 10.2 -> 11.3 and 2048 x 768 16.2 -> 18.4.
#include "pvt_norm.cuh"

namespace pvt {
namespace norm {
namespace {

constexpr uint32_t kSumThreads = 512, kAhead = 10;

struct GradParams {
  const void *x, *dy, *dres;
  void* dx;
  int64_t ldx, lddy, lddr, lddx;
  const void* weight;
  const float* stats;
  float* partial;  // [2][sets][pitch_of(cols)], or null
  Shape s;
  uint32_t x_image, g_image;  // bytes
  uint32_t sets;              // blocks or clusters: sets of sums
  uint32_t stages;            // three or four
  int32_t w_dtype;
  bool layer, w_wide, sums[2];  // of dw and db
};

// floats from one set of sums to the next: every set begins where a thread may store eight at once
__host__ __device__ inline uint32_t pitch_of(uint32_t cols) { return (cols + 7) / 8 * 8; }

// How many blocks or clusters share the rows: as many as are resident, but four rows at least to each where there are rows for all SMs,
// since each has a sum per column for the workspace.
uint32_t sets_of(const Shape& s, size_t bytes, int regs, int sm_count) {
  const uint32_t most = resident_sets(s, bytes, regs, sm_count), sms = (uint32_t)sm_count / s.parts;
  const uint32_t need = (uint32_t)(((uint64_t)s.rows + s.teams - 1) / s.teams);
  uint32_t n = need / 4 > sms ? need / 4 : sms;
  if (n > need) n = need;
  return n < most ? n : most;
}

// MEAN: the norm takes the mean off, or db is wanted
template <typename T, typename TG, int L, int G, bool MEAN>
__global__ void __launch_bounds__(L == kRagged && G == 1 ? kRaggedBound : kMostThreads) norm_grad_kernel(const __grid_constant__ GradParams p) {
  constexpr bool WIDE = L != kRagged;
  extern __shared__ __align__(128) unsigned char ring[];
  constexpr int N = MEAN ? 2 : 1;  // sums of a row
  __shared__ float slots[2][kMostParts * kMostWarps][N];
  __shared__ float sums[kTeamThreads / 32][kSpanCols];
  pdl_trigger();
  pdl_wait();
  const Shape& s = p.s;
  const uint32_t rank = blockIdx.x % s.parts, set = blockIdx.x / s.parts;
  const Place<L, G> at(s, rank);
  const float inv = 1.0f / (float)s.cols;
  const T* const x = static_cast<const T*>(p.x);
  const TG *const dy = static_cast<const TG*>(p.dy), *const dres = static_cast<const TG*>(p.dres);
  // a stage: the images of every team's x, dy and dres
  const uint32_t dy_at = s.teams * p.x_image + at.team * p.g_image, dres_at = dy_at + s.teams * p.g_image;
  const uint32_t stage = s.teams * (p.x_image + (dres ? 2 : 1) * p.g_image), base = m1::smem_u32(ring), x_at = at.team * p.x_image;
  const uint32_t stride = p.sets * s.teams;
  auto ask = [&](uint64_t row, uint32_t k) {
    if (row < s.rows) {
      const uint32_t to = base + k * stage;
      at.ask(to + x_at, x + (int64_t)row * p.ldx);
      at.ask(to + dy_at, dy + (int64_t)row * p.lddy);
      if (dres) at.ask(to + dres_at, dres + (int64_t)row * p.lddr);
    }
    copies_end();
  };
  // Round n takes the sums of row n and finishes row n - 1; what is asked for then goes where row n - 2 was.
  const uint64_t first = (uint64_t)set * s.teams;
  const uint32_t rounds = first < s.rows ? (uint32_t)((s.rows - first + stride - 1) / stride) : 0;
  uint64_t row = first + at.team;
  for (uint32_t k = 0; k + 2 < p.stages; ++k) ask(row + (uint64_t)k * stride, k);
  float w[G][8], dw[G][8], db[G][8], xh[G][8], u[G][8], sum[N] = {}, rstd = 0.0f;
  at.weights(p.weight, p.w_dtype, p.w_wide, 1.0f, w);
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[g][i] = db[g][i] = xh[g][i] = u[g][i] = 0.0f;
  auto stats_of = [&](uint64_t r) { return r < s.rows ? *reinterpret_cast<const float2*>(p.stats + 2 * r) : make_float2(0.0f, 0.0f); };
  float2 next = stats_of(row);
  uint32_t k = 0;  // stage of row n
  for (uint32_t n = 0; n <= rounds; ++n, row += stride) {
    copies_wait(p.stages > 3);
    // the sums of row n - 1 are here, what others have copied is, and row n - 2 has been read by all
    if (!WIDE || s.warps > 1 || s.parts > 1) row_barrier(s);
    ask(row + (uint64_t)(p.stages - 2) * stride, k >= 2 ? k - 2 : k + p.stages - 2);
    const unsigned char* const from = ring + k * stage;
    const unsigned char* const before = ring + (k == 0 ? p.stages - 1 : k - 1) * stage;
    k = k == p.stages - 1 ? 0 : k + 1;
    if (n > 0) {
      sums_get<N>(sum, s, slots[(n - 1) & 1]);
      const uint64_t last = row - stride;
      if (last < s.rows) {
        const float c1 = MEAN && p.layer ? sum[0] * inv * rstd : 0.0f, c2 = sum[N - 1] * inv * rstd;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float out[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) out[i] = fmaf(-c2, xh[g][i], fmaf(u[g][i], rstd, -c1));
          if (dres) {
            float d[8];
            at.take(before + dres_at, dres + (int64_t)last * p.lddr, g, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] += d[i];
          }
          at.put(static_cast<TG*>(p.dx) + (int64_t)last * p.lddx, g, out);
        }
      }
    }
    if (n == rounds) break;
    sum[0] = sum[N - 1] = 0.0f;
    const float mean = next.x;
    rstd = next.y;
    next = stats_of(row + stride);
    if (row < s.rows) {  // (otherwise the team's shared memory holds anything)
      const T* const x_row = x + (int64_t)row * p.ldx;
      const TG* const dy_row = dy + (int64_t)row * p.lddy;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        at.take(from + x_at, x_row, g, xh[g]);
        at.take(from + dy_at, dy_row, g, u[g]);
        if (!at.full(g)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) xh[g][i] = at.has(g, i) ? xh[g][i] : mean;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          xh[g][i] = (xh[g][i] - mean) * rstd;
          dw[g][i] = fmaf(u[g][i], xh[g][i], dw[g][i]);
          if (MEAN) db[g][i] += u[g][i];
          u[g][i] *= w[g][i];
        }
        if (MEAN) sum[0] += sum8(u[g]);
        sum[N - 1] += dot8(u[g], xh[g]);
      }
    }
    sums_put<N>(sum, s, rank, slots[n & 1]);
  }
  copies_wait(false);
  if (!p.partial) return;
  __syncwarp();
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (!p.sums[which] || (which && !MEAN)) continue;
    float* const to = p.partial + ((size_t)which * p.sets + set) * pitch_of(s.cols);
    if (s.teams == 1) {
#pragma unroll
      for (int g = 0; g < G; ++g) at.put(to, g, which ? db[g] : dw[g]);
    } else {  // the teams' sums first, always in the same order
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v = which ? db[0][i] : dw[0][i];
        if (s.lanes < 32) v += __shfl_xor_sync(0xffffffffu, v, 16);
        if (s.lanes < 16) v += __shfl_xor_sync(0xffffffffu, v, 8);
        if (at.lane < s.lanes && at.has(0, i)) sums[at.warp][at.c0 + i * at.step] = v;
      }
      __syncthreads();
      if (threadIdx.x < s.cols) {
        float v = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < kTeamThreads / 32; ++i) v += sums[i][threadIdx.x];
        to[threadIdx.x] = v;
      }
      __syncthreads();
    }
  }
}

// 32 columns of dw or db to a block: its warps have the sums of every sixteenth of the blocks ahead
__global__ void __launch_bounds__(kSumThreads) norm_grad_sum_kernel(const float* partial, uint32_t blocks, uint32_t cols, void* dweight,
                                                                    void* dbias, bool wide, bool accumulate) {
  __shared__ double sums[kSumThreads / 32][33];
  pdl_trigger();
  pdl_wait();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tiles = (cols + 31) / 32;
  const bool second = dweight == nullptr || blockIdx.x >= tiles;
  const uint32_t col = blockIdx.x % tiles * 32 + lane;
  void* const out = second ? dbias : dweight;
  double sum = 0.0;
  if (col < cols) {
    const uint32_t pitch = pitch_of(cols);
    const float* from = partial + (size_t)(second ? blocks : 0) * pitch + col;
    for (uint32_t b0 = warp; b0 < blocks; b0 += kAhead * (kSumThreads / 32)) {
      float v[kAhead];  // (all under way at once)
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) {
        const uint32_t b = b0 + k * (kSumThreads / 32);
        v[k] = b < blocks ? from[(size_t)b * pitch] : 0.0f;
      }
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) sum += (double)v[k];
    }
  }
  sums[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && col < cols) {
    sum = 0.0;
#pragma unroll
    for (uint32_t k = 0; k < kSumThreads / 32; ++k) sum += sums[k][lane];
    if (wide) {
      double* const to = static_cast<double*>(out) + col;
      *to = accumulate ? *to + sum : sum;
    } else {
      float* const to = static_cast<float*>(out) + col;
      *to = (float)(accumulate ? (double)*to + sum : sum);
    }
  }
}

size_t ring_bytes(const GradParams& p, uint32_t stages) {
  return (size_t)stages * p.s.teams * (p.x_image + (p.dres ? 2 : 1) * p.g_image);
}

// (the number of sets goes to the kernel that adds them up)
template <typename T, typename TG, int L, int G, bool MEAN>
cudaError_t start(GradParams& p, int sm_count, cudaStream_t stream) {
  const Shape& s = p.s;
  // two rows ahead where as many blocks have room for them as have registers
  p.stages = ring_bytes(p, 4) * (kMostThreads / s.threads) <= kRingBytes ? 4 : 3;
  const size_t bytes = ring_bytes(p, p.stages);
  int regs;
  const cudaError_t e = set_up<norm_grad_kernel<T, TG, L, G, MEAN>>(&regs);
  if (e != cudaSuccess) return e;
  p.sets = sets_of(s, bytes, regs, sm_count);
  if (s.parts == 1) return launch_dependent(norm_grad_kernel<T, TG, L, G, MEAN>, p.sets, s.threads, bytes, stream, p);
  return mma::launch_clusters(norm_grad_kernel<T, TG, L, G, MEAN>, p.sets * s.parts, s.parts, s.threads, bytes, stream, p);
}
template <typename T, typename TG, int L, int G>
cudaError_t start(GradParams& p, int sm_count, cudaStream_t stream) {
  return p.layer || p.sums[1] ? start<T, TG, L, G, true>(p, sm_count, stream) : start<T, TG, L, G, false>(p, sm_count, stream);
}
template <typename T, typename TG>
cudaError_t grad(GradParams& p, bool wide, uint32_t rows, uint32_t cols, int sm_count, cudaStream_t stream) {
  for (uint32_t parts = 1;; parts *= 2) {
    p.s = shape_of(rows, cols, wide, parts);
    p.x_image = image_bytes(p.s, sizeof(T), wide), p.g_image = image_bytes(p.s, sizeof(TG), wide);
    if (ring_bytes(p, 3) <= kRingBytes) break;
  }
  const bool one = p.s.groups == 1;
  switch (layout_of(p.s, wide)) {
    case kRagged: return one ? start<T, TG, kRagged, 1>(p, sm_count, stream) : start<T, TG, kRagged, 2>(p, sm_count, stream);
    case kWide: return one ? start<T, TG, kWide, 1>(p, sm_count, stream) : start<T, TG, kWide, 2>(p, sm_count, stream);
    default: return one ? start<T, TG, kExact, 1>(p, sm_count, stream) : start<T, TG, kExact, 2>(p, sm_count, stream);
  }
}

}  // namespace

// of the most sets that any types and alignment come to
size_t grad_workspace_bytes(int64_t rows, int32_t cols, int sm_count) {
  uint32_t most = 1;
  for (uint32_t parts = 1; parts <= kMostParts; parts *= 2)
    for (int narrow = 0; narrow < 2; ++narrow) {
      const uint32_t n = sets_of(shape_of((uint32_t)rows, (uint32_t)cols, narrow != 0, parts), 1, 64, sm_count);
      most = n > most ? n : most;
    }
  return align_up((size_t)2 * most * pitch_of((uint32_t)cols) * 4, 256);
}

cudaError_t launch_grad(const pvt_norm& n, const float* stats, int32_t dtype, const void* dy, int64_t lddy, const void* dres,
                        int64_t lddr, void* dx, int64_t lddx, void* dweight, void* dbias, int32_t dw_dtype, bool accumulate, void* ws,
                        int sm_count, cudaStream_t stream) {
  const bool sums = dweight || dbias;
  GradParams p = {};
  p.x = n.x, p.ldx = n.ldx, p.dy = dy, p.lddy = lddy, p.dres = dres, p.lddr = lddr, p.dx = dx, p.lddx = lddx;
  p.weight = n.weight, p.w_dtype = n.weight_dtype, p.stats = stats, p.layer = n.kind == PVT_NORM_LAYER;
  p.sums[0] = dweight, p.sums[1] = dbias;
  p.w_wide = rows_aligned(n.weight, 0, n.weight_dtype == PVT_F32 ? 4 : 2);
  p.partial = sums ? static_cast<float*>(ws) : nullptr;
  timing_begin(kKernNorm, stream);
  cudaError_t e = with_type(n.dtype, [&](auto* type) {
    using T = std::remove_pointer_t<decltype(type)>;
    return with_type(dtype, [&](auto* g_type) {
      using TG = std::remove_pointer_t<decltype(g_type)>;
      const bool wide = rows_aligned(n.x, n.ldx, sizeof(T)) && rows_aligned(dy, lddy, sizeof(TG)) &&
                        rows_aligned(dres, lddr, sizeof(TG)) && rows_aligned(dx, lddx, sizeof(TG));
      return grad<T, TG>(p, wide, (uint32_t)n.rows, (uint32_t)n.cols, sm_count, stream);
    });
  });
  if (e == cudaSuccess && sums) {
    const unsigned tiles = ((unsigned)n.cols + 31) / 32;
    e = launch_dependent(norm_grad_sum_kernel, tiles * (dweight && dbias ? 2 : 1), kSumThreads, 0, stream, (const float*)ws,
                         p.sets, (uint32_t)n.cols, dweight, dbias, dw_dtype == PVT_F64, accumulate);
  }
  timing_end(kKernNorm, stream);
  count_launches(sums ? 2 : 1);
  return e;
}

}  // namespace norm
}  // namespace pvt
