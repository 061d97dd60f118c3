// Gradients of the norm: by its rows and by its weights.
//
//   xh = (x - mean) rstd,  u = w dy,  dx = rstd (u - mean(u) - xh mean(u xh)) + dresidual   (without the mean: no mean(u))
//   dw = sum over rows of dy xh,  db = sum over rows of dy
//
// One reading of x and dy does both.  Blocks stay and take row after row; a thread has the same columns in each and keeps their
// sums for dw and db in registers, in binary32.  The next row's elements are asked for before this one's two means, which cost a
// barrier.  What the blocks have summed goes to the workspace, and a second kernel adds it up column by column in binary64, always in
// the order of blocks: which rows a block has depends on the shapes and the device only.  Rows of more than 8192 columns are shared
// by a cluster of two or four blocks, whose parts of the means meet in shared memory.
#include "pvt_mma.cuh"
#include "pvt_norm.cuh"

namespace pvt {
namespace norm {
namespace {

constexpr uint32_t kTeamThreads = 256;  // of a block where rows share it
constexpr uint32_t kMostWarps = 16, kMostParts = 4;
constexpr uint32_t kSumThreads = 512;

struct GradParams {
  const void *x, *dy, *dres;
  void* dx;
  int64_t ldx, lddy, lddr, lddx;
  const void* weight;
  const float* stats;
  float* partial;  // [2][blocks][cols], or null
  Shape s;
  uint32_t parts;  // blocks of a row
  uint32_t blocks;  // sets of sums
  int32_t w_dtype;
  bool layer, w_wide;
};

// how the rows are spread
struct Plan {
  uint32_t groups, parts, blocks;
  Shape s;
};
Plan plan_of(uint32_t rows, uint32_t cols, int sm_count) {
  Plan t = {};
  const uint32_t spans = (cols + kSpanCols - 1) / kSpanCols;
  t.groups = spans <= 8 ? 1 : 2;
  t.parts = 1;
  while (spans > t.parts * t.groups * kMostWarps) t.parts *= 2;
  t.s = shape_of(rows, cols, t.groups * t.parts, kTeamThreads, true);
  // as many blocks as are resident, but four rows at least to each where there are rows for all SMs
  const uint32_t warps = t.s.warps > 1 ? t.s.warps : kTeamThreads / 32;
  const uint32_t per_sm = (t.groups == 1 ? 24 : 16) / warps;
  const uint32_t most = (uint32_t)sm_count * (per_sm > 1 ? per_sm : 1) / t.parts, sms = (uint32_t)sm_count / t.parts;
  const uint32_t need = (uint32_t)(((uint64_t)rows + t.s.teams - 1) / t.s.teams);
  t.blocks = need / 4 > sms ? need / 4 : sms;
  if (t.blocks > need) t.blocks = need;
  if (t.blocks > most) t.blocks = most;
  return t;
}

template <typename T, typename TG, bool WIDE, int G>
__global__ void __launch_bounds__(G == 1 ? 256 : 512, G == 1 ? 3 : 1) norm_grad_kernel(const __grid_constant__ GradParams p) {
  __shared__ float2 slots[2][kMostParts * kMostWarps];
  __shared__ float sums[G == 1 ? kTeamThreads / 32 : 1][kSpanCols];
  pdl_trigger();
  pdl_wait();
  const Shape& s = p.s;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t in_row = s.warps > 1 ? warp : 0, l = lane & (s.lanes - 1), step = WIDE ? 1 : s.lanes;
  const uint32_t team = s.warps > 1 ? 0 : tid / s.lanes;
  const uint32_t rank = blockIdx.x % p.parts, set = blockIdx.x / p.parts;
  const float inv = 1.0f / (float)s.cols;
  uint32_t c[G];
  float w[G][8], dw[G][8], db[G][8];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    c[g] = (rank * s.warps * G + g * s.warps + in_row) * kSpanCols + (WIDE ? 8 * l : l);
    take_weights<WIDE>(p.weight, p.w_dtype, p.w_wide, c[g], step, s.cols, 1.0f, w[g]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[g][i] = db[g][i] = 0.0f;
  }
  T x[G][8];
  TG dy[G][8];
  float2 stats = make_float2(0.0f, 0.0f);
  auto fetch = [&](uint64_t row) {
    const bool here = row < s.rows;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      take<WIDE>(static_cast<const T*>(p.x) + (int64_t)row * p.ldx, c[g], step, here ? s.cols : 0, x[g]);
      take<WIDE>(static_cast<const TG*>(p.dy) + (int64_t)row * p.lddy, c[g], step, here ? s.cols : 0, dy[g]);
    }
    stats = here ? *reinterpret_cast<const float2*>(p.stats + 2 * row) : make_float2(0.0f, 0.0f);
  };
  uint32_t turn = 0;
  uint64_t row = (uint64_t)set * s.teams + team;
  const uint64_t stride = (uint64_t)p.blocks * s.teams;
  fetch(row);
  for (uint64_t first = (uint64_t)set * s.teams; first < s.rows; first += stride, row += stride, turn ^= 1) {
    const bool here = row < s.rows;
    const uint32_t cols = here ? s.cols : 0;
    const float mean = stats.x, rstd = stats.y;
    float xh[G][8], u[G][8];
    float2 sum = make_float2(0.0f, 0.0f);
    TG res[G][8];
#pragma unroll
    for (int g = 0; g < G; ++g) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xh[g][i] = c[g] + i * step < cols ? (widen<T>(x[g][i]) - mean) * rstd : 0.0f;
        const float d = widen<TG>(dy[g][i]);
        dw[g][i] = fmaf(d, xh[g][i], dw[g][i]);
        db[g][i] += d;
        u[g][i] = d * w[g][i];
        sum.x += u[g][i];
        sum.y = fmaf(u[g][i], xh[g][i], sum.y);
      }
      if (p.dres) take<WIDE>(static_cast<const TG*>(p.dres) + (int64_t)row * p.lddr, c[g], step, cols, res[g]);
    }
    fetch(row + stride);
    if (p.layer) sum.x = team_sum(sum.x, s.lanes);
    sum.y = team_sum(sum.y, s.lanes);
    if (s.warps > 1) {
      if (p.parts == 1) {
        if (lane == 0) slots[turn][warp] = sum;
        __syncthreads();
      } else {
        if (lane < p.parts) {
          const uint32_t at = mma::cluster_address(m1::smem_u32(&slots[turn][rank * s.warps + warp]), lane);
          asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(sum.x), "f"(sum.y) : "memory");
        }
        mma::cluster_sync();
      }
      sum = make_float2(0.0f, 0.0f);
      for (uint32_t i = lane; i < p.parts * s.warps; i += 32) sum.x += slots[turn][i].x, sum.y += slots[turn][i].y;
      sum.x = team_sum(sum.x, 32), sum.y = team_sum(sum.y, 32);
    }
    const float c1 = p.layer ? sum.x * inv : 0.0f, c2 = sum.y * inv;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float out[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i] = (u[g][i] - c1 - xh[g][i] * c2) * rstd;
      if (p.dres) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] += widen<TG>(res[g][i]);
      }
      put<WIDE>(static_cast<TG*>(p.dx) + (int64_t)row * p.lddx, c[g], step, cols, out);
    }
  }
  if (!p.partial) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* const to = p.partial + ((size_t)which * p.blocks + set) * s.cols;
    if (G > 1 || s.warps > 1) {
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c[g] + i * step < s.cols) to[c[g] + i * step] = which ? db[g][i] : dw[g][i];
    } else {  // the teams' sums first, always in the same order
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v = which ? db[0][i] : dw[0][i];
        if (s.lanes < 32) v += __shfl_xor_sync(0xffffffffu, v, 16);
        if (s.lanes < 16) v += __shfl_xor_sync(0xffffffffu, v, 8);
        if (lane < s.lanes && c[0] + i * step < kSpanCols) sums[G == 1 ? warp : 0][c[0] + i * step] = v;
      }
      __syncthreads();
      if (tid < s.cols) {
        float v = 0.0f;
#pragma unroll
        for (uint32_t k = 0; k < (G == 1 ? kTeamThreads / 32 : 1); ++k) v += sums[k][tid];
        to[tid] = v;
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
    const float* from = partial + (size_t)(second ? blocks : 0) * cols + col;
#pragma unroll 8
    for (uint32_t b = warp; b < blocks; b += kSumThreads / 32) sum += (double)from[(size_t)b * cols];
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

template <typename T, typename TG, bool WIDE, int G>
cudaError_t grad(const GradParams& p, cudaStream_t stream) {
  const uint32_t threads = p.s.warps > 1 ? 32 * p.s.warps : kTeamThreads;
  if (p.parts == 1) return launch_dependent(norm_grad_kernel<T, TG, WIDE, G>, p.blocks, threads, 0, stream, p);
  return mma::launch_clusters(norm_grad_kernel<T, TG, WIDE, G>, p.blocks * p.parts, p.parts, threads, 0, stream, p);
}

}  // namespace

size_t grad_workspace_bytes(int64_t rows, int32_t cols, int sm_count) {
  return align_up((size_t)2 * plan_of((uint32_t)rows, (uint32_t)cols, sm_count).blocks * (size_t)cols * 4, 256);
}

cudaError_t launch_grad(const pvt_norm& n, const float* stats, int32_t dtype, const void* dy, int64_t lddy, const void* dres,
                        int64_t lddr, void* dx, int64_t lddx, void* dweight, void* dbias, int32_t dw_dtype, bool accumulate, void* ws,
                        int sm_count, cudaStream_t stream) {
  const Plan plan = plan_of((uint32_t)n.rows, (uint32_t)n.cols, sm_count);
  const bool sums = dweight || dbias;
  GradParams p = {};
  p.x = n.x, p.ldx = n.ldx, p.dy = dy, p.lddy = lddy, p.dres = dres, p.lddr = lddr, p.dx = dx, p.lddx = lddx;
  p.weight = n.weight, p.w_dtype = n.weight_dtype, p.stats = stats, p.layer = n.kind == PVT_NORM_LAYER;
  p.w_wide = rows_aligned(n.weight, 0, n.weight_dtype == PVT_F32 ? 4 : 2);
  p.partial = sums ? static_cast<float*>(ws) : nullptr;
  p.s = plan.s, p.parts = plan.parts, p.blocks = plan.blocks;
  timing_begin(kKernNorm, stream);
  cudaError_t e = with_type(n.dtype, [&](auto* type) {
    using T = std::remove_pointer_t<decltype(type)>;
    return with_type(dtype, [&](auto* g_type) {
      using TG = std::remove_pointer_t<decltype(g_type)>;
      const bool wide = rows_aligned(n.x, n.ldx, sizeof(T)) && rows_aligned(dy, lddy, sizeof(TG)) &&
                        rows_aligned(dres, lddr, sizeof(TG)) && rows_aligned(dx, lddx, sizeof(TG));
      if (wide) return plan.groups == 1 ? grad<T, TG, true, 1>(p, stream) : grad<T, TG, true, 2>(p, stream);
      return plan.groups == 1 ? grad<T, TG, false, 1>(p, stream) : grad<T, TG, false, 2>(p, stream);
    });
  });
  if (e == cudaSuccess && sums) {
    const unsigned tiles = ((unsigned)n.cols + 31) / 32;
    e = launch_dependent(norm_grad_sum_kernel, tiles * (dweight && dbias ? 2 : 1), kSumThreads, 0, stream, (const float*)ws,
                         p.blocks, (uint32_t)n.cols, dweight, dbias, dw_dtype == PVT_F64, accumulate);
  }
  timing_end(kKernNorm, stream);
  count_launches(sums ? 2 : 1);
  return e;
}

}  // namespace norm
}  // namespace pvt
