// Norm of the rows of x + residual, into floats or straight into 4-bit block floating point.
//
// A row stays in registers from its one reading to its one writing: the sum with the residual is rounded to x's type first, as
// it is kept; then the mean, then the mean of the squared differences from it (a second pass over registers, so a mean far from
// 0 costs no digits).  Bound by HBM; the weights come from the L1 and L2 again for each row.
//
// 4-bit results: a lane's eight columns are a quarter or half of a block, as in quantisation by itself; rows of no alignment are
// turned in shared memory first.
#include "pvt_mx_block.cuh"
#include "pvt_norm.cuh"

namespace pvt {
namespace norm {
namespace {

using mx::kStrip;

constexpr uint32_t kTeamThreads = 256;  // of a block where rows share it

struct ApplyParams {
  const void *x, *residual;
  void* total;
  int64_t ldx, ldr, ldt, ldy;
  const void *weight, *bias;
  void* y;
  float* stats;
  mx::Held q;
  Shape s;
  uint32_t padded;  // rows, or those of whole strips where scales are written
  int32_t w_dtype, y_dtype;
  float eps;
  bool layer, w_wide;
};

// over all warps of a row; `slots`: shared, one per warp, not in use by an earlier sum
__device__ __forceinline__ float row_sum(float v, const Shape& s, float* slots) {
  v = team_sum(v, s.lanes);
  if (s.warps == 1) return v;
  const uint32_t lane = threadIdx.x & 31;
  if (lane == 0) slots[threadIdx.x >> 5] = v;
  __syncthreads();
  return team_sum(lane < s.warps ? slots[lane] : 0.0f, 32);
}

// G: spans to a warp
template <typename T, bool WIDE, int G>
__global__ void __launch_bounds__(G == 1 ? 1024 : 512) norm_apply_kernel(const __grid_constant__ ApplyParams p) {
  __shared__ float slots[2][2][32];
  __shared__ float buffer[WIDE ? 1 : (G == 1 ? 32 : 16)][mx::kSpan + 8 * mx::kSpan / 32];
  pdl_trigger();
  pdl_wait();
  const Shape& s = p.s;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t in_row = s.warps > 1 ? warp : 0, l = lane & (s.lanes - 1), step = WIDE ? 1 : s.lanes;
  const uint32_t team = s.warps > 1 ? 0 : tid / s.lanes;
  const mx::TensorScale scale(p.q.tensor_scale);
  uint32_t turn = 0;
  for (uint64_t first = (uint64_t)blockIdx.x * s.teams; first < p.padded; first += (uint64_t)gridDim.x * s.teams, turn ^= 1) {
    const uint32_t row = (uint32_t)first + team;
    const bool here = row < s.rows;
    float v[G][8];
    const T* const x = static_cast<const T*>(p.x) + (int64_t)row * p.ldx;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint32_t c = (g * s.warps + in_row) * kSpanCols + (WIDE ? 8 * l : l);
      T e[8];
      take<WIDE>(x, c, step, here ? s.cols : 0, e);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[g][i] = widen<T>(e[i]);
      if (p.residual) {
        take<WIDE>(static_cast<const T*>(p.residual) + (int64_t)row * p.ldr, c, step, here ? s.cols : 0, e);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[g][i] = widen<T>(narrow<T>(v[g][i] + widen<T>(e[i])));
      }
      if (p.total) put<WIDE>(static_cast<T*>(p.total) + (int64_t)row * p.ldt, c, step, here ? s.cols : 0, v[g]);
    }
    float mean = 0.0f, sum = 0.0f;
    if (p.layer) {
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[g][i];
      mean = row_sum(sum, s, slots[turn][0]) / (float)s.cols;
      sum = 0.0f;
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint32_t c = (g * s.warps + in_row) * kSpanCols + (WIDE ? 8 * l : l);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[g][i] = c + i * step < s.cols ? v[g][i] - mean : 0.0f;
        sum = fmaf(v[g][i], v[g][i], sum);
      }
    }
    const float rstd = 1.0f / sqrtf(row_sum(sum, s, slots[turn][1]) / (float)s.cols + p.eps);
    if (p.stats && here && in_row == 0 && l == 0) *reinterpret_cast<float2*>(p.stats + 2 * (size_t)row) = make_float2(mean, rstd);
    if (!p.y && !p.q.codes) continue;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint32_t span = g * s.warps + in_row, c = span * kSpanCols + (WIDE ? 8 * l : l);
      if (span >= s.spans) break;
      float w[8], b[8];
      take_weights<WIDE>(p.weight, p.w_dtype, p.w_wide, c, step, s.cols, 1.0f, w);
      take_weights<WIDE>(p.bias, p.w_dtype, p.w_wide, c, step, s.cols, 0.0f, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[g][i] = fmaf(v[g][i] * rstd, w[i], b[i]);
      if (p.y)
        with_type(p.y_dtype, [&](auto* type) {
          using U = std::remove_pointer_t<decltype(type)>;
          put<WIDE>(static_cast<U*>(p.y) + (int64_t)row * p.ldy, c, step, here ? s.cols : 0, v[g]);
        });
      if (p.q.codes) {  // (a row is a warp's at least)
        if (!WIDE) mx::turn<false>(buffer[warp], v[g], lane);
        const uint32_t c0 = span * kSpanCols + 8 * lane;
        if (p.q.format == PVT_MX_E8M0_32)
          mx::put_eight<PVT_MX_E8M0_32>(p.q, row, c0, here, row < p.padded, scale, v[g]);
        else
          mx::put_eight<PVT_MX_E4M3_16>(p.q, row, c0, here, row < p.padded, scale, v[g]);
      }
    }
  }
}

template <typename T, bool WIDE, int G>
cudaError_t apply(ApplyParams p, uint32_t rows, uint32_t cols, int sm_count, cudaStream_t stream) {
  p.s = shape_of(rows, cols, G, kTeamThreads, !p.q.codes);
  const uint32_t threads = p.s.warps > 1 ? 32 * p.s.warps : kTeamThreads;
  const uint64_t need = ((uint64_t)p.padded + p.s.teams - 1) / p.s.teams, most = (uint64_t)sm_count * 64;
  return launch_dependent(norm_apply_kernel<T, WIDE, G>, (unsigned)(need < most ? need : most), threads, 0, stream, p);
}

template <typename T, bool WIDE>
cudaError_t apply(const ApplyParams& p, uint32_t rows, uint32_t cols, int sm_count, cudaStream_t stream) {
  const uint32_t spans = (cols + kSpanCols - 1) / kSpanCols;
  // few rows: as many warps to each as there are spans
  if (spans == 1 || (spans <= 32 && rows <= (uint32_t)sm_count)) return apply<T, WIDE, 1>(p, rows, cols, sm_count, stream);
  if (spans <= 16) return apply<T, WIDE, 2>(p, rows, cols, sm_count, stream);
  if (spans <= 64) return apply<T, WIDE, 4>(p, rows, cols, sm_count, stream);
  return apply<T, WIDE, 8>(p, rows, cols, sm_count, stream);
}

}  // namespace

cudaError_t launch_apply(const pvt_norm& n, void* total, int64_t ldt, void* y, int32_t y_dtype, int64_t ldy, const pvt_mx* yq,
                         float* stats, int sm_count, cudaStream_t stream) {
  ApplyParams p = {};
  p.x = n.x, p.ldx = n.ldx, p.residual = n.residual, p.ldr = n.ldr, p.total = total, p.ldt = ldt;
  p.weight = n.weight, p.bias = n.bias, p.w_dtype = n.weight_dtype;
  p.y = y, p.ldy = ldy, p.y_dtype = y_dtype, p.stats = stats, p.eps = n.eps, p.layer = n.kind == PVT_NORM_LAYER;
  p.padded = (uint32_t)n.rows;
  if (yq) {
    p.q = mx::held(*yq);
    p.padded = (uint32_t)((n.rows + kStrip - 1) / kStrip * kStrip);
  }
  const size_t w_size = n.weight_dtype == PVT_F32 ? 4 : 2, y_size = y_dtype == PVT_F32 ? 4 : 2;
  p.w_wide = rows_aligned(n.weight, 0, w_size) && rows_aligned(n.bias, 0, w_size);
  timing_begin(kKernNorm, stream);
  const cudaError_t e = with_type(n.dtype, [&](auto* type) {
    using T = std::remove_pointer_t<decltype(type)>;
    const bool wide = rows_aligned(n.x, n.ldx, sizeof(T)) && rows_aligned(n.residual, n.ldr, sizeof(T)) &&
                      rows_aligned(total, ldt, sizeof(T)) && rows_aligned(y, ldy, y_size);
    return wide ? apply<T, true>(p, (uint32_t)n.rows, (uint32_t)n.cols, sm_count, stream)
                : apply<T, false>(p, (uint32_t)n.rows, (uint32_t)n.cols, sm_count, stream);
  });
  timing_end(kKernNorm, stream);
  count_launches(1);
  return e;
}

}  // namespace norm
}  // namespace pvt
