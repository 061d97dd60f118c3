// Norm of the rows of x + residual, into floats or straight into 4-bit block floating point.
//
// A row is read once and stays in registers to its end: the sum with the residual is rounded to x's type first, as it is
// kept; then the mean, then the mean of the squared differences from it (a second pass over registers, so a mean far from 0 costs no
// digits).  Two barriers a row, one without the mean; where rows are many, a team
// has two at a time and both share them.  (Two elements to an instruction, here and in quantisation: 4096 x 4096 into 4 bits 33 -> 30 us.)
//
// 4-bit results: a lane's eight columns are a quarter or half of a block, as in quantisation by itself; rows of no alignment are
// turned in shared memory first.
//
// What bounds it: 4096 x 8192 in bfloat16 with the residual, 268 MB, 47 us, 88 % of a copy's rate, the issue slots 55 % taken (the
// second barrier of a row costs less than what would save it: means of each warp, 55 us).  Into 4 bits the latency of a row's
// chain with four warps to a scheduler, 53 % of the slots taken and the bytes a fifth: 2048 x 4096 18 us under e8m0 and 20 under e4m3 for 14 into
// bfloat16.  2047 x 5001 in float16, rows of no alignment, 20 us of 9.5, the same (five warps, 51 %, elements taken and stored one
// by one).  One row of 4096 2.5 us behind the kernel ahead.
#include "pvt_mx_block.cuh"
#include "pvt_norm.cuh"

namespace pvt {
namespace norm {
namespace {

using mx::kStrip;

constexpr uint32_t kTurn = mx::kSpan + 8 * mx::kSpan / 32;  // floats of a warp

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
  uint32_t image;   // bytes
  uint32_t sets;    // blocks or clusters
  uint32_t stages;  // two or three
  int32_t w_dtype, y_dtype;
  float eps;
  bool layer, w_wide;
};

// G: spans of a warp, R: rows of a team at a time
template <typename T, int L, int G, int R>
__global__ void __launch_bounds__(L == kRagged ? kRaggedBound : kMostThreads) norm_apply_kernel(const __grid_constant__ ApplyParams p) {
  constexpr bool WIDE = L != kRagged;
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ float slots[2][2][kMostParts * kMostWarps][R];
  pdl_trigger();
  pdl_wait();
  const Shape& s = p.s;
  const uint32_t rank = blockIdx.x % s.parts, set = blockIdx.x / s.parts;
  const Place<L, G> at(s, rank);
  const mx::TensorScale scale(p.q.tensor_scale);
  const T* const x = static_cast<const T*>(p.x);
  const T* const residual = static_cast<const T*>(p.residual);
  // a stage: x's images of R rows of every team, then the residual's
  const uint32_t row_at = s.teams * p.image, res_at = R * row_at, stage = (residual ? 2 : 1) * res_at, own = at.team * p.image;
  const uint32_t base = m1::smem_u32(ring) + own, stride = p.sets * s.teams * R;
  auto ask = [&](uint64_t row0, uint32_t k) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint64_t row = row0 + r * s.teams;
      if (row < s.rows) {
        at.ask(base + k * stage + r * row_at, x + (int64_t)row * p.ldx);
        if (residual) at.ask(base + k * stage + res_at + r * row_at, residual + (int64_t)row * p.ldr);
      }
    }
    copies_end();
  };
  uint64_t row0 = (uint64_t)set * s.teams * R + at.team;
  for (uint32_t k = 0; k + 1 < p.stages; ++k) ask(row0 + (uint64_t)k * stride, k);
  float w[G][8], b[G][8];
  at.weights(p.weight, p.w_dtype, p.w_wide, 1.0f, w);
  at.weights(p.bias, p.w_dtype, p.w_wide, 0.0f, b);
  const float inv = 1.0f / (float)s.cols;
  if (s.parts > 1) mma::cluster_sync();  // every block of the cluster runs: from here on others write to its shared memory
  uint32_t turn = 0, k = 0;
  // (all of a block's teams go round as often as its first one)
  for (uint64_t first = (uint64_t)set * s.teams * R; first < p.padded; first += stride, row0 += stride, turn ^= 1) {
    copies_wait(p.stages > 2);
    if (!WIDE) {  // what others have copied is here, and the stage that is asked for next has been read by all
      if (s.warps > 1)
        __syncthreads();
      else
        __syncwarp();
    }
    ask(row0 + (uint64_t)(p.stages - 1) * stride, k == 0 ? p.stages - 1 : k - 1);
    const unsigned char* const image = ring + own + k * stage;
    k = k == p.stages - 1 ? 0 : k + 1;
    float v[R][G][8], sum[R], mean[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint64_t row = row0 + r * s.teams;
      mean[r] = 0.0f;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        at.take(image + r * row_at, x + (int64_t)row * p.ldx, g, v[r][g]);
        if (residual) {
          float e[8];
          at.take(image + res_at + r * row_at, residual + (int64_t)row * p.ldr, g, e);
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            T kept[2];
            const float2 sum = add2(two(v[r][g] + i), two(e + i));
            narrow_pair(sum.x, sum.y, kept);
            v[r][g][i] = widen<T>(kept[0]), v[r][g][i + 1] = widen<T>(kept[1]);
          }
        }
        if (p.total && row < s.rows) at.put(static_cast<T*>(p.total) + (int64_t)row * p.ldt, g, v[r][g]);
        if (p.layer) mean[r] += sum8(v[r][g]);
      }
    }
    if (p.layer) {
      row_sums<R>(mean, s, rank, slots[turn][0]);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        mean[r] *= inv;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          if (at.full(g)) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) set2(v[r][g] + i, add2(two(v[r][g] + i), both(-mean[r])));
          } else {
            at.each(g, [&](int i) { v[r][g][i] -= mean[r]; });
          }
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      sum[r] = 0.0f;
#pragma unroll
      for (int g = 0; g < G; ++g) sum[r] += dot8(v[r][g], v[r][g]);
    }
    row_sums<R>(sum, s, rank, slots[turn][1]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint64_t row = row0 + r * s.teams;
      const bool here = row < s.rows;
      const float rstd = inverse_root(fmaf(sum[r], inv, p.eps));
      if (p.stats && here && rank == 0 && at.in_team == 0)
        *reinterpret_cast<float2*>(p.stats + 2 * row) = make_float2(p.layer ? mean[r] : 0.0f, rstd);
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < 8; i += 2) set2(v[r][g] + i, fma2(mul2(two(v[r][g] + i), both(rstd)), two(w[g] + i), two(b[g] + i)));
      if (p.y && here)
        with_type(p.y_dtype, [&](auto* type) {
          using U = std::remove_pointer_t<decltype(type)>;
#pragma unroll
          for (int g = 0; g < G; ++g) at.put(static_cast<U*>(p.y) + (int64_t)row * p.ldy, g, v[r][g]);
        });
      if (p.q.codes) {  // (a row is a warp's at least)
#pragma unroll
        for (int g = 0; g < G; ++g) {
          if (!WIDE) mx::turn<false>(reinterpret_cast<float*>(ring + p.stages * stage) + at.warp * kTurn, v[r][g], at.lane);
          const uint32_t c0 = at.part0 + (s.teams > 1 ? 0 : at.warp * kSpanCols) + g * at.next + 8 * at.lane;
          if (p.q.format == PVT_MX_E8M0_32)
            mx::put_eight<PVT_MX_E8M0_32>(p.q, (uint32_t)row, c0, here, row < p.padded, scale, v[r][g]);
          else
            mx::put_eight<PVT_MX_E4M3_16>(p.q, (uint32_t)row, c0, here, row < p.padded, scale, v[r][g]);
        }
      }
    }
  }
  copies_wait(false);
}

// shared memory of a block
size_t ring_bytes(const ApplyParams& p, uint32_t rows, uint32_t stages, bool turned) {
  return (size_t)stages * (p.residual ? 2 : 1) * rows * p.s.teams * p.image + (turned ? p.s.threads / 32 * kTurn * 4 : 0);
}

template <typename T, int L, int G, int R>
cudaError_t start(ApplyParams p, uint32_t stages, int sm_count, cudaStream_t stream) {
  const Shape& s = p.s;
  const size_t bytes = ring_bytes(p, R, stages, L == kRagged && p.q.codes);
  int regs;
  const cudaError_t e = set_up<norm_apply_kernel<T, L, G, R>>(&regs);
  if (e != cudaSuccess) return e;
  const uint64_t rows_each = (uint64_t)s.teams * R, need = (p.padded + rows_each - 1) / rows_each;
  const uint64_t most = resident_sets(s, bytes, regs, sm_count);
  p.sets = (uint32_t)(need < most ? need : most), p.stages = stages;
  if (s.parts == 1) return launch_dependent(norm_apply_kernel<T, L, G, R>, p.sets, s.threads, bytes, stream, p);
  return mma::launch_clusters(norm_apply_kernel<T, L, G, R>, p.sets * s.parts, s.parts, s.threads, bytes, stream, p);
}

template <typename T, int L, int G>
cudaError_t start(const ApplyParams& p, int sm_count, cudaStream_t stream) {
  const bool turned = L == kRagged && p.q.codes;
  const uint32_t blocks = kMostThreads / p.s.threads;  // of an SM
  // two rows at a time if all blocks have some, and rings of three stages, or of two; not floats without the mean, which share one barrier
  // only, beyond four rows to a block (4096 x 8192 in bfloat16 48 and 44 us, 4096 x 4096 25 and 23; but 1024 x 4096 6.7 and 7.5)
  const uint32_t all = (uint32_t)sm_count * blocks / p.s.parts * p.s.teams;
  if constexpr (L != kRagged)
    if (p.s.rows > 2 * all && (p.layer || p.q.codes || p.s.rows <= 4 * all) && ring_bytes(p, 2, 2, turned) * blocks <= kRingBytes)
      return start<T, L, G, 2>(p, ring_bytes(p, 2, 3, turned) * blocks <= kRingBytes ? 3 : 2, sm_count, stream);
  return start<T, L, G, 1>(p, ring_bytes(p, 1, 3, turned) * blocks <= kRingBytes ? 3 : 2, sm_count, stream);
}

template <typename T>
cudaError_t apply(ApplyParams p, bool wide, uint32_t rows, uint32_t cols, int sm_count, cudaStream_t stream) {
  for (uint32_t parts = 1;; parts *= 2) {
    p.s = shape_of(rows, cols, wide && !p.q.codes, parts);
    p.image = image_bytes(p.s, sizeof(T), wide);
    if (ring_bytes(p, 1, 2, !wide && p.q.codes) <= kRingBytes) break;
  }
  const bool one = p.s.groups == 1;
  switch (layout_of(p.s, wide)) {
    case kRagged: return one ? start<T, kRagged, 1>(p, sm_count, stream) : start<T, kRagged, 2>(p, sm_count, stream);
    case kWide: return one ? start<T, kWide, 1>(p, sm_count, stream) : start<T, kWide, 2>(p, sm_count, stream);
    default: return one ? start<T, kExact, 1>(p, sm_count, stream) : start<T, kExact, 2>(p, sm_count, stream);
  }
}

}  // namespace

cudaError_t launch_apply(const pvt_norm& n, void* total, int64_t ldt, void* y, int32_t y_dtype, int64_t ldy, const pvt_mx* yq,
                         float* stats, int sm_count, cudaStream_t stream) {
  ApplyParams p = {};
  p.x = n.x, p.ldx = n.ldx, p.residual = n.residual, p.ldr = n.ldr, p.total = total, p.ldt = ldt;
  p.weight = n.weight, p.bias = n.bias, p.w_dtype = n.weight_dtype;
  p.y = y, p.ldy = ldy, p.y_dtype = y_dtype, p.stats = stats, p.eps = n.eps, p.layer = n.kind == PVT_NORM_LAYER;
  p.padded = (uint32_t)n.rows;
  const size_t w_size = n.weight_dtype == PVT_F32 ? 4 : 2;
  p.w_wide = rows_aligned(n.weight, 0, w_size) && rows_aligned(n.bias, 0, w_size);
  if (yq) {
    p.q = mx::held(*yq);
    p.padded = (uint32_t)((n.rows + kStrip - 1) / kStrip * kStrip);
  }
  const size_t y_size = y_dtype == PVT_F32 ? 4 : 2;
  timing_begin(kKernNorm, stream);
  const cudaError_t e = with_type(n.dtype, [&](auto* type) {
    using T = std::remove_pointer_t<decltype(type)>;
    const bool wide = rows_aligned(n.x, n.ldx, sizeof(T)) && rows_aligned(n.residual, n.ldr, sizeof(T)) &&
                      rows_aligned(total, ldt, sizeof(T)) && rows_aligned(y, ldy, y_size);
    return apply<T>(p, wide, (uint32_t)n.rows, (uint32_t)n.cols, sm_count, stream);
  });
  timing_end(kKernNorm, stream);
  count_launches(1);
  return e;
}

}  // namespace norm
}  // namespace pvt
