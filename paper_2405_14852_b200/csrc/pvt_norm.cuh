// What the two directions of the norm share: types known at run time, rows in registers, launch parameters.
//
// A row's columns are spans of 256, one to a warp at a time, eight elements to a lane: neighbouring ones where every row begins
// on eight elements' boundary, otherwise (WIDE = false) `lanes` apart, so that a warp's accesses run along the row.  Rows of one
// span share a block's warps, and those of at most 64 or 128 columns share a warp: a row is then a team of 8 or 16 lanes.
#pragma once

#include <type_traits>

#include "pvt_mx.cuh"

namespace pvt {
namespace norm {

constexpr uint32_t kSpanCols = 256;

struct Shape {
  uint32_t rows, cols;
  uint32_t spans;  // of 256 columns
  uint32_t lanes;  // of a row, where one warp or less has it; 32 otherwise
  uint32_t warps;  // of a row
  uint32_t teams;  // rows that a block has at a time
};
// `groups` spans to a warp; threads: of a block, where a row takes less
inline Shape shape_of(uint32_t rows, uint32_t cols, uint32_t groups, uint32_t threads, bool narrow) {
  Shape s = {rows, cols, (cols + kSpanCols - 1) / kSpanCols, 32, 1, 1};
  s.warps = (s.spans + groups - 1) / groups;
  if (s.warps > 1) return s;
  if (narrow && cols <= 128) s.lanes = cols <= 64 ? 8 : 16;
  s.teams = threads / s.lanes;
  return s;
}

cudaError_t launch_apply(const pvt_norm& n, void* total, int64_t ldt, void* y, int32_t y_dtype, int64_t ldy, const pvt_mx* yq,
                         float* stats, int sm_count, cudaStream_t stream);
size_t grad_workspace_bytes(int64_t rows, int32_t cols, int sm_count);
cudaError_t launch_grad(const pvt_norm& n, const float* stats, int32_t dtype, const void* dy, int64_t lddy, const void* dres,
                        int64_t lddr, void* dx, int64_t lddx, void* dweight, void* dbias, int32_t dw_dtype, bool accumulate, void* ws,
                        int sm_count, cudaStream_t stream);

inline bool rows_aligned(const void* p, int64_t ld, size_t size) {
  return !p || (reinterpret_cast<uintptr_t>(p) % (8 * size) == 0 && ld % 8 == 0);
}

// calls f with a null pointer to the type
#ifdef __CUDACC__
#pragma nv_exec_check_disable
#endif
template <typename F>
__host__ __device__ __forceinline__ auto with_type(int32_t dtype, F f) {
  if (dtype == PVT_F32) return f(static_cast<float*>(nullptr));
  if (dtype == PVT_F16) return f(static_cast<__half*>(nullptr));
  return f(static_cast<__nv_bfloat16*>(nullptr));
}

#ifdef __CUDACC__
using mx::Eight;
using mx::narrow;
using mx::widen;

// eight elements of a row from column c on, `step` apart (1 if WIDE); 0 behind its end
template <bool WIDE, typename T>
__device__ __forceinline__ void take(const T* row, uint32_t c, uint32_t step, uint32_t cols, T* v) {
  if (WIDE && c + 8 <= cols) {
    const Eight<T> e = *reinterpret_cast<const Eight<T>*>(row + c);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i * step < cols ? row[c + i * step] : narrow<T>(0.0f);
  }
}
template <bool WIDE, typename T>
__device__ __forceinline__ void put(T* row, uint32_t c, uint32_t step, uint32_t cols, const float* v) {
  if (WIDE && c + 8 <= cols) {
    Eight<T> e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = narrow<T>(v[i]);
    *reinterpret_cast<Eight<T>*>(row + c) = e;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i * step < cols) row[c + i * step] = narrow<T>(v[i]);
  }
}
// the weights of eight columns, `other` where there are none
template <bool WIDE>
__device__ __forceinline__ void take_weights(const void* w, int32_t dtype, bool wide, uint32_t c, uint32_t step, uint32_t cols,
                                             float other, float* v) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = other;
    return;
  }
  with_type(dtype, [&](auto* type) {
    using U = std::remove_pointer_t<decltype(type)>;
    U e[8];
    if (WIDE && wide)
      take<true>(static_cast<const U*>(w), c, 1, cols, e);
    else
      take<false>(static_cast<const U*>(w), c, step, cols, e);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = widen<U>(e[i]);
  });
}

// over the lanes of a team
__device__ __forceinline__ float team_sum(float v, uint32_t lanes) {
  if (lanes > 16) v += __shfl_xor_sync(0xffffffffu, v, 16);
  if (lanes > 8) v += __shfl_xor_sync(0xffffffffu, v, 8);
#pragma unroll
  for (int s = 4; s > 0; s /= 2) v += __shfl_xor_sync(0xffffffffu, v, s);
  return v;
}
#endif

}  // namespace norm
}  // namespace pvt
