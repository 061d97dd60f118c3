// Quantisation to 4-bit block floating point and back.
//
// One pass over the matrix: a warp takes 256 or 512 columns of a row, 32 bytes to a lane, so that the lane's codes are one
// 4- or 8-byte store, and a block's largest magnitude is an exchange between at most four lanes.  The scale bytes of four
// blocks leave as one word into their tile.  Bound by HBM for binary32 (28672 x 8192 e8m0 162 us, 164 at the copy's rate), by
// instructions for 16-bit elements under e4m3.
#include "pvt_mx_block.cuh"

namespace pvt {
namespace {

using namespace mx;

constexpr int kQThreads = 256;

// elements of a lane: 32 bytes, or eight where a row is read element by element
template <typename T, bool WIDE>
constexpr int kLaneElements = WIDE ? 32 / (int)sizeof(T) : 8;

template <typename T, int FMT, bool WIDE>
__global__ void __launch_bounds__(kQThreads) mx_quantize_kernel(const T* x, int64_t ldx, uint8_t* codes, int64_t ld, uint8_t* scales,
                                                                const float* tensor_scale, uint32_t rows, uint32_t cols,
                                                                uint32_t tiles, FastDiv spans_div, uint32_t spans,
                                                                uint32_t total) {
  constexpr int E = kLaneElements<T, WIDE>, LANES = (FMT == PVT_MX_E8M0_32 ? 32 : 16) / E;  // of a block
  __shared__ float buffer[WIDE ? 1 : kQThreads / 32][kSpan + 8 * kSpan / 32];
  pdl_trigger();
  pdl_wait();
  const uint32_t lane = threadIdx.x & 31;
  const TensorScale t(FMT == PVT_MX_E4M3_16 ? tensor_scale : nullptr);
  for (uint32_t at = blockIdx.x * (kQThreads / 32) + threadIdx.x / 32; at < total; at += gridDim.x * (kQThreads / 32)) {
    // (a strip's rows that do not exist are spans too: their scales are written)
    const uint32_t row = fast_div(at, spans_div), c0 = (at - row * spans) * (32 * E) + E * lane;
    const uint32_t block = c0 / (E * LANES);
    uint32_t* const to_scales = reinterpret_cast<uint32_t*>(scales + scale_at(row, block, tiles));
    const bool leads = lane % (4 * LANES) == 0 && block / 4 < tiles;  // has the word of four blocks
    if (row >= rows) {
      if (leads) *to_scales = 0;
      continue;
    }
    float v[E];
    const T* const from = x + (int64_t)row * ldx;
    if (!WIDE) {  // lane by lane along the row, then turned
      const uint32_t span0 = c0 - E * lane;
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = span0 + 32 * i + lane < cols ? widen<T>(from[span0 + 32 * i + lane]) : 0.0f;
      turn<false>(buffer[threadIdx.x / 32], v, lane);
    } else if (c0 + E <= cols) {
      T e[E];
#pragma unroll
      for (int i = 0; i < E; i += 8) *reinterpret_cast<Eight<T>*>(e + i) = *reinterpret_cast<const Eight<T>*>(from + c0 + i);
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = widen<T>(e[i]);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = c0 + i < cols ? widen<T>(from[c0 + i]) : 0.0f;
    }
    uint32_t top = 0;  // bits of the largest magnitude: NaN and infinity above every number
#pragma unroll
    for (int i = 0; i < E; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
    for (int s = 1; s < LANES; s *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
    uint32_t word[E / 8], byte = quantize_block<FMT, E>(v, top, t, word);
    if (c0 >= cols) byte = 0;  // no such block, whatever the tensor scale is
    uint32_t four = byte | __shfl_down_sync(0xffffffffu, byte, LANES) << 8;
    four |= __shfl_down_sync(0xffffffffu, four, 2 * LANES) << 16;
    if (leads) *to_scales = four;
    uint8_t* const to = codes + (int64_t)row * ld + c0 / 2;
    if (c0 + E <= cols) {
      if (E == 16)
        *reinterpret_cast<uint2*>(to) = make_uint2(word[0], word[E / 8 - 1]);
      else
        *reinterpret_cast<uint32_t*>(to) = word[0];
    } else if (c0 < cols) {
#pragma unroll
      for (uint32_t i = 0; i < E / 2; ++i)
        if (2 * i < cols - c0) to[i] = (uint8_t)(word[i / 4] >> (8 * (i % 4)));
    }
  }
}

// eight elements times their scale and the tensor's
template <int FMT>
__device__ __forceinline__ void values_of(uint32_t w, uint32_t byte, float ts, float* v) {
  const float s = FMT == PVT_MX_E8M0_32 ? e8m0_value(byte) : e4m3_float(byte);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // the three bits of the magnitude as the low exponent bits and the first fraction bit of a binary32, whose bias
    // is 126 more: a product with 2^126 gives the element, 0.5 from a number without its leading one included
    const uint32_t n = w >> (4 * i);
    const float el = __uint_as_float((n & 7u) << 22 | (n & 8u) << 28) * 8.507059173023462e37f;
    v[i] = el * s * ts;
  }
}

// Few columns: one row after the other would leave most lanes without work, so a warp takes 32 / LANES rows of up to 8 LANES
// columns, eight to a lane.  Between memory and lanes they go by way of shared memory: a warp reads or writes 32 elements
// at a time, in the order of rows.  By a row to a warp and so: 5581843 x 21 fp16 to e8m0 1166 and 277 us, back to binary32 1099 and
// 221; 118801 x 110, back, rows of no alignment, 28 and 20.  (Wide accesses of 65 columns and more: 1000000 x 128 back 148 us by a row
// to a warp, 175 so.)
template <int LANES>
struct NarrowRows {
  static constexpr uint32_t kRows = 32 / LANES;
  uint32_t lane, row0, n;  // n: elements of the warp's rows
  __device__ __forceinline__ NarrowRows(uint32_t at, uint32_t rows, uint32_t cols)
      : lane(threadIdx.x & 31), row0(at * kRows), n(row0 < rows ? min(kRows, rows - row0) * cols : 0) {}
  __device__ __forceinline__ uint32_t row() const { return row0 + lane / LANES; }
  __device__ __forceinline__ uint32_t col() const { return lane % LANES * 8; }
  // place of an element of this lane's row in shared memory
  __device__ __forceinline__ uint32_t place(uint32_t c, uint32_t cols) const { return lane / LANES * cols + c; }
};

template <typename T, int FMT, int LANES>
__global__ void __launch_bounds__(kQThreads) mx_quantize_narrow_kernel(const T* x, int64_t ldx, uint8_t* codes, int64_t ld, uint8_t* scales,
                                                                       const float* tensor_scale, uint32_t rows, FastDiv by_cols,
                                                                       uint32_t cols, uint32_t tiles, uint32_t total) {
  constexpr int OF_BLOCK = FMT == PVT_MX_E8M0_32 ? 4 : 2;           // lanes
  constexpr int WORDS = LANES > 4 * OF_BLOCK ? LANES / (4 * OF_BLOCK) : 1;  // of four scales that a row's lanes have
  __shared__ float buffer[kQThreads / 32][kSpan];
  pdl_trigger();
  pdl_wait();
  const TensorScale t(FMT == PVT_MX_E4M3_16 ? tensor_scale : nullptr);
  float* const own = buffer[threadIdx.x / 32];
  for (uint32_t at = blockIdx.x * (kQThreads / 32) + threadIdx.x / 32; at < total; at += gridDim.x * (kQThreads / 32)) {
    const NarrowRows<LANES> m(at, rows, cols);
    __syncwarp();
    for (uint32_t i = m.lane; i < m.n; i += 32) {
      const uint32_t r = fast_div(i, by_cols);
      own[i] = widen<T>(x[(int64_t)(m.row0 + r) * ldx + (i - r * cols)]);
    }
    __syncwarp();
    const uint32_t row = m.row(), c0 = m.col();
    const bool here = row < rows && c0 < cols;
    float v[8];
    uint32_t top = 0, word;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = here && c0 + i < cols ? own[m.place(c0 + i, cols)] : 0.0f;
      top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    }
#pragma unroll
    for (int s = 1; s < OF_BLOCK; s *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
    uint32_t byte = quantize_block<FMT, 8>(v, top, t, &word);
    if (!here) byte = 0;
    uint32_t four = byte;
    if (LANES >= 2 * OF_BLOCK) four |= __shfl_down_sync(0xffffffffu, byte, OF_BLOCK) << 8;
    if (LANES >= 4 * OF_BLOCK) four |= __shfl_down_sync(0xffffffffu, four, 2 * OF_BLOCK) << 16;
    // (a strip's rows that do not exist, and blocks that do not, have scales too)
    const uint32_t first = m.lane % LANES;
    if (first % (4 * OF_BLOCK) == 0) *reinterpret_cast<uint32_t*>(scales + scale_at(row, first / OF_BLOCK, tiles)) = four;
    if (first == 0)
      for (uint32_t w = WORDS; w < tiles; ++w) *reinterpret_cast<uint32_t*>(scales + scale_at(row, 4 * w, tiles)) = 0;
    if (!here) continue;
    uint8_t* const to = codes + (int64_t)row * ld + c0 / 2;
    if (c0 + 8 <= cols) {
      *reinterpret_cast<uint32_t*>(to) = word;
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (2 * i < cols - c0) to[i] = (uint8_t)(word >> (8 * i));
    }
  }
}

template <typename T, int FMT, int LANES>
__global__ void __launch_bounds__(kQThreads) mx_dequant_narrow_kernel(const uint8_t* codes, int64_t ld, const uint8_t* scales,
                                                                      const float* tensor_scale, T* values, int64_t ldv, uint32_t rows,
                                                                      FastDiv by_cols, uint32_t cols, uint32_t tiles, uint32_t total) {
  __shared__ float buffer[kQThreads / 32][kSpan];
  pdl_trigger();
  pdl_wait();
  const float ts = FMT == PVT_MX_E4M3_16 && tensor_scale ? *tensor_scale : 1.0f;
  float* const own = buffer[threadIdx.x / 32];
  for (uint32_t at = blockIdx.x * (kQThreads / 32) + threadIdx.x / 32; at < total; at += gridDim.x * (kQThreads / 32)) {
    const NarrowRows<LANES> m(at, rows, cols);
    const uint32_t row = m.row(), c0 = m.col();
    __syncwarp();
    if (row < rows && c0 < cols) {  // (the four bytes lie in the row: ld is a multiple of 16)
      float v[8];
      values_of<FMT>(*reinterpret_cast<const uint32_t*>(codes + (int64_t)row * ld + c0 / 2),
                     scales[scale_at(row, c0 / (FMT == PVT_MX_E8M0_32 ? 32 : 16), tiles)], ts, v);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c0 + i < cols) own[m.place(c0 + i, cols)] = v[i];
    }
    __syncwarp();
    for (uint32_t i = m.lane; i < m.n; i += 32) {
      const uint32_t r = fast_div(i, by_cols);
      values[(int64_t)(m.row0 + r) * ldv + (i - r * cols)] = narrow<T>(own[i]);
    }
  }
}

// Eight elements to a lane; the next span's codes are asked for ahead of this one's stores.
template <typename T, int FMT, bool WIDE>
__global__ void __launch_bounds__(kQThreads) mx_dequant_kernel(const uint8_t* codes, int64_t ld, const uint8_t* scales,
                                                               const float* tensor_scale, T* values, int64_t ldv, uint32_t rows,
                                                               uint32_t cols, uint32_t tiles, FastDiv spans_div,
                                                               uint32_t spans, uint32_t total) {
  constexpr int BLOCK = FMT == PVT_MX_E8M0_32 ? 32 : 16;
  __shared__ float buffer[WIDE ? 1 : kQThreads / 32][kSpan + 8 * kSpan / 32];
  pdl_trigger();
  pdl_wait();
  const uint32_t lane = threadIdx.x & 31;
  const float ts = FMT == PVT_MX_E4M3_16 && tensor_scale ? *tensor_scale : 1.0f;
  const uint32_t warps = gridDim.x * (kQThreads / 32);
  uint32_t row, c0, word, byte;
  auto ask = [&](uint32_t at) {
    row = fast_div(at, spans_div), c0 = (at - row * spans) * kSpan + 8 * lane, word = byte = 0;
    if (at < total && c0 < cols) {  // (the four bytes lie in the row: ld is a multiple of 16)
      word = *reinterpret_cast<const uint32_t*>(codes + (int64_t)row * ld + c0 / 2);
      byte = scales[scale_at(row, c0 / BLOCK, tiles)];
    }
  };
  uint32_t next = blockIdx.x * (kQThreads / 32) + threadIdx.x / 32;
  ask(next);
  while (next < total) {
    const uint32_t r = row, c = c0, w = word, b = byte;
    ask(next += warps);
    float v[8];
    values_of<FMT>(w, b, ts, v);
    T* const to = values + (int64_t)r * ldv;
    if (!WIDE) {
      turn<true>(buffer[threadIdx.x / 32], v, lane);
      const uint32_t span0 = c - 8 * lane;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (span0 + 32 * i + lane < cols) to[span0 + 32 * i + lane] = narrow<T>(v[i]);
    } else if (c + 8 <= cols) {
      if constexpr (sizeof(T) == 4) {
        store8(to + c, true, v);
      } else {
        Eight<T> e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = narrow<T>(v[i]);
        *reinterpret_cast<Eight<T>*>(to + c) = e;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < cols) to[c + i] = narrow<T>(v[i]);
    }
  }
}

// eight elements at a time, wherever a lane's begin
bool rows_aligned(const void* p, int64_t ld, size_t size) {
  return reinterpret_cast<uintptr_t>(p) % (8 * size) == 0 && ld % 8 == 0;
}

unsigned span_grid(uint32_t total, int per_sm, int sm_count) {
  const uint32_t need = (total + kQThreads / 32 - 1) / (kQThreads / 32), most = (uint32_t)(sm_count * per_sm);
  return need < most ? need : most;
}
// Blocks per SM on the way back: as many as are resident, or many that follow one another where the values are far more than
// the L2 holds (28672 x 8192 to binary32: 198 and 168 us, 8192 x 8192 57 and 51; 2047 x 5001 11.4 and 13.3).
int blocks_back(uint32_t total) { return total > 150000 ? 64 : 8; }

template <typename T, int FMT, bool WIDE>
cudaError_t quantize(const pvt_mx& m, const T* x, int64_t ldx, int sm_count, cudaStream_t stream) {
  constexpr uint32_t span = 32 * kLaneElements<T, WIDE>;
  const uint32_t spans = ((uint32_t)m.cols + span - 1) / span;
  const uint32_t total = ((uint32_t)m.rows + kStrip - 1) / kStrip * kStrip * spans;
  return launch_dependent(mx_quantize_kernel<T, FMT, WIDE>, span_grid(total, 8, sm_count), kQThreads, 0, stream, x, ldx, m.codes,
                          m.ld, m.scales, m.tensor_scale, (uint32_t)m.rows, (uint32_t)m.cols,
                          strip_tiles(m.cols, block_of(FMT)), make_fast_div(spans), spans, total);
}
template <typename T, int FMT, int LANES>
cudaError_t quantize_narrow(const pvt_mx& m, const T* x, int64_t ldx, int sm_count, cudaStream_t stream) {
  const uint32_t total = ((uint32_t)m.rows + kStrip - 1) / kStrip * kStrip / (32 / LANES);
  return launch_dependent(mx_quantize_narrow_kernel<T, FMT, LANES>, span_grid(total, 8, sm_count), kQThreads, 0, stream, x, ldx, m.codes,
                          m.ld, m.scales, m.tensor_scale, (uint32_t)m.rows, make_fast_div((uint32_t)m.cols), (uint32_t)m.cols,
                          strip_tiles(m.cols, block_of(FMT)), total);
}
template <typename T, int FMT>
cudaError_t quantize(const pvt_mx& m, const T* x, int64_t ldx, int sm_count, cudaStream_t stream) {
  if (m.cols <= 32) return quantize_narrow<T, FMT, 4>(m, x, ldx, sm_count, stream);
  if (m.cols <= 64) return quantize_narrow<T, FMT, 8>(m, x, ldx, sm_count, stream);
  if (m.cols <= 128 && !rows_aligned(x, ldx, sizeof(T))) return quantize_narrow<T, FMT, 16>(m, x, ldx, sm_count, stream);
  return rows_aligned(x, ldx, sizeof(T)) ? quantize<T, FMT, true>(m, x, ldx, sm_count, stream)
                                         : quantize<T, FMT, false>(m, x, ldx, sm_count, stream);
}

template <typename T, int FMT, int LANES>
cudaError_t dequant_narrow(const pvt_mx& m, T* values, int64_t ldv, int sm_count, cudaStream_t stream) {
  const uint32_t total = ((uint32_t)m.rows + 32 / LANES - 1) / (32 / LANES);
  return launch_dependent(mx_dequant_narrow_kernel<T, FMT, LANES>, span_grid(total, 8, sm_count), kQThreads, 0, stream,
                          (const uint8_t*)m.codes, m.ld, (const uint8_t*)m.scales, m.tensor_scale, values, ldv, (uint32_t)m.rows,
                          make_fast_div((uint32_t)m.cols), (uint32_t)m.cols, strip_tiles(m.cols, block_of(FMT)), total);
}
template <typename T, int FMT>
cudaError_t dequant(const pvt_mx& m, T* values, int64_t ldv, int sm_count, cudaStream_t stream) {
  if (m.cols <= 32) return dequant_narrow<T, FMT, 4>(m, values, ldv, sm_count, stream);
  if (m.cols <= 64) return dequant_narrow<T, FMT, 8>(m, values, ldv, sm_count, stream);
  if (m.cols <= 128 && !rows_aligned(values, ldv, sizeof(T))) return dequant_narrow<T, FMT, 16>(m, values, ldv, sm_count, stream);
  const uint32_t spans = ((uint32_t)m.cols + kSpan - 1) / kSpan, total = (uint32_t)m.rows * spans;
  auto kernel = rows_aligned(values, ldv, sizeof(T)) ? mx_dequant_kernel<T, FMT, true> : mx_dequant_kernel<T, FMT, false>;
  return launch_dependent(kernel, span_grid(total, blocks_back(total), sm_count), kQThreads, 0, stream, (const uint8_t*)m.codes, m.ld,
                          (const uint8_t*)m.scales, m.tensor_scale, values, ldv, (uint32_t)m.rows, (uint32_t)m.cols,
                          strip_tiles(m.cols, block_of(FMT)), make_fast_div(spans), spans, total);
}

template <typename T>
cudaError_t quantize(const pvt_mx& m, const void* x, int64_t ldx, int sm_count, cudaStream_t stream) {
  return m.format == PVT_MX_E8M0_32 ? quantize<T, PVT_MX_E8M0_32>(m, static_cast<const T*>(x), ldx, sm_count, stream)
                                    : quantize<T, PVT_MX_E4M3_16>(m, static_cast<const T*>(x), ldx, sm_count, stream);
}
template <typename T>
cudaError_t dequant(const pvt_mx& m, void* values, int64_t ldv, int sm_count, cudaStream_t stream) {
  return m.format == PVT_MX_E8M0_32 ? dequant<T, PVT_MX_E8M0_32>(m, static_cast<T*>(values), ldv, sm_count, stream)
                                    : dequant<T, PVT_MX_E4M3_16>(m, static_cast<T*>(values), ldv, sm_count, stream);
}

}  // namespace

cudaError_t launch_mx_quantize(const pvt_mx& m, const void* x, int32_t dtype, int64_t ldx, int sm_count, cudaStream_t stream) {
  timing_begin(kKernMx, stream);
  const cudaError_t e = dtype == PVT_F32   ? quantize<float>(m, x, ldx, sm_count, stream)
                        : dtype == PVT_F16 ? quantize<__half>(m, x, ldx, sm_count, stream)
                                           : quantize<__nv_bfloat16>(m, x, ldx, sm_count, stream);
  timing_end(kKernMx, stream);
  count_launches(1);
  return e;
}

cudaError_t launch_mx_dequant(const pvt_mx& m, void* values, int32_t dtype, int64_t ldv, int sm_count, cudaStream_t stream) {
  timing_begin(kKernMx, stream);
  const cudaError_t e = dtype == PVT_F32   ? dequant<float>(m, values, ldv, sm_count, stream)
                        : dtype == PVT_F16 ? dequant<__half>(m, values, ldv, sm_count, stream)
                                           : dequant<__nv_bfloat16>(m, values, ldv, sm_count, stream);
  timing_end(kKernMx, stream);
  count_launches(1);
  return e;
}

}  // namespace pvt
