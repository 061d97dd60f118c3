// 4-bit block floating point: sizes, where a scale lies, loads and stores of rows of any alignment.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pvt_internal.h"

namespace pvt {
namespace mx {

constexpr int kStrip = 128;      // rows of a strip of scale tiles
constexpr int kTileBytes = 512;  // 128 rows x 4 blocks
constexpr int kSpan = 256;       // columns that scales are laid out for at a time: one step of the product

inline int block_of(int format) { return format == PVT_MX_E8M0_32 ? 32 : 16; }
// tiles of a strip
__host__ __device__ inline uint32_t strip_tiles(int cols, int block) {
  return ((uint32_t)cols + kSpan - 1) / kSpan * (uint32_t)(kSpan / 4 / block);
}
inline size_t scale_bytes(int rows, int cols, int format) {
  return (size_t)((rows + kStrip - 1) / kStrip) * strip_tiles(cols, block_of(format)) * kTileBytes;
}

#ifdef __CUDACC__
// byte of block b of row r
__device__ __forceinline__ size_t scale_at(uint32_t r, uint32_t b, uint32_t tiles) {
  return ((size_t)(r / kStrip) * tiles + b / 4) * kTileBytes + (r % 32) * 16 + (r % kStrip / 32) * 4 + b % 4;
}

template <typename T>
__device__ __forceinline__ float widen(T v);
template <>
__device__ __forceinline__ float widen<float>(float v) { return v; }
template <>
__device__ __forceinline__ float widen<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// eight elements as they lie in memory, 16 or 32 bytes
template <typename T>
struct alignas(8 * sizeof(T)) Eight {
  T v[8];
};

// the value of an e4m3 scale byte without its sign: exact in binary32
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  const uint32_t e = byte >> 3 & 15, m = byte & 7;
  if ((byte & 127) == 127) return __uint_as_float(0x7fc00000u);
  return e ? __uint_as_float((e + 120) << 23 | m << 20) : (float)m * 0.001953125f;
}
// the same by the conversion unit, through binary16
__device__ __forceinline__ float e4m3_float(uint32_t byte) {
  uint32_t two;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(two) : "h"((uint16_t)byte));
  return __low2float(*reinterpret_cast<const __half2*>(&two));
}
// What a sum is multiplied by, one after the other, for two factors of its terms: their product and 1, or both by themselves, the
// larger one first, where the product is no normal number (a sum that is 0 stays 0, and no bits are lost).
struct Factors {
  float first, second;
  __device__ __forceinline__ Factors(float a, float b) {
    const float both = a * b;
    const bool normal = both >= 1.17549435e-38f && both <= 3.40282347e38f;
    first = normal ? both : a > b ? a : b;
    second = normal ? 1.0f : a > b ? b : a;
  }
  __device__ __forceinline__ float operator()(float sum) const { return sum * first * second; }
};
// 2^(byte - 127); 255 is NaN
__device__ __forceinline__ float e8m0_value(uint32_t byte) {
  return byte == 255 ? __uint_as_float(0x7fc00000u) : byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
}
#endif

}  // namespace mx

cudaError_t launch_mx_quantize(const pvt_mx& m, const void* x, int32_t dtype, int64_t ldx, int sm_count, cudaStream_t stream);
cudaError_t launch_mx_dequant(const pvt_mx& m, void* values, int32_t dtype, int64_t ldv, int sm_count, cudaStream_t stream);
cudaError_t launch_mx_product(const pvt_mx& x, const pvt_mx& w, void* y, int32_t dtype, int64_t ldy, uint32_t* status,
                              int sm_count, cudaStream_t stream);
// dx (input) or dw (weight): a 16-bit matrix times a held one along the held one's rows
cudaError_t launch_mx_grad_input(const void* dy, int64_t lddy, int32_t tokens, const pvt_mx& w, void* dx, int32_t dtype,
                                 int64_t lddx, uint32_t* status, int sm_count, cudaStream_t stream);
cudaError_t launch_mx_grad_weight(const void* dy, int64_t lddy, int32_t n, const pvt_mx& x, float* dw, int64_t lddw,
                                  bool accumulate, uint32_t* status, int sm_count, cudaStream_t stream);

}  // namespace pvt
