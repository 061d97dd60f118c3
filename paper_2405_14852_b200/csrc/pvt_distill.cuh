// Distillation from a teacher's top logits: rows of any alignment in pieces of 16 bytes, running sums of exponentials.
#pragma once

#include "pvt_mma.cuh"
#include "pvt_mx.cuh"

namespace pvt {
namespace distill {

constexpr int kThreads = 512;

#ifdef __CUDACC__
using mx::narrow;
using mx::widen;

template <typename T>
struct alignas(16) Piece {
  static constexpr uint32_t N = 16 / sizeof(T);
  T v[N];
};

// A row of n elements as a head of fewer than N, pieces on 16-byte boundaries, and a tail of fewer than N; and the share of one
// of `blocks` blocks of it: a range of pieces, the head to the first block, the tail to the last.
template <typename T>
struct RowShare {
  uint32_t head, lo, hi, tail;  // pieces [lo, hi); the tail begins at element `tail`
  bool first, last;
  uint32_t n;
  __device__ __forceinline__ RowShare(const T* row, uint32_t n_, uint32_t rank, uint32_t blocks) : n(n_) {
    constexpr uint32_t N = Piece<T>::N;
    head = min((uint32_t)(-(int64_t)(reinterpret_cast<uintptr_t>(row) / sizeof(T))) % N, n);
    const uint32_t pieces = (n - head) / N;
    tail = head + pieces * N;
    lo = (uint32_t)((uint64_t)pieces * rank / blocks);
    hi = (uint32_t)((uint64_t)pieces * (rank + 1) / blocks);
    first = rank == 0;
    last = rank + 1 == blocks;
  }
  // elements outside the pieces that this block has: numbers 0 .. loose() - 1
  __device__ __forceinline__ uint32_t loose() const { return (first ? head : 0) + (last ? n - tail : 0); }
  __device__ __forceinline__ uint32_t loose_at(uint32_t i) const { return first && i < head ? i : tail + i - (first ? head : 0); }
  // elements [from, to) of the row are this block's
  __device__ __forceinline__ uint32_t from() const { return first ? 0 : head + lo * Piece<T>::N; }
  __device__ __forceinline__ uint32_t to() const { return last ? n : head + hi * Piece<T>::N; }
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kMinusInf = -__builtin_huge_valf();

// Largest value and the sums of 2^(c (x - largest)) relative to it.  Differences are formed before the product with c: the terms
// that make up the sum have small ones.
struct Running {
  float m = kMinusInf, z = 0.0f, r = 0.0f;
  // the sums relative to a larger (or equal) value; -infinity stands for no terms
  __device__ __forceinline__ void raise(float to, float c) {
    if (m < to) {
      const float f = m == kMinusInf ? 0.0f : ex2((m - to) * c);
      // (z is 0, or a NaN that stays one, as long as m is -infinity)
      z *= f, r *= f, m = to;
    }
  }
  // (1 at the largest, an infinite one included; without any, -infinity adds nothing and a NaN itself)
  __device__ __forceinline__ float term(float x, float c) const {
    return x == m ? (m == kMinusInf ? 0.0f : 1.0f) : ex2((x - m) * c);
  }
};

__device__ __forceinline__ Running merge(Running a, Running b, float c) {
  const float m = fmaxf(a.m, b.m);
  a.raise(m, c), b.raise(m, c);
  a.z += b.z, a.r += b.r;
  return a;
}
__device__ __forceinline__ Running warp_merge(Running a, float c) {
#pragma unroll
  for (int s = 16; s >= 1; s /= 2) {
    Running b;
    b.m = __shfl_xor_sync(0xffffffffu, a.m, s);
    b.z = __shfl_xor_sync(0xffffffffu, a.z, s);
    b.r = __shfl_xor_sync(0xffffffffu, a.r, s);
    a = merge(a, b, c);
  }
  return a;
}
// over the block, the same in every thread; `sh`: a slot per warp
__device__ __forceinline__ Running block_merge(Running a, float c, Running* sh) {
  a = warp_merge(a, c);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x / 32] = a;
  __syncthreads();
  a = sh[0];
  for (int w = 1; w < kThreads / 32; ++w) a = merge(a, sh[w], c);
  return a;
}
#endif

// blocks that share a row: as many as leave no SM without work, while each has a few pieces per thread
inline uint32_t row_blocks(int64_t rows, int64_t row_bytes, int sm_count) {
  uint32_t c = 1;
  while (c < 8 && rows * c * 2 <= 2 * (int64_t)sm_count && row_bytes / (c * 2) >= kThreads * 16) c *= 2;
  return c;
}

}  // namespace distill

cudaError_t launch_distill_top(const void* logits, int32_t dtype, int64_t ld, int64_t rows, int32_t vocab, int32_t k,
                               float temperature, int32_t* top_idx, float* top_logit, float* lse, int sm_count,
                               cudaStream_t stream);
cudaError_t launch_distill_loss(const pvt_distill& d, float* loss, float* stats, const float* upstream, void* grad,
                                int32_t grad_dtype, int64_t ldg, uint32_t* status, int sm_count, cudaStream_t stream);
cudaError_t launch_distill_grad(const pvt_distill& d, const float* stats, const float* upstream, void* grad, int32_t grad_dtype,
                                int64_t ldg, uint32_t* status, int sm_count, cudaStream_t stream);

}  // namespace pvt
