// Distillation from a teacher's top logits: rows of any alignment in pieces of 16 bytes, running sums of exponentials.
#pragma once

#include "pvt_mma.cuh"
#include "pvt_mx.cuh"

namespace pvt {
namespace distill {

constexpr int kThreads = 256;
constexpr int kResident = 4;  // blocks per SM: while some settle their lists the others' loads are in flight
constexpr int kMaxBlocks = 8;  // of a row

#ifdef __CUDACC__
using mx::narrow;
using mx::widen;

constexpr float kMinusInf = -__builtin_huge_valf();

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

// ---- two binary32 numbers per instruction --------------------------------------------------------------
using Two = unsigned long long;
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 each(Two v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// the larger one; a NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// elements 2 i and 2 i + 1 of a piece
__device__ __forceinline__ Two pair_of(const Piece<float>& p, int i) { return two(p.v[2 * i], p.v[2 * i + 1]); }
__device__ __forceinline__ Two pair_of(const Piece<__half>& p, int i) {
  const float2 f = __half22float2(reinterpret_cast<const __half2*>(p.v)[i]);
  return two(f.x, f.y);
}
__device__ __forceinline__ Two pair_of(const Piece<__nv_bfloat16>& p, int i) {
  const uint32_t u = reinterpret_cast<const uint32_t*>(p.v)[i];
  return two(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
// the largest element, a NaN if there is one
__device__ __forceinline__ float largest(const Piece<float>& p) {
  return max_nan(max_nan(p.v[0], p.v[1]), max_nan(p.v[2], p.v[3]));
}
__device__ __forceinline__ float largest(const Piece<__half>& p) {
  const __half2* h = reinterpret_cast<const __half2*>(p.v);
  const __half2 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return __half2float(__hmax_nan(__low2half(m), __high2half(m)));
}
__device__ __forceinline__ float largest(const Piece<__nv_bfloat16>& p) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(p.v);
  const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return __bfloat162float(__hmax_nan(__low2bfloat16(m), __high2bfloat16(m)));
}

// ---- sums of exponentials ---------------------------------------------------------------------------------
// Largest value so far, and sums of 2^(c (x - base)) where base is the largest value, or 0 as long as that is infinite: a sum
// over -infinity alone is 0, one with infinity infinite, one with a NaN a NaN.  Differences are formed before the product
// with c, for the terms that make up the sum have small ones.
struct Running {
  float m = kMinusInf, z = 0.0f, r = 0.0f;
  __device__ __forceinline__ float base() const { return fabsf(m) == -kMinusInf ? 0.0f : m; }
  __device__ __forceinline__ void raise(float to, float c) {
    if (to > m) {
      const float f = m == kMinusInf || to == -kMinusInf ? 0.0f : ex2((m - to) * c);
      z *= f, r *= f, m = to;
    }
  }
};
// the N terms of a piece, added in pairs
template <typename T>
__device__ __forceinline__ float terms(const Piece<T>& p, float base, float c) {
  const Two b = two(-base, -base), cc = two(c, c);
  Two sum = 0;
#pragma unroll
  for (uint32_t i = 0; i < Piece<T>::N / 2; ++i) {
    const float2 y = each(mul2(add2(pair_of(p, i), b), cc));
    sum = add2(sum, two(ex2(y.x), ex2(y.y)));
  }
  const float2 s = each(sum);
  return s.x + s.y;
}

__device__ __forceinline__ Running merge(Running a, Running b, float c) {
  const float m = fmaxf(a.m, b.m);
  a.raise(m, c), b.raise(m, c);
  a.z += b.z, a.r += b.r;
  return a;
}
// over `lanes` lanes (a power of two) that begin at a multiple of it
__device__ __forceinline__ Running warp_merge(Running a, float c, int lanes = 32) {
  for (int s = lanes / 2; s >= 1; s /= 2) {
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
  constexpr int kWarps = kThreads / 32;
  a = warp_merge(a, c);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x / 32] = a;
  __syncthreads();
  return warp_merge(sh[threadIdx.x % kWarps], c, kWarps);
}
// over the cluster, the same in every thread; `mine`: the block's own sums, in shared memory before the cluster's barrier
__device__ __forceinline__ Running cluster_merge(const Running* mine, uint32_t blocks, float c) {
  const uint32_t at = mma::smem_u32(mine), q = threadIdx.x % kMaxBlocks;
  Running a;
  if (q < blocks) {
    a.m = mma::cluster_load(at + (uint32_t)offsetof(Running, m), q);
    a.z = mma::cluster_load(at + (uint32_t)offsetof(Running, z), q);
    a.r = mma::cluster_load(at + (uint32_t)offsetof(Running, r), q);
  }
  __syncwarp();
  return warp_merge(a, c, kMaxBlocks);
}
#endif

// blocks that share a row: as many as leave no SM without work, while each has a few pieces per thread
inline uint32_t row_blocks(int64_t rows, int64_t row_bytes, int sm_count) {
  uint32_t c = 1;
  while (c < (uint32_t)kMaxBlocks && rows * c * 2 <= 2 * (int64_t)sm_count && row_bytes / (c * 2) >= 2 * kThreads * 16) c *= 2;
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
