// Distillation from a teacher's top logits: rows of any alignment in pieces of 16 bytes, running sums of exponentials.
#pragma once

#include "pvt_mma.cuh"
#include "pvt_mx.cuh"

namespace pvt {
namespace distill {

// A block takes a row, or a part of one.  Where many short rows leave 256 threads little to do, it has 64 (20000 x 2000 bf16, 20
// listed: the list 155 and 122 us, loss and gradient 155 and 115; 9358 x 1042 fp32, 13 listed: 73 and 50, 89 and 60).
constexpr int kWide = 256, kNarrow = 64;
// blocks per SM: while some settle their lists the others' loads are in flight
constexpr int kResident = 5, kResidentNarrow = 20;
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
// The largest elements, NaN where there is one: in as many places as a register holds (Top), and of those.
template <typename T>
struct Tops;
template <>
struct Tops<float> {
  using Top = float;
  static __device__ __forceinline__ Top lowest() { return kMinusInf; }
  static __device__ __forceinline__ Top max(Top a, Top b) { return max_nan(a, b); }
  static __device__ __forceinline__ Top of(const Piece<float>& p) { return max_nan(max_nan(p.v[0], p.v[1]), max_nan(p.v[2], p.v[3])); }
  static __device__ __forceinline__ float value(Top a) { return a; }
  static __device__ __forceinline__ Top limit(float x) { return x; }
  static __device__ __forceinline__ bool reaches(Top a, Top least) { return !(a < least); }  // a NaN does
};
template <>
struct Tops<__half> {
  using Top = __half2;
  static __device__ __forceinline__ Top lowest() { return __float2half2_rn(kMinusInf); }
  static __device__ __forceinline__ Top max(Top a, Top b) { return __hmax2_nan(a, b); }
  static __device__ __forceinline__ Top of(const Piece<__half>& p) {
    const __half2* h = reinterpret_cast<const __half2*>(p.v);
    return max(max(h[0], h[1]), max(h[2], h[3]));
  }
  static __device__ __forceinline__ float value(Top a) { return max_nan(__low2float(a), __high2float(a)); }
  // the smallest one that is not below x
  static __device__ __forceinline__ Top limit(float x) { return __half2half2(__float2half_ru(x)); }
  static __device__ __forceinline__ bool reaches(Top a, Top least) { return __hgeu2_mask(a, least) != 0; }
};
template <>
struct Tops<__nv_bfloat16> {
  using Top = __nv_bfloat162;
  static __device__ __forceinline__ Top lowest() { return __float2bfloat162_rn(kMinusInf); }
  static __device__ __forceinline__ Top max(Top a, Top b) { return __hmax2_nan(a, b); }
  static __device__ __forceinline__ Top of(const Piece<__nv_bfloat16>& p) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(p.v);
    return max(max(h[0], h[1]), max(h[2], h[3]));
  }
  static __device__ __forceinline__ float value(Top a) { return max_nan(__low2float(a), __high2float(a)); }
  static __device__ __forceinline__ Top limit(float x) { return __bfloat162bfloat162(__float2bfloat16_ru(x)); }
  static __device__ __forceinline__ bool reaches(Top a, Top least) { return __hgeu2_mask(a, least) != 0; }
};

// ---- sums of exponentials ---------------------------------------------------------------------------------
// Largest value so far, and the sum of 2^(c (x - base)) where base is the largest value, or 0 as long as that is infinite: a sum
// over -infinity alone is 0, one with infinity infinite, one with a NaN a NaN.  Differences are formed before the product
// with c: those of the terms that make up the sum are small, and no product overflows that matters.
struct Running {
  float m = kMinusInf, z = 0.0f;
  __device__ __forceinline__ float base() const { return fabsf(m) == -kMinusInf ? 0.0f : m; }
  __device__ __forceinline__ void raise(float to, float c) {
    if (to > m) {
      const float f = m == kMinusInf || to == -kMinusInf ? 0.0f : ex2((m - to) * c);
      z *= f, m = to;
    }
  }
  __device__ __forceinline__ float term(float x, float c) const { return ex2((x - base()) * c); }
};
// the N terms of a piece, added in pairs
template <typename T>
__device__ __forceinline__ float terms(const Piece<T>& p, float base, float c) {
  const Two bb = two(-base, -base), cc = two(c, c);
  Two sum = 0;
#pragma unroll
  for (uint32_t i = 0; i < Piece<T>::N / 2; ++i) {
    const float2 y = each(mul2(add2(pair_of(p, i), bb), cc));
    const Two t = two(ex2(y.x), ex2(y.y));
    sum = i ? add2(sum, t) : t;
  }
  const float2 s = each(sum);
  return s.x + s.y;
}

// order of numbers as that of integers (no NaN)
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i ^ (i >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i ^ (i >> 31 & 0x7fffffff)); }
// over `lanes` lanes (a power of two) that begin at a multiple of it; the same in all of them
__device__ __forceinline__ Running warp_merge(Running a, float c, int lanes = 32) {
  // (over all lanes: those beyond hold parts of the same sum)
  a.raise(from_ordered(__reduce_max_sync(0xffffffffu, ordered(a.m))), c);
  for (int s = lanes / 2; s >= 1; s /= 2) a.z += __shfl_xor_sync(0xffffffffu, a.z, s);
  return a;
}
// over the block, the same in every thread; `sh`: a slot per warp
template <int THREADS>
__device__ __forceinline__ Running block_merge(Running a, float c, Running* sh) {
  constexpr int kWarps = THREADS / 32;
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
  }
  __syncwarp();
  return warp_merge(a, c, kMaxBlocks);
}
#endif

// Blocks that share a row: as many as leave no SM without work, while each has a few pieces per thread; long parts are worth
// having as many as are resident (loss and gradient of 249 x 75587 fp32 57 and 49 us, 300 x 128256 bf16 54 and 46; but 200 x 32000
// bf16 11.3 and 13.9).
inline uint32_t row_blocks(int64_t rows, int64_t row_bytes, int sm_count) {
  uint32_t c = 1;
  while (c < (uint32_t)kMaxBlocks && row_bytes / (c * 2) >= 2 * kWide * 16 &&
         rows * c * 2 <= (row_bytes / (c * 2) >= 64 * 1024 ? kResident : 2) * (int64_t)sm_count)
    c *= 2;
  return c;
}
// many of at most 16 KB
inline bool short_rows(int64_t rows, int64_t row_bytes, int sm_count) { return row_bytes <= kNarrow * 16 * 16 && rows >= 4 * (int64_t)sm_count; }

}  // namespace distill

cudaError_t launch_distill_top(const void* logits, int32_t dtype, int64_t ld, int64_t rows, int32_t vocab, int32_t k,
                               float temperature, int32_t* top_idx, float* top_logit, float* lse, int sm_count,
                               cudaStream_t stream);
cudaError_t launch_distill_loss(const pvt_distill& d, float* loss, float* stats, const float* upstream, void* grad,
                                int32_t grad_dtype, int64_t ldg, uint32_t* status, int sm_count, cudaStream_t stream);
cudaError_t launch_distill_grad(const pvt_distill& d, const float* stats, const float* upstream, void* grad, int32_t grad_dtype,
                                int64_t ldg, uint32_t* status, int sm_count, cudaStream_t stream);

}  // namespace pvt
