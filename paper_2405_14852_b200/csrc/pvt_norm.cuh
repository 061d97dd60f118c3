// What the two directions of the norm share: how rows are spread over threads, their way in through shared memory, types known at
// run time.
//
// A row's columns are spans of 256; a warp has one or two of them, a lane eight elements of each: neighbouring ones where every row
// begins on eight elements' boundary (kWide; kExact if there is no place without an element either), otherwise (kRagged) 32
// apart, so that a warp's accesses run along the row.  What a
// thread does once for a row, sums and barriers, is a hundred instructions and more, so it wants elements enough; a thread has the same
// columns in every row and their weights in registers, which with four spans did not fit any more.  Rows of one span share a block's warps, and those of at most 64 or 128 columns may share a warp: a
// row is then a team of 8 or 16 lanes.  Rows of more than 8192 columns, or of more than fit a block's ring, are shared by a cluster of two,
// four or eight blocks.
//
// Blocks stay and take rows from a ring in shared memory that asynchronous copies fill one or two rows ahead: HBM needs some 40 KB on
// their way to each SM at any time, more than registers would hold beside a row at work.  Wide: a thread copies what it will read, in
// pieces of 16 bytes, and needs no one else.  Otherwise a row's image is copied by aligned pieces of 16 bytes, the first of which may
// begin with the end of what lies before the row, and the last of which is cut at the row's end; all threads wait for all copies.
#pragma once

#include <type_traits>

#include "pvt_mma.cuh"
#include "pvt_mx.cuh"

namespace pvt {
namespace norm {

constexpr uint32_t kSpanCols = 256, kMostWarps = 16, kMostGroups = 2, kMostParts = 8;
constexpr uint32_t kMostThreads = 32 * kMostWarps;
constexpr uint32_t kTeamThreads = 256;           // of a block where rows share it
constexpr uint32_t kRaggedBound = 640;           // threads that registers are for, so that two blocks of 320 fit an SM
constexpr uint32_t kRingBytes = 208 * 1024;      // that the blocks of an SM have for their rings
static_assert(kSpanCols * kMostWarps * kMostGroups * 4 >= PVT_NORM_MAX_COLS, "every row fits a cluster of four");

enum Layout { kRagged = 0, kWide = 1, kExact = 2 };

struct Shape {
  uint32_t rows, cols;
  uint32_t parts;   // blocks of a row
  uint32_t groups;  // spans of a warp
  uint32_t warps;   // of a row in a block
  uint32_t lanes;   // of a row, where one warp or less has it; 32 otherwise
  uint32_t teams;   // rows that a block has at a time
  uint32_t threads;
};
// `narrow`: a row may be less than a warp (wide layouts only); parts: blocks at least, a power of two
inline Shape shape_of(uint32_t rows, uint32_t cols, bool narrow, uint32_t parts = 1) {
  Shape s = {rows, cols, parts, 1, 1, 32, 1, 0};
  const uint32_t spans = (cols + kSpanCols - 1) / kSpanCols;
  while (spans > s.parts * kMostWarps * kMostGroups) s.parts *= 2;
  const uint32_t own = (spans + s.parts - 1) / s.parts;
  s.groups = own <= 4 ? 1 : 2;
  s.warps = (own + s.groups - 1) / s.groups;
  if (s.parts == 1 && spans == 1) {
    if (narrow && cols <= 128) s.lanes = cols <= 64 ? 8 : 16;
    s.teams = kTeamThreads / s.lanes;
  }
  s.threads = s.teams > 1 ? kTeamThreads : 32 * s.warps;
  return s;
}
// bytes of a row's image in shared memory: of a thread's elements for each, or of the block's part of a row from any boundary on
inline uint32_t image_bytes(const Shape& s, uint32_t size, bool wide) {
  if (wide) return s.threads / s.teams * s.groups * 8 * size;
  const uint32_t most = s.groups * s.warps * kSpanCols, part = most < s.cols ? most : s.cols;
  return (part * size + 15 + 15) / 16 * 16;
}
// Blocks or clusters that are resident at once, of `bytes` of shared memory and `regs` registers to a thread.  (Not every SM finds others
// for a cluster of four or eight.)
inline uint32_t resident_sets(const Shape& s, size_t bytes, int regs, int sm_count) {
  uint32_t per_sm = 65536 / (uint32_t)((regs < 64 ? 64 : (regs + 7) / 8 * 8) * s.threads);
  if (per_sm * bytes > kRingBytes) per_sm = (uint32_t)(kRingBytes / bytes);
  if (per_sm < 1) per_sm = 1;
  const uint32_t sms = (uint32_t)sm_count * (s.parts == 8 ? 5 : s.parts == 4 ? 7 : 8) / 8;
  const uint32_t n = sms * per_sm / s.parts;
  return n > 0 ? n : 1;
}
#ifdef __CUDACC__
// registers of a kernel, which is set up for large shared memory at the same time; the driver is asked once per kernel and device
template <auto kernel>
cudaError_t set_up(int* regs) {
  static std::atomic<int> known[kMaxDevices];
  const int dev = device_slot();
  *regs = dev >= 0 ? known[dev].load(std::memory_order_relaxed) : 0;
  if (*regs > 0) return cudaSuccess;
  cudaError_t e = allow_smem<kernel>();
  cudaFuncAttributes fa;
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, kernel);
  if (e != cudaSuccess) return e;
  *regs = fa.numRegs;
  if (dev >= 0) known[dev].store(fa.numRegs, std::memory_order_relaxed);
  return cudaSuccess;
}
#endif

cudaError_t launch_apply(const pvt_norm& n, void* total, int64_t ldt, void* y, int32_t y_dtype, int64_t ldy, const pvt_mx* yq,
                         float* stats, int sm_count, cudaStream_t stream);
size_t grad_workspace_bytes(int64_t rows, int32_t cols, int sm_count);
cudaError_t launch_grad(const pvt_norm& n, const float* stats, int32_t dtype, const void* dy, int64_t lddy, const void* dres,
                        int64_t lddr, void* dx, int64_t lddx, void* dweight, void* dbias, int32_t dw_dtype, bool accumulate, void* ws,
                        int sm_count, cudaStream_t stream);

inline Layout layout_of(const Shape& s, bool wide) {
  return !wide ? kRagged : s.teams == 1 && s.cols == s.parts * s.warps * s.groups * kSpanCols ? kExact : kWide;
}
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
using mx::add2;
using mx::both;
using mx::Eight;
using mx::fma2;
using mx::mul2;
using mx::narrow;
using mx::set2;
using mx::two;
using mx::widen;

// 16 bytes from a 16-byte boundary, of which the first `bytes` are read and the others become 0
__device__ __forceinline__ void copy16(uint32_t to, const void* from, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// all groups but the last one, or all, have landed (for the thread that asked for them)
__device__ __forceinline__ void copies_wait(bool but_one) {
  if (but_one)
    asm volatile("cp.async.wait_group 1;" ::: "memory");
  else
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}
// (short chains: with few warps to an SM their latency would show)
__device__ __forceinline__ float sum8(const float* v) {
  const float2 s = add2(add2(two(v), two(v + 2)), add2(two(v + 4), two(v + 6)));
  return s.x + s.y;
}
__device__ __forceinline__ float dot8(const float* a, const float* b) {
  const float2 s = add2(fma2(two(a + 2), two(b + 2), mul2(two(a), two(b))), fma2(two(a + 6), two(b + 6), mul2(two(a + 4), two(b + 4))));
  return s.x + s.y;
}

// two values rounded at a time: one conversion, where one by itself takes the slower unit
__device__ __forceinline__ void narrow_pair(float a, float b, float* to) { to[0] = a, to[1] = b; }
__device__ __forceinline__ void narrow_pair(float a, float b, __half* to) {
  const __half2 v = __floats2half2_rn(a, b);
  to[0] = v.x, to[1] = v.y;
}
__device__ __forceinline__ void narrow_pair(float a, float b, __nv_bfloat16* to) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  to[0] = v.x, to[1] = v.y;
}
// 1 / sqrt(v), v > 0: the approximation (2^-22.9) and one step of Newton's; 0 if v is infinite
__device__ __forceinline__ float inverse_root(float v) {
  const float r = rsqrtf(v);
  return r > 0.0f ? fmaf(0.5f * r, fmaf(-v * r, r, 1.0f), r) : r;
}

// A thread's place among the rows.  G: spans of a warp
template <int L, int G>
struct Place {
  static constexpr bool WIDE = L != kRagged;
  uint32_t lane, warp, team, in_team, team_threads;
  uint32_t c0, next;        // its first column, and from one span to the next
  static constexpr uint32_t step = WIDE ? 1 : 32;  // from one element to the next
  uint32_t part0, end;      // the block's columns
  __device__ __forceinline__ Place(const Shape& s, uint32_t rank) {
    const uint32_t tid = threadIdx.x;
    lane = tid & 31, warp = tid >> 5;
    team_threads = s.teams > 1 ? s.lanes : s.threads;
    team = s.teams > 1 ? tid / s.lanes : 0, in_team = s.teams > 1 ? tid & (s.lanes - 1) : tid;
    part0 = rank * s.warps * G * kSpanCols;
    end = min(s.cols, part0 + s.warps * G * kSpanCols);
    next = s.warps * kSpanCols;
    c0 = part0 + (WIDE ? 8 * in_team : in_team / 32 * kSpanCols + (in_team & 31));
  }
  __device__ __forceinline__ uint32_t col(int g) const { return c0 + g * next; }
  __device__ __forceinline__ bool has(int g, int i) const { return L == kExact || col(g) + i * step < end; }
  __device__ __forceinline__ bool full(int g) const { return L == kExact || col(g) + 7 * step < end; }
  // f(i) for the elements that exist
  template <typename F>
  __device__ __forceinline__ void each(int g, F f) const {
    if (full(g)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f(i);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (has(g, i)) f(i);
    }
  }

  // asks for the team's row, if there is one
  template <typename T>
  __device__ __forceinline__ void ask(uint32_t image, const T* from) const {
    constexpr uint32_t SIZE = sizeof(T), PIECES = 8 * SIZE / 16;
    if (WIDE) {
      const char* const own = reinterpret_cast<const char*>(from + c0);
      const uint32_t to = image + in_team * 16;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if (full(g)) {
#pragma unroll
          for (uint32_t k = 0; k < PIECES; ++k) copy16(to + (g * PIECES + k) * team_threads * 16, own + g * next * SIZE + 16 * k, 16);
        } else {
#pragma unroll
          for (uint32_t k = 0; k < PIECES; ++k) {
            const uint32_t bytes = col(g) < end ? (end - col(g)) * SIZE : 0, n = bytes > 16 * k ? min(16u, bytes - 16 * k) : 0;
            copy16(to + (g * PIECES + k) * team_threads * 16, n ? own + g * next * SIZE + 16 * k : reinterpret_cast<const char*>(from), n);
          }
        }
      }
    } else if (part0 < end) {
      const uint64_t last = reinterpret_cast<uint64_t>(from + end), from16 = reinterpret_cast<uint64_t>(from + part0) & ~15ull;
      const uint32_t bytes = (uint32_t)(last - from16);
      for (uint32_t k = 16 * in_team; k < bytes; k += 16 * team_threads)
        copy16(image + k, reinterpret_cast<const void*>(from16 + k), min(16u, bytes - k));
    }
  }
  // the thread's elements of that row, of one span; 0 behind its end
  template <typename T>
  __device__ __forceinline__ void take(const unsigned char* image, const T* from, int g, float* v) const {
    constexpr uint32_t SIZE = sizeof(T);
    if (WIDE) {
      const unsigned char* const own = image + (g * (8 * SIZE / 16) * team_threads + in_team) * 16;
      if (SIZE == 4) {
        const float4 a = *reinterpret_cast<const float4*>(own), b = *reinterpret_cast<const float4*>(own + team_threads * 16);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
      } else {
        const Eight<T> e = *reinterpret_cast<const Eight<T>*>(own);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = widen<T>(e.v[i]);
      }
    } else {
      const unsigned char* const own = image + ((uint32_t)reinterpret_cast<uint64_t>(from + part0) & 15u) + (col(g) - part0) * SIZE;
      if (!full(g)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
      }
      each(g, [&](int i) { v[i] = widen<T>(*reinterpret_cast<const T*>(own + i * step * SIZE)); });
    }
  }
  template <typename T>
  __device__ __forceinline__ void put(T* row, int g, const float* v) const {
    if (WIDE && full(g)) {
      Eight<T> e;
#pragma unroll
      for (int i = 0; i < 8; i += 2) narrow_pair(v[i], v[i + 1], &e.v[i]);
      *reinterpret_cast<Eight<T>*>(row + col(g)) = e;
    } else {
      each(g, [&](int i) { row[col(g) + i * step] = narrow<T>(v[i]); });
    }
  }
  // the weights of its columns, `other` where there are none; wide: eight of them begin on 16 bytes
  __device__ __forceinline__ void weights(const void* w, int32_t dtype, bool wide, float other, float (*v)[8]) const {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[g][i] = other;
    if (!w) return;
    with_type(dtype, [&](auto* type) {
      using U = std::remove_pointer_t<decltype(type)>;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const U* const from = static_cast<const U*>(w) + col(g);
        if (WIDE && wide && full(g)) {
          const Eight<U> e = *reinterpret_cast<const Eight<U>*>(from);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[g][i] = widen<U>(e.v[i]);
        } else {
          each(g, [&](int i) { v[g][i] = widen<U>(from[i * step]); });
        }
      }
    });
  }
};

// over the lanes of a team
__device__ __forceinline__ float team_sum(float v, uint32_t lanes) {
  if (lanes > 16) v += __shfl_xor_sync(0xffffffffu, v, 16);
  if (lanes > 8) v += __shfl_xor_sync(0xffffffffu, v, 8);
#pragma unroll
  for (int s = 4; s > 0; s /= 2) v += __shfl_xor_sync(0xffffffffu, v, s);
  return v;
}
// The same of two values: after the first exchange half of the lanes add up one of them, half the other.
__device__ __forceinline__ void warp_sums(float* v, uint32_t lane) {
  const bool upper = lane & 16;
  const float other = __shfl_xor_sync(0xffffffffu, upper ? v[0] : v[1], 16);
  float mine = (upper ? v[1] : v[0]) + other;
#pragma unroll
  for (int s = 8; s > 0; s /= 2) mine += __shfl_xor_sync(0xffffffffu, mine, s);
  v[0] = __shfl_sync(0xffffffffu, mine, 0), v[1] = __shfl_sync(0xffffffffu, mine, 16);
}
// N sums over all threads of a row, in all of its blocks, in two halves with a barrier of them all between (row_barrier): this one leaves
// a warp's sums in `slots` (shared, not in use by the sums before), or the whole row's in v where a warp has it.
template <int N>
__device__ __forceinline__ void sums_put(float* v, const Shape& s, uint32_t rank, float (*slots)[N]) {
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (N == 2 && s.lanes == 32) {
    warp_sums(v, lane);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = team_sum(v[k], s.lanes);
  }
  if (s.warps == 1 && s.parts == 1) return;
  if (s.parts == 1) {
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) slots[warp][k] = v[k];
    }
  } else if (lane < s.parts) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const uint32_t at = mma::cluster_address(m1::smem_u32(&slots[rank * s.warps + warp][k]), lane);
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v[k]) : "memory");
    }
  }
}
__device__ __forceinline__ void row_barrier(const Shape& s) {
  if (s.parts > 1)
    mma::cluster_sync();
  else if (s.warps > 1)
    __syncthreads();
  else
    __syncwarp();
}
template <int N>
__device__ __forceinline__ void sums_get(float* v, const Shape& s, const float (*slots)[N]) {
  if (s.warps == 1 && s.parts == 1) return;
  const uint32_t lane = threadIdx.x & 31;
  if (s.parts == 1) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lane % kMostWarps < s.warps ? slots[lane % kMostWarps][k] : 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int d = kMostWarps / 2; d > 0; d /= 2) v[k] += __shfl_xor_sync(0xffffffffu, v[k], d);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.0f;
    for (uint32_t i = lane; i < s.parts * s.warps; i += 32)
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += slots[i][k];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = team_sum(v[k], 32);
  }
}
template <int N>
__device__ __forceinline__ void row_sums(float* v, const Shape& s, uint32_t rank, float (*slots)[N]) {
  sums_put<N>(v, s, rank, slots);
  if (s.warps > 1 || s.parts > 1) row_barrier(s);
  sums_get<N>(v, s, slots);
}
#endif

}  // namespace norm
}  // namespace pvt
