// The k largest logits of each row, in order, and the logarithm of the sum of all exponentials.
//
// One pass over the row keeps, besides the running sum, the largest value of each of 2048 parts of it, eight per thread.  Every
// warp takes the j-th largest of its maxima (of a thread's largest, for k up to 128), j = ceil(k / warps), and at least k
// elements reach the smallest of these, so everything that is listed is among the elements that do; with parts in no relation
// to the values those are not many more.  (The k-th largest of the block's 256 would leave fewer, 74 for k = 64, but one
// warp finds it while the others wait.)  The pieces of the parts that reach it, 16 bytes each, are looked at once more, and
// their candidates are put in order in shared memory.  (With a second pass over the whole row,
// which the L2 served, 64 / 257 largest of 4096 x 32000 bf16 took 87 / 148 us, not 78 / 133.)  A row in which too many elements reach the bound (equal ones, or a
// list nearly as long as the parts are many) is settled by counting the digits of its keys instead.  A few long rows are
// shared by clusters: each block lists its part, and an entry's place is its own plus those that the other blocks' lists
// hold ahead of it.
// 4096 x 32000 bf16 are 40 us of HBM; the bound is the issue slots, 73 % used by six blocks per SM.
#include "pvt_distill.cuh"

namespace pvt {
namespace {

using namespace distill;
using namespace mma;

constexpr uint32_t kParts = 8;      // of each thread: runs of its pieces
constexpr uint32_t kLowest = 0x007fffffu;  // key of -infinity

// Order of the list: larger keys first; NaN above all, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key >> 31 ? key ^ 0x80000000u : ~key); }
// ascending: larger key first, then lower index
__device__ __forceinline__ uint64_t entry_of(uint32_t key, uint32_t at) { return (uint64_t)(~key) << 32 | at; }

struct TopParams {
  const void* logits;
  int64_t ld;
  uint32_t vocab, k, blocks;
  float c;            // log2(e) / temperature
  float inv_t;
  int32_t* top_idx;
  float* top_logit;
  float* lse;
};

constexpr int kResidentFew = 6;  // blocks per SM where lists are short

// Few: lists of up to half as many as there are threads; many: longer ones, up to kMost
template <int THREADS>
constexpr uint32_t kMost = THREADS == kWide ? PVT_DISTILL_MAX_K : 2 * THREADS;
template <bool MANY, int THREADS>
struct TopShared {
  static constexpr int kThreads = THREADS, kWarps = THREADS / 32;
  static constexpr uint32_t kCandidates = MANY ? 8 * THREADS : THREADS == kWide ? 512 : 256;  // that are put in order at once
  static constexpr uint32_t kSorted = MANY ? kMost<THREADS> : THREADS;
  Running run[kWarps];
  Running mine;
  uint32_t bound[kWarps];
  uint32_t hist[256];
  uint32_t digit, above, count, n;
  uint32_t first[kThreads + 1];                  // place of a bucket's first entry
  uint32_t part[kParts * kThreads];              // largest elements of a part, a Top
  alignas(8) uint64_t entries[kCandidates];
  union {
    uint64_t by_bucket[kCandidates];
    uint16_t reached[kParts * kThreads];         // parts that may hold candidates
  };
  uint64_t sorted[kSorted];
};

// The digit (8 bits) in which the `want`-th largest key falls, and how many keys have larger digits: hist[d] holds the number of
// keys with digit d.  If there are fewer than `want` keys the digit is 0.
template <typename Shared>
__device__ __forceinline__ void find_digit(Shared& sm, uint32_t want) {
  if (threadIdx.x < 32) {
    const uint32_t lane = threadIdx.x;
    uint32_t own[8], sum = 0;  // digits 255 - 8 lane downwards
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += own[i] = sm.hist[255 - 8 * lane - i];
    uint32_t before = sum;
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
      const uint32_t o = __shfl_up_sync(0xffffffffu, before, s);
      if (lane >= s) before += o;
    }
    const uint32_t total = __shfl_sync(0xffffffffu, before, 31);
    before -= sum;
    if (before < want && want <= before + sum) {
      int i = 0;
      while (before + own[i] < want) before += own[i++];
      sm.digit = 255 - 8 * lane - i;
      sm.above = before;
    }
    if (lane == 0 && total < want) sm.digit = 0, sm.above = total - sm.hist[0];
  }
  __syncthreads();
}

template <int kThreads, typename T, typename F>
__device__ __forceinline__ void for_each(const T* row, const RowShare<T>& s, F f) {
  for (uint32_t i = s.lo + threadIdx.x; i < s.hi; i += kThreads) {
    const Piece<T> p = *reinterpret_cast<const Piece<T>*>(row + s.head + i * Piece<T>::N);
#pragma unroll
    for (uint32_t e = 0; e < Piece<T>::N; ++e) f(key_of(widen<T>(p.v[e])), s.head + i * Piece<T>::N + e);
  }
  if (threadIdx.x < s.loose()) {
    const uint32_t at = s.loose_at(threadIdx.x);
    f(key_of(widen<T>(row[at])), at);
  }
}

// n entries (at most kCandidates) in order; the first min(n, k) to sm.sorted.  Keys from `most` (or above) down to `least` fall
// into as many buckets as there are threads, in proportion; an entry's place is its bucket's first, and the number of those
// ahead of it in the bucket.  (300 / 1400 entries of a row among 4096: 16 / 75 us of a block's time by bitonic sort.)  Where
// many keys are (nearly) equal buckets are long, and a bitonic sort takes over; its steps of up to 32 stay within the 64
// entries of a warp.
template <typename Shared>
__device__ __forceinline__ void put_in_order(Shared& sm, uint32_t n, uint32_t k, uint32_t most, uint32_t least) {
  constexpr uint32_t kThreads = Shared::kThreads;
  constexpr uint32_t kLongBucket = 64;
  const uint32_t tid = threadIdx.x, lane = tid & 31;
  const float scale = (float)kThreads / ((float)(most - least) + 1.0f);
  auto bucket_of = [&](uint64_t entry) {
    const uint32_t key = ~(uint32_t)(entry >> 32);
    return key >= most ? 0u : min((uint32_t)((float)(most - key) * scale), (uint32_t)kThreads - 1);
  };
  sm.hist[tid] = 0;
  __syncthreads();
  for (uint32_t i = tid; i < n; i += kThreads) atomicAdd(&sm.hist[bucket_of(sm.entries[i])], 1u);
  __syncthreads();
  const uint32_t own = sm.hist[tid];
  uint32_t before = own;
#pragma unroll
  for (uint32_t s = 1; s < 32; s *= 2) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, before, s);
    if (lane >= s) before += o;
  }
  if (lane == 31) sm.bound[tid / 32] = before;
  const bool long_bucket = __syncthreads_or(own > kLongBucket);
  if (!long_bucket) {
    for (uint32_t w = 0; w < tid / 32; ++w) before += sm.bound[w];
    sm.first[tid] = before - own;
    sm.hist[tid] = before - own;
    if (tid == kThreads - 1) sm.first[kThreads] = n;
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kThreads) {
      const uint64_t entry = sm.entries[i];
      sm.by_bucket[atomicAdd(&sm.hist[bucket_of(entry)], 1u)] = entry;
    }
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kThreads) {
      const uint64_t entry = sm.by_bucket[i];
      const uint32_t bucket = bucket_of(entry), end = sm.first[bucket + 1];
      uint32_t place = sm.first[bucket];
      if (place >= k) continue;
      const uint32_t begin = place;
      for (uint32_t j = begin; j < end; ++j) place += sm.by_bucket[j] < entry;
      if (place < k) sm.sorted[place] = entry;
    }
  } else {
    uint32_t size = kThreads;
    while (size < n) size *= 2;
    for (uint32_t i = n + tid; i < size; i += kThreads) sm.entries[i] = ~0ull;
    __syncthreads();
    for (uint32_t run = 2; run <= size; run *= 2)
      for (uint32_t step = run / 2; step > 0; step /= 2) {
        for (uint32_t i = tid; i < size / 2; i += kThreads) {
          const uint32_t a = 2 * i - (i & (step - 1)), b = a + step;
          const uint64_t x = sm.entries[a], y = sm.entries[b];
          if ((x > y) == ((a & run) == 0)) sm.entries[a] = y, sm.entries[b] = x;
        }
        if (step > 32 || (step == 1 && run > 32))
          __syncthreads();
        else
          __syncwarp();
      }
    __syncthreads();
    for (uint32_t i = tid; i < min(n, k); i += kThreads) sm.sorted[i] = sm.entries[i];
  }
  __syncthreads();
}

// The same for a row whose candidates are too many: the k-th largest key by its digits, every larger one, and of its equals those
// with the lowest indices.
template <typename T, typename Shared>
__device__ __noinline__ uint32_t by_digits(Shared& sm, const T* row, const RowShare<T>& s, uint32_t k) {
  constexpr uint32_t kThreads = Shared::kThreads;
  uint32_t prefix = 0, want = k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (uint32_t i = threadIdx.x; i < 256; i += kThreads) sm.hist[i] = 0;
    __syncthreads();
    const uint32_t above = shift == 24 ? 0 : prefix >> (shift + 8);
    for_each<kThreads>(row, s, [&](uint32_t key, uint32_t) {
      if (key > kLowest && (shift == 24 || key >> (shift + 8) == above)) atomicAdd(&sm.hist[key >> shift & 255], 1u);
    });
    __syncthreads();
    find_digit(sm, want);
    prefix |= sm.digit << shift;
    want -= sm.above;
    __syncthreads();
  }
  // `want` of those equal to prefix (more than kCandidates elements reach the bound, so k exist above -infinity)
  if (threadIdx.x == 0) sm.count = 0;
  __syncthreads();
  for_each<kThreads>(row, s, [&](uint32_t key, uint32_t at) {
    if (key > prefix) sm.entries[atomicAdd(&sm.count, 1u)] = entry_of(key, at);
  });
  __syncthreads();
  const uint32_t larger = sm.count;
  uint32_t found = 0;
  for (uint32_t at0 = s.from(); at0 < s.to() && found < want; at0 += kThreads) {
    const uint32_t at = at0 + threadIdx.x;
    const bool equal = at < s.to() && key_of(widen<T>(row[at])) == prefix;
    const uint32_t ballot = __ballot_sync(0xffffffffu, equal);
    if ((threadIdx.x & 31) == 0) sm.hist[threadIdx.x / 32] = __popc(ballot);
    __syncthreads();
    uint32_t before = found, all = found;
    for (uint32_t w = 0; w < kThreads / 32; ++w) {
      if (w < threadIdx.x / 32) before += sm.hist[w];
      all += sm.hist[w];
    }
    before += __popc(ballot & ((1u << (threadIdx.x & 31)) - 1));
    if (equal && before < want) sm.entries[larger + before] = entry_of(prefix, at);
    found = all;
    __syncthreads();
  }
  put_in_order(sm, k, k, 0xffffffffu, prefix);
  return k;
}

// the upper half of the j-th largest of the warp's keys (PARTS in each lane), with zeros below
template <uint32_t PARTS>
__device__ __forceinline__ uint32_t warp_bound(const uint32_t* key, uint32_t j) {
  uint32_t bound = 0;  // at least j keys reach it
#pragma unroll
  for (uint32_t bit = 1u << 31; bit >= 1u << 16; bit /= 2) {
    uint32_t n = 0;
#pragma unroll
    for (uint32_t u = 0; u < PARTS; ++u) n += key[u] >= (bound | bit);
    n = PARTS == 1 ? __popc(__ballot_sync(0xffffffffu, n)) : __reduce_add_sync(0xffffffffu, n);
    if (n >= j) bound |= bit;
  }
  return bound;
}

template <typename T, bool MANY, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS != kWide ? kResidentNarrow : MANY ? kResident : kResidentFew)
    distill_top_kernel(const TopParams p) {
  extern __shared__ __align__(16) unsigned char raw[];
  using Shared = TopShared<MANY, THREADS>;
  constexpr uint32_t kThreads = THREADS, kWarps = THREADS / 32;
  Shared& sm = *reinterpret_cast<Shared*>(raw);
  pdl_trigger();
  pdl_wait();
  using Top = Tops<T>;
  constexpr uint32_t N = Piece<T>::N, UNROLL = 4;
  const uint32_t tid = threadIdx.x, rank = blockIdx.x % p.blocks, r = blockIdx.x / p.blocks, k = p.k;
  const T* row = static_cast<const T*>(p.logits) + (int64_t)r * p.ld;
  const RowShare<T> s(row, p.vocab, rank, p.blocks);
  const Piece<T>* const pieces = reinterpret_cast<const Piece<T>*>(row + s.head);

  // A thread's pieces are s.lo + tid + n kThreads; its part e are those with n >> lg = e.
  uint32_t lg = 0;
  while ((kParts << lg) * kThreads < s.hi - s.lo) ++lg;
  typename Top::Top* const part = reinterpret_cast<typename Top::Top*>(sm.part) + tid;
  Running run;
  uint32_t n = 0;
  auto keep = [&](typename Top::Top m) {
    typename Top::Top* const of = part + (n >> lg) * kThreads;
    *of = n & ((1u << lg) - 1) ? Top::max(*of, m) : m;
  };
  uint32_t i0 = s.lo + tid;
  for (; i0 + (UNROLL - 1) * kThreads < s.hi; i0 += UNROLL * kThreads, n += UNROLL) {
    Piece<T> piece[UNROLL];
#pragma unroll
    for (uint32_t u = 0; u < UNROLL; ++u) piece[u] = pieces[i0 + u * kThreads];
    typename Top::Top m[UNROLL];
#pragma unroll
    for (uint32_t u = 0; u < UNROLL; ++u) m[u] = Top::of(piece[u]);
    const auto low = Top::max(m[0], m[1]), high = Top::max(m[2], m[3]), top = Top::max(low, high);
    if (lg >= 2) {
      keep(top);
    } else if (lg == 1) {
      part[n / 2 * kThreads] = low, part[(n / 2 + 1) * kThreads] = high;
    } else {
#pragma unroll
      for (uint32_t u = 0; u < UNROLL; ++u) part[(n + u) * kThreads] = m[u];
    }
    run.raise(Top::value(top), p.c);
#pragma unroll
    for (uint32_t u = 0; u < UNROLL; ++u) run.z += terms(piece[u], run.base(), p.c);
  }
  for (; i0 < s.hi; i0 += kThreads, ++n) {
    const Piece<T> piece = pieces[i0];
    const auto m = Top::of(piece);
    keep(m);
    run.raise(Top::value(m), p.c);
    run.z += terms(piece, run.base(), p.c);
  }
  const uint32_t parts = (n + (1u << lg) - 1) >> lg;  // of this thread
  float loose = kMinusInf;
  if (tid < s.loose()) {
    loose = widen<T>(row[s.loose_at(tid)]);
    run.raise(loose, p.c);
    run.z += run.term(loose, p.c);
  }
  if (tid == 0) sm.count = sm.digit = 0;
  uint32_t bound;
  if (MANY) {
    uint32_t key[kParts];
#pragma unroll
    for (uint32_t e = 0; e < kParts; ++e)
      key[e] = key_of(max_nan(e < parts ? Top::value(part[e * kThreads]) : kMinusInf, e ? kMinusInf : loose));
    bound = warp_bound<kParts>(key, (k + kWarps - 1) / kWarps);
  } else {
    auto all = Top::lowest();
    for (uint32_t e = 0; e < parts; ++e) all = Top::max(all, part[e * kThreads]);
    const uint32_t key = key_of(max_nan(Top::value(all), loose));
    bound = warp_bound<1>(&key, (k + kWarps - 1) / kWarps);
  }
  if (tid % 32 == 0) sm.bound[tid / 32] = bound;
  run = block_merge<THREADS>(run, p.c, sm.run);
  bound = __reduce_min_sync(0xffffffffu, sm.bound[tid % kWarps]);
  if (tid == 0) sm.mine = run;
  // what is below reaches no place of the list; -infinity never does
  bound = max(bound, kLowest + 1);
  const float least = value_of(bound);
  const auto limit = Top::limit(least);
  for (uint32_t e = 0; e < parts; ++e)
    if (Top::reaches(part[e * kThreads], limit)) sm.reached[atomicAdd(&sm.digit, 1u)] = (uint16_t)(e * kThreads + tid);
  __syncthreads();
  // their pieces, one to a thread
  constexpr uint32_t kCandidates = Shared::kCandidates, AT_ONCE = MANY ? 4 : 1;
  const uint32_t reached = sm.digit << lg;
  for (uint32_t j0 = tid; j0 < reached; j0 += AT_ONCE * kThreads) {
    uint32_t i[AT_ONCE];
    Piece<T> piece[AT_ONCE];
#pragma unroll
    for (uint32_t u = 0; u < AT_ONCE; ++u) {
      const uint32_t j = j0 + u * kThreads, which = j < reached ? sm.reached[j >> lg] : 0;
      i[u] = s.lo + which % kThreads + ((which / kThreads << lg) + (j & ((1u << lg) - 1))) * kThreads;
      if (j >= reached || i[u] >= s.hi) i[u] = ~0u;
      if (i[u] != ~0u) piece[u] = pieces[i[u]];
    }
#pragma unroll
    for (uint32_t u = 0; u < AT_ONCE; ++u) {
      if (i[u] == ~0u || !Top::reaches(Top::of(piece[u]), limit)) continue;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        const float x = widen<T>(piece[u].v[e]);
        if (x < least) continue;
        const uint32_t place = atomicAdd(&sm.count, 1u);
        if (place < kCandidates) sm.entries[place] = entry_of(key_of(x), s.head + i[u] * N + e);
      }
    }
  }
  if (tid < s.loose()) {
    const float x = widen<T>(row[s.loose_at(tid)]);
    if (!(x < least)) {
      const uint32_t place = atomicAdd(&sm.count, 1u);
      if (place < kCandidates) sm.entries[place] = entry_of(key_of(x), s.loose_at(tid));
    }
  }
  __syncthreads();
  const uint32_t found = sm.count;
  n = min(found, k);
  if (found <= kCandidates)
    put_in_order(sm, found, k, key_of(run.m), bound);
  else
    n = by_digits(sm, row, s, k);

  int32_t* idx = p.top_idx + (int64_t)r * k;
  float* val = p.top_logit + (int64_t)r * k;
  auto put = [&](uint32_t place, uint64_t entry) {
    idx[place] = (int32_t)(uint32_t)entry;
    val[place] = value_of(~(uint32_t)(entry >> 32));
  };
  uint32_t total = n;
  if (p.blocks == 1) {
    for (uint32_t i = tid; i < n; i += kThreads) put(i, sm.sorted[i]);
  } else {
    if (tid == 0) sm.n = n;
    cluster_sync();
    run = cluster_merge(&sm.mine, p.blocks, p.c);
    // the other blocks' lists, side by side, behind this block's own memory
    uint64_t* lists = reinterpret_cast<uint64_t*>(raw + sizeof(Shared));
    uint32_t size[kMaxBlocks];
#pragma unroll
    for (uint32_t q = 0; q < kMaxBlocks; ++q)
      size[q] = q < p.blocks ? __float_as_uint(cluster_load(smem_u32(&sm.n), q)) : 0;
    for (uint32_t i = tid; i < k; i += kThreads) {
      uint64_t entry[kMaxBlocks];
#pragma unroll
      for (uint32_t q = 0; q < kMaxBlocks; ++q)
        if (i < size[q]) entry[q] = cluster_load64(smem_u32(sm.sorted + i), q);
#pragma unroll
      for (uint32_t q = 0; q < kMaxBlocks; ++q)
        if (i < size[q]) lists[q * k + i] = entry[q];
    }
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kThreads) {
      // how many of every list come ahead of it (of its own: i), all lists at once: 257 entries of 24 blocks 12100 cycles
      // list by list
      const uint64_t own = sm.sorted[i];
      uint32_t ahead[kMaxBlocks] = {};
      for (uint32_t by = 1u << (31 - __clz(k)); by; by /= 2)
#pragma unroll
        for (uint32_t q = 0; q < kMaxBlocks; ++q) {
          const uint32_t to = ahead[q] + by;
          if (to <= size[q] && lists[q * k + to - 1] < own) ahead[q] = to;
        }
      uint32_t place = 0;
#pragma unroll
      for (uint32_t q = 0; q < kMaxBlocks; ++q) place += ahead[q];
      if (place < k) put(place, own);
    }
    total = 0;
#pragma unroll
    for (uint32_t q = 0; q < kMaxBlocks; ++q) total += size[q];
    cluster_sync();  // no block leaves while another reads its lists
  }
  if (rank == 0) {
    for (uint32_t i = total + tid; i < k; i += kThreads) {
      idx[i] = -1;
      val[i] = kMinusInf;
    }
    if (tid == 0 && p.lse)
      p.lse[r] = run.base() * p.inv_t + logf(run.z);
  }
}

template <typename T, bool MANY, int THREADS>
cudaError_t top(const TopParams& p, int64_t rows, cudaStream_t stream) {
  const cudaError_t e = allow_smem<distill_top_kernel<T, MANY, THREADS>>();
  if (e != cudaSuccess) return e;
  const size_t smem = sizeof(TopShared<MANY, THREADS>) + (p.blocks > 1 ? (size_t)p.blocks * p.k * 8 : 0);
  return launch_clusters(distill_top_kernel<T, MANY, THREADS>, (unsigned)(rows * p.blocks), p.blocks, THREADS, smem, stream, p);
}
template <typename T, int THREADS>
cudaError_t top(const TopParams& p, int64_t rows, cudaStream_t stream) {
  return p.k <= (uint32_t)THREADS / 2 ? top<T, false, THREADS>(p, rows, stream) : top<T, true, THREADS>(p, rows, stream);
}
template <typename T>
cudaError_t top(const TopParams& p, int64_t rows, int sm_count, cudaStream_t stream) {
  return p.k <= kMost<kNarrow> && short_rows(rows, (int64_t)p.vocab * sizeof(T), sm_count) ? top<T, kNarrow>(p, rows, stream)
                                                                                            : top<T, kWide>(p, rows, stream);
}

}  // namespace

cudaError_t launch_distill_top(const void* logits, int32_t dtype, int64_t ld, int64_t rows, int32_t vocab, int32_t k,
                               float temperature, int32_t* top_idx, float* top_logit, float* lse, int sm_count,
                               cudaStream_t stream) {
  TopParams p = {};
  p.logits = logits, p.ld = ld, p.vocab = (uint32_t)vocab, p.k = (uint32_t)k;
  p.c = (float)(1.4426950408889634 / (double)temperature), p.inv_t = (float)(1.0 / (double)temperature);
  p.top_idx = top_idx, p.top_logit = top_logit, p.lse = lse;
  p.blocks = row_blocks(rows, (int64_t)vocab * (dtype == PVT_F32 ? 4 : 2), sm_count);
  if (rows * p.blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  timing_begin(kKernDistill, stream);
  const cudaError_t e = dtype == PVT_F32   ? top<float>(p, rows, sm_count, stream)
                        : dtype == PVT_F16 ? top<__half>(p, rows, sm_count, stream)
                                           : top<__nv_bfloat16>(p, rows, sm_count, stream);
  timing_end(kKernDistill, stream);
  count_launches(1);
  return e;
}

}  // namespace pvt
