// The distillation loss of a row and its gradient.
//
// The row is read once for its largest logit and the sum of exponentials relative to it and, for
// the gradient, a second time, which the L2 serves: with y = 2^(c (x - largest)) every unlisted logit gets y times one factor.
// The listed ones are overwritten after that.  What concerns the k listed entries alone, the teacher's probabilities and the loss, is
// computed in binary64, where the remaining mass 1 - sum p is a small difference too.  With that mass as one more outcome
// the pass sums what is not listed, told from the rest by one bit per entry of the vocabulary in shared memory, relative to the
// largest logit that is not listed (beside a listed one the sum could be 0 in binary32 although its logarithm is a number),
// and the listed exponentials are added in binary64: a sum of all less the listed ones would lose what a student near its
// teacher leaves to the rest, and its loss, a small difference of log sums, is as good as the two sums agree.
// A few long rows are shared by clusters of blocks.
// 4096 x 32000 bf16, loss and gradient in one pass: 102 us, 81 at the copy's rate.  Issue slots 64 % (two exponentials and a
// rounding per element), and about as much of the L2 as five blocks per SM may hold of rows between their two readings: six
// take 124 us.  With the remaining mass 110 us, issue slots 60 %.
#include "pvt_distill.cuh"

namespace pvt {
namespace {

using namespace distill;
using namespace mma;

constexpr int kUnroll = 4;  // pieces in flight per thread
constexpr uint32_t kAsked = 128 * 1024;  // bytes of a row that are asked for ahead

// A binary32 lse is off by its own rounding, 2^-24 of it, and by its sum's: roundings of the largest logit over the temperature (at
// most the lse and the logarithm of the sum, which is below 7 for a list's worth of entries), of the logarithm, and 40 2^-24 of
// the terms and their additions.  Together that is less than 2^-22 (18 + |lse|), and a probability as much of itself.
constexpr double kLseNoise = 1.0 / (1 << 22);
constexpr double kFewest = 1.0 / 1024;  // of the teacher's rest

enum { kLoss = 1, kGrad = 2, kBoth = 3 };

struct DistillParams {
  const void* logits;
  int64_t ld;
  uint32_t vocab, k, blocks;
  float c;          // log2(e) / temperature
  double inv_t;
  const int32_t* top_idx;
  const float* top_logit;
  const float* teacher_lse;
  const float* weight;
  const float* upstream;
  float* loss;
  float* stats;      // written with the loss, read for the gradient alone
  void* grad;
  int64_t ldg;
  uint32_t* status;
};

// stats of a row: largest logit, factor of y at the listed and at the other logits, logarithm of the teacher's sum in two parts, whether
// the row has any effect, what y at the other logits is relative to
enum { kStatMax = 0, kStatListed = 1, kStatRest = 2, kStatNorm = 3, kStatNormLow = 4, kStatActive = 5, kStatRestMax = 6 };

// What a warp has added up of the teacher's list: exponentials e = exp(a), a = logit / temperature - shift, and
// e (a - (x - near) / temperature), near the largest of the student's logits there (or 0 as long as that is infinite); with a
// remaining mass also exp((x - near) / temperature).  The shift is the row's, not the warp's: where e is 0 the student may have no mass, and an e that
// is 0 beside the row's largest must not be a number beside the warp's.
struct Teacher {
  double mass, cross, own;
  float near, most;  // (most: infinite too)
  uint32_t any;      // an entry above -infinity
};

template <int THREADS>
struct DistillShared {
  Running run[THREADS / 32];
  Running mine;
  Teacher teacher[THREADS / 32];
  float top[THREADS / 32];          // the teacher's largest listed logit, by warp
  uint32_t repeated;
  uint32_t next;                    // run of pieces of the gradient that no warp has taken yet
  float stat[PVT_DISTILL_STATS];
  // behind it, k each: the list's entries, -1 for those that are left out; the student's logits there; the teacher's
  __device__ __forceinline__ int32_t* idx() { return reinterpret_cast<int32_t*>(this + 1); }
  __device__ __forceinline__ float* x(uint32_t k) { return reinterpret_cast<float*>(this + 1) + k; }
  __device__ __forceinline__ float* val(uint32_t k) { return reinterpret_cast<float*>(this + 1) + 2 * k; }
};

// zeros over this block's share of the gradient
template <int THREADS, typename G>
__device__ __forceinline__ void clear(G* grad, uint32_t from, uint32_t to) {
  for (uint32_t i = from + threadIdx.x; i < to; i += THREADS) grad[i] = narrow<G>(0.0f);
}

template <typename T, typename G, int MODE, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == kWide ? kResident : kResidentNarrow) distill_kernel(const DistillParams p) {
  extern __shared__ __align__(16) unsigned char raw[];
  using Shared = DistillShared<THREADS>;
  Shared& sm = *reinterpret_cast<Shared*>(raw);
  // a bit per entry of the vocabulary, moved so that a piece's bits lie in one word: piece i has those from (i + 1) N on
  uint32_t* const listed = reinterpret_cast<uint32_t*>(raw + sizeof(Shared) + 12 * (size_t)p.k);
  pdl_trigger();
  pdl_wait();
  constexpr uint32_t N = Piece<T>::N;
  const uint32_t tid = threadIdx.x, rank = blockIdx.x % p.blocks, r = blockIdx.x / p.blocks, k = p.k;
  int32_t* const list_idx = sm.idx();
  float *const list_x = sm.x(k), *const list_val = sm.val(k);
  const T* row = static_cast<const T*>(p.logits) + (int64_t)r * p.ld;
  G* const grad = MODE & kGrad ? static_cast<G*>(p.grad) + (int64_t)r * p.ldg : nullptr;
  const RowShare<T> s(row, p.vocab, rank, p.blocks);
  const Piece<T>* const pieces = reinterpret_cast<const Piece<T>*>(row + s.head);
  // the row is on its way while the list is looked at (4096 x 32000 bf16: 106 us without, 101 with)
  if (tid == 0 && s.lo < s.hi) prefetch_l2(pieces + s.lo, min((s.hi - s.lo) * (uint32_t)sizeof(Piece<T>), kAsked));
  const bool tail = p.teacher_lse != nullptr;
  // everything that is fetched by itself is asked for at once
  const int32_t first_idx = tid < k ? p.top_idx[(int64_t)r * k + tid] : -1;
  const float first_val = tid < k ? p.top_logit[(int64_t)r * k + tid] : 0.0f;
  const float upstream = (MODE & kGrad) && p.upstream ? p.upstream[r] : 1.0f;
  const float lse = (MODE & kLoss) && tail ? p.teacher_lse[r] : 0.0f;
  const float weight = p.weight ? p.weight[r] : 1.0f;
  float* const stats = p.stats ? p.stats + (int64_t)r * PVT_DISTILL_STATS : nullptr;

  for (uint32_t i = tid; i < (p.vocab + N + 31) / 32; i += THREADS) listed[i] = 0;
  if (tid == 0) sm.next = 0, sm.repeated = 0;
  __syncthreads();
  // (the same in all blocks of the row: they leave together)
  bool active = weight != 0.0f;
  if (MODE == kGrad) active = active && stats[kStatActive] != 0.0f;

  // the list: entries outside the vocabulary or named before are left out
  T first_x = narrow<T>(0.0f);
  if (active) {
    bool bad = false;
    float top = kMinusInf;
    auto keep_top = [&] {
      top = from_ordered(__reduce_max_sync(0xffffffffu, ordered(top)));
      if (tid % 32 == 0) sm.top[tid / 32] = top;
    };
    for (uint32_t i = tid; i < k; i += THREADS) {
      int32_t at = i == tid ? first_idx : p.top_idx[(int64_t)r * k + i];
      if (at >= (int32_t)p.vocab) bad = true, at = -1;
      if (at >= 0) {
        const uint32_t bit = (uint32_t)at + N - s.head;
        if (atomicOr(&listed[bit / 32], 1u << (bit % 32)) >> (bit % 32) & 1u) sm.repeated = 1;
      }
      list_idx[i] = at < 0 ? -1 : at;
      const float val = i == tid ? first_val : p.top_logit[(int64_t)r * k + i];
      list_val[i] = val;
      if (at >= 0) top = fmaxf(top, val);  // (a NaN shows in the sums)
      // before any block writes the gradient over the logits; a thread's first is looked at after the pass over the row
      if (i != tid)
        list_x[i] = at >= 0 ? widen<T>(row[at]) : 0.0f;
      else if (at >= 0)
        first_x = row[at];
    }
    if (MODE & kLoss) keep_top();
    __syncthreads();
    if (sm.repeated) {
      uint32_t again = 0;  // of this thread's entries
      top = kMinusInf;
      for (uint32_t i = tid, n = 0; i < k; i += THREADS, ++n)
        for (uint32_t j = 0; j < i; ++j)
          if (list_idx[i] >= 0 && list_idx[j] == list_idx[i]) again |= 1u << n;
      __syncthreads();
      for (uint32_t i = tid, n = 0; i < k; i += THREADS, ++n)
        if (again >> n & 1u)
          list_idx[i] = -1, bad = true;
        else if (list_idx[i] >= 0)
          top = fmaxf(top, list_val[i]);
      if (MODE & kLoss) keep_top();
      __syncthreads();
    }
    if (bad && p.status) atomicOr(p.status, PVT_DEV_BAD_INDEX);
  }

  float m = 0.0f, f_rest = 0.0f;  // what y of what is not listed is relative to, and its factor
  if (MODE & kLoss) {
    Running run;
    double shift = lse;
    if (active) {
      using Top = Tops<T>;
      // With a remaining mass listed elements of piece i become -infinity, which add nothing and raise nothing.
      auto leave_out = [&](Piece<T>& piece, uint32_t i) {
        const uint32_t bit = (i + 1) * N, mask = listed[bit / 32] >> (bit % 32) & ((1u << N) - 1);
        if (mask) {
#pragma unroll
          for (uint32_t e = 0; e < N; ++e)
            if (mask >> e & 1u) piece.v[e] = narrow<T>(kMinusInf);
        }
      };
      uint32_t i0 = s.lo + tid;
      for (; i0 + (kUnroll - 1) * THREADS < s.hi; i0 += kUnroll * THREADS) {
        Piece<T> piece[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) piece[u] = pieces[i0 + u * THREADS];
        if (tail) {
#pragma unroll
          for (int u = 0; u < kUnroll; ++u) leave_out(piece[u], i0 + u * THREADS);
        }
        auto top = Top::of(piece[0]);
#pragma unroll
        for (int u = 1; u < kUnroll; ++u) top = Top::max(top, Top::of(piece[u]));
        run.raise(Top::value(top), p.c);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) run.z += terms(piece[u], run.base(), p.c);
      }
      for (; i0 < s.hi; i0 += THREADS) {
        Piece<T> piece = pieces[i0];
        if (tail) leave_out(piece, i0);
        run.raise(Top::value(Top::of(piece)), p.c);
        run.z += terms(piece, run.base(), p.c);
      }
      if (tid < s.loose()) {
        const uint32_t at = s.loose_at(tid), bit = at + N - s.head;
        if (!tail || !(listed[bit / 32] >> (bit % 32) & 1u)) {
          const float x = widen<T>(row[at]);
          run.raise(x, p.c);
          run.z += run.term(x, p.c);
        }
      }
      // the teacher's sums of this warp's entries
      if (tid < k) list_x[tid] = widen<T>(first_x);
      float most = kMinusInf;
      bool any = false;
      for (uint32_t i = tid; i < k; i += THREADS)
        if (list_idx[i] >= 0) {
          any |= list_val[i] != kMinusInf;  // (a NaN shows in the sums)
          most = fmaxf(most, list_x[i]);
        }
      Teacher t = {};
      t.any = __any_sync(0xffffffffu, any);
      t.most = from_ordered(__reduce_max_sync(0xffffffffu, ordered(most)));
      t.near = fabsf(t.most) == -kMinusInf ? 0.0f : t.most;
      if (!tail) {
        const float top = from_ordered(__reduce_max_sync(0xffffffffu, ordered(sm.top[tid % (THREADS / 32)])));
        shift = top == kMinusInf ? 0.0 : (double)top * p.inv_t;
      }
      for (uint32_t i = tid; i < k; i += THREADS)
        if (list_idx[i] >= 0) {
          const double a = (double)list_val[i] * p.inv_t - shift, e = exp(a);
          t.mass += e;
          const double b = ((double)list_x[i] - (double)t.near) * p.inv_t;
          if (e != 0.0) t.cross += e * (a - b);
          if (tail) t.own += exp(b);
        }
      if (t.any) {
#pragma unroll
        for (int st = 16; st >= 1; st /= 2) {
          t.mass += __shfl_xor_sync(0xffffffffu, t.mass, st);
          t.cross += __shfl_xor_sync(0xffffffffu, t.cross, st);
        }
      }
      if (tail) {
#pragma unroll
        for (int st = 16; st >= 1; st /= 2) t.own += __shfl_xor_sync(0xffffffffu, t.own, st);
      }
      if (tid % 32 == 0) sm.teacher[tid / 32] = t;
      run = block_merge<THREADS>(run, p.c, sm.run);
    }
    if (p.blocks > 1) {
      if (tid == 0) sm.mine = run;
      cluster_sync();
      run = cluster_merge(&sm.mine, p.blocks, p.c);
      cluster_sync();
    }
    bool any = false;
    if (active) any = __any_sync(0xffffffffu, sm.teacher[tid % (THREADS / 32)].any);
    // Without a remaining mass every logit's factor is 1 / z: the others go on to the gradient meanwhile.
    const float f_all = 1.0f / run.z;
    if (!tail) active = any && !(run.m == kMinusInf && run.z == 0.0f);
    // One warp puts it together: the teacher's sums, the factors, the loss
    //   sum p (log p - (x - largest) / T) + log z (P + p_rest) + p_rest (log p_rest - log r),
    // r the sum over what is not listed, relative to the largest logit like z.
    if (tid < 32) {
      constexpr uint32_t kWarps = THREADS / 32;
      double norm = 0.0, value = 0.0;
      float f_listed = 0.0f, f_rest = 0.0f;
      Running whole_row = run;  // (its m alone)
      if (active) {
        const Teacher t = sm.teacher[tid % kWarps];
        if (tail) whole_row.m = fmaxf(run.m, from_ordered(__reduce_max_sync(0xffffffffu, ordered(t.most))));
        const double base = whole_row.base();
        double mass = t.any ? t.mass : 0.0;
        double cross = t.any ? t.cross + (base - (double)t.near) * p.inv_t * t.mass : 0.0;
#pragma unroll
        for (int st = kWarps / 2; st >= 1; st /= 2) {
          mass += __shfl_xor_sync(0xffffffffu, mass, st);
          cross += __shfl_xor_sync(0xffffffffu, cross, st);
        }
        // what is not listed: its sum's factor and the factor's logarithm, relative to the largest logit of all
        const double below = ((double)run.base() - base) * p.inv_t;
        double z = run.z, f_below = 1.0;
        if (tail) {
          z = t.own != 0.0 ? t.own * exp(((double)t.near - base) * p.inv_t) : 0.0;
#pragma unroll
          for (int st = kWarps / 2; st >= 1; st /= 2) z += __shfl_xor_sync(0xffffffffu, z, st);
          f_below = exp(below);
          if (run.z != 0.0f) z += (double)run.z * f_below;
          // (a row of -infinity alone has no student; z is then 0, or a NaN that shows)
          active = any && !(whole_row.m == kMinusInf && z == 0.0);
        }
        if (active) {
          double rest = tail ? (mass == mass ? fmax(0.0, 1.0 - mass) : mass) : 0.0;
          if (tail && rest > 0.0) {
            // Where nothing is left to list there is no mass left, and next to nothing may be the rounding of the list's lse alone: a
            // student that has (nearly) none there either is not asked for it, its logarithm would make much of that.
            uint32_t named = 0;
            if (k >= p.vocab) {
              for (uint32_t i = tid; i < (p.vocab + N + 31) / 32; i += 32) named += __popc(listed[i]);
              named = __reduce_add_sync(0xffffffffu, named);
            }
            if (named == p.vocab ||
                (rest <= mass * kLseNoise * (18.0 + fabs(shift)) && (double)run.z * f_below < rest * z * kFewest))
              rest = 0.0;
          }
          const double lane_log = log(tid == 0 ? z : tid == 1 ? mass : tid == 2 ? rest : (double)run.z);
          const double log_z = __shfl_sync(0xffffffffu, lane_log, 0), log_mass = __shfl_sync(0xffffffffu, lane_log, 1);
          const double log_rest = __shfl_sync(0xffffffffu, lane_log, 2), log_r = __shfl_sync(0xffffffffu, lane_log, 3);
          const double listed = tail ? mass : 1.0, whole = listed + rest;
          norm = tail ? shift : shift + log_mass;
          value = (tail ? cross : cross / mass - log_mass) + log_z * whole;
          if (rest != 0.0) value += rest * (log_rest - (log_r + below));
          f_listed = f_rest = f_all;
          if (tail) {
            f_listed = (float)(whole / z);
            // nothing unlisted left in the student: no factor is needed there, but for a NaN that shows
            f_rest = run.z != 0.0f ? (float)(whole * f_below / z - (rest != 0.0 ? rest / (double)run.z : 0.0)) : z == z ? 0.0f : (float)z;
          }
        }
      }
      if (tid == 0) {
        sm.stat[kStatMax] = whole_row.m, sm.stat[kStatListed] = f_listed, sm.stat[kStatRest] = f_rest;
        sm.stat[kStatNorm] = (float)norm, sm.stat[kStatNormLow] = (float)(norm - (double)(float)norm);
        sm.stat[kStatActive] = active ? 1.0f : 0.0f, sm.stat[kStatRestMax] = run.m == kMinusInf ? 0.0f : run.m, sm.stat[7] = 0.0f;
        if (rank == 0) p.loss[r] = active ? (float)((double)weight * value) : 0.0f;
      }
      __syncwarp();
      if (rank == 0 && stats && tid < PVT_DISTILL_STATS) stats[tid] = sm.stat[tid];
    }
    if (MODE & kGrad) {
      m = run.m, f_rest = f_all;
      if (tail) {
        __syncthreads();
        active = sm.stat[kStatActive] != 0.0f, m = sm.stat[kStatRestMax], f_rest = sm.stat[kStatRest];
      }
    }
  }

  if (MODE & kGrad) {
    if (MODE == kGrad) {
      if (tid < PVT_DISTILL_STATS) sm.stat[tid] = stats[tid];
      if (active && tid < k) list_x[tid] = widen<T>(first_x);
      // in place: no block overwrites logits that another has yet to gather
      if (p.blocks > 1) cluster_sync();
      __syncthreads();
      m = sm.stat[kStatRestMax], f_rest = sm.stat[kStatRest];
    }
    if (!active) {
      clear<THREADS>(grad, s.from(), s.to());
      return;
    }
    const float up = (float)((double)weight * (double)upstream * p.inv_t);
    f_rest *= up;
    auto y_of = [&](float x, float of) { return ex2((x - of) * p.c); };
    if (sizeof(G) == sizeof(T) && (reinterpret_cast<uintptr_t>(grad) - reinterpret_cast<uintptr_t>(row)) % 16 == 0) {
      const Two bb = two(-m, -m), cc = two(p.c, p.c), ff = two(f_rest, f_rest);
      Piece<G>* const to = reinterpret_cast<Piece<G>*>(grad + s.head);
      auto write = [&](const Piece<T>& piece, uint32_t i) {
        Piece<G> out;
#pragma unroll
        for (uint32_t e = 0; e < N / 2; ++e) {
          const float2 y = each(mul2(add2(pair_of(piece, e), bb), cc));
          const float2 g = each(mul2(two(ex2(y.x), ex2(y.y)), ff));
          out.v[2 * e % Piece<G>::N] = narrow<G>(g.x), out.v[(2 * e + 1) % Piece<G>::N] = narrow<G>(g.y);
        }
        to[i] = out;
      };
      // Run by run, as each warp gets there: one of them comes late.
      const uint32_t lane = tid % 32;
      for (;;) {
        uint32_t run = 0;
        if (lane == 0) run = atomicAdd(&sm.next, 1u);
        const uint32_t i0 = s.lo + __shfl_sync(0xffffffffu, run, 0) * (kUnroll * 32) + lane;
        if (i0 - lane >= s.hi) break;
        if (i0 - lane + kUnroll * 32 <= s.hi) {
          Piece<T> piece[kUnroll];
#pragma unroll
          for (int u = 0; u < kUnroll; ++u) piece[u] = pieces[i0 + u * 32];
#pragma unroll
          for (int u = 0; u < kUnroll; ++u) write(piece[u], i0 + u * 32);
        } else {
          for (uint32_t i = i0; i < s.hi; i += 32) write(pieces[i], i);
        }
      }
      if (tid < s.loose()) {
        const uint32_t at = s.loose_at(tid);
        grad[at] = narrow<G>(y_of(widen<T>(row[at]), m) * f_rest);
      }
    } else {
      // rows of unlike alignment: element by element, a warp along the row
      const uint32_t to = s.to();
      uint32_t at = s.from() + tid;
      for (; at + 7 * THREADS < to; at += 8 * THREADS) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = widen<T>(row[at + u * THREADS]);
#pragma unroll
        for (int u = 0; u < 8; ++u) grad[at + u * THREADS] = narrow<G>(y_of(x[u], m) * f_rest);
      }
      for (; at < to; at += THREADS) grad[at] = narrow<G>(y_of(widen<T>(row[at]), m) * f_rest);
    }
    __syncthreads();
    const double norm = (double)sm.stat[kStatNorm] + (double)sm.stat[kStatNormLow];
    const float f_listed = sm.stat[kStatListed], largest = sm.stat[kStatMax];
    for (uint32_t i = tid; i < k; i += THREADS) {
      const int32_t at = list_idx[i];
      if (at < 0 || (uint32_t)at < s.from() || (uint32_t)at >= s.to()) continue;
      const float prob = (float)exp((double)list_val[i] * p.inv_t - norm);
      grad[at] = narrow<G>((y_of(list_x[i], largest) * f_listed - prob) * up);
    }
  }
}

template <typename T, typename G, int MODE, int THREADS>
cudaError_t start(const DistillParams& p, int64_t rows, cudaStream_t stream) {
  const cudaError_t e = allow_smem<distill_kernel<T, G, MODE, THREADS>>();
  if (e != cudaSuccess) return e;
  const size_t smem = sizeof(DistillShared<THREADS>) + 12 * (size_t)p.k + (size_t)(p.vocab + Piece<T>::N + 31) / 32 * 4;
  return launch_clusters(distill_kernel<T, G, MODE, THREADS>, (unsigned)(rows * p.blocks), p.blocks, THREADS, smem, stream, p);
}
template <typename T, typename G, int MODE>
cudaError_t start(const DistillParams& p, int64_t rows, int sm_count, cudaStream_t stream) {
  return short_rows(rows, (int64_t)p.vocab * sizeof(T), sm_count) ? start<T, G, MODE, kNarrow>(p, rows, stream)
                                                                   : start<T, G, MODE, kWide>(p, rows, stream);
}
template <typename T, int MODE>
cudaError_t by_grad(const DistillParams& p, int64_t rows, int32_t grad_dtype, int sm_count, cudaStream_t stream) {
  return grad_dtype == PVT_F32   ? start<T, float, MODE>(p, rows, sm_count, stream)
         : grad_dtype == PVT_F16 ? start<T, __half, MODE>(p, rows, sm_count, stream)
                                 : start<T, __nv_bfloat16, MODE>(p, rows, sm_count, stream);
}
template <typename T>
cudaError_t by_mode(const DistillParams& p, int64_t rows, int32_t grad_dtype, int sm_count, cudaStream_t stream) {
  if (!p.grad) return start<T, T, kLoss>(p, rows, sm_count, stream);
  return p.loss ? by_grad<T, kBoth>(p, rows, grad_dtype, sm_count, stream) : by_grad<T, kGrad>(p, rows, grad_dtype, sm_count, stream);
}

cudaError_t launch(const pvt_distill& d, DistillParams& p, int32_t grad_dtype, int sm_count, cudaStream_t stream) {
  p.logits = d.logits, p.ld = d.ld, p.vocab = (uint32_t)d.vocab, p.k = (uint32_t)d.k;
  p.c = (float)(1.4426950408889634 / (double)d.temperature), p.inv_t = 1.0 / (double)d.temperature;
  p.top_idx = d.top_idx, p.top_logit = d.top_logit, p.teacher_lse = d.teacher_lse, p.weight = d.weight;
  p.blocks = row_blocks(d.rows, (int64_t)d.vocab * (d.dtype == PVT_F32 ? 4 : 2), sm_count);
  if (d.rows * p.blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  timing_begin(kKernDistill, stream);
  const cudaError_t e = d.dtype == PVT_F32   ? by_mode<float>(p, d.rows, grad_dtype, sm_count, stream)
                        : d.dtype == PVT_F16 ? by_mode<__half>(p, d.rows, grad_dtype, sm_count, stream)
                                             : by_mode<__nv_bfloat16>(p, d.rows, grad_dtype, sm_count, stream);
  timing_end(kKernDistill, stream);
  count_launches(1);
  return e;
}

}  // namespace

cudaError_t launch_distill_loss(const pvt_distill& d, float* loss, float* stats, const float* upstream, void* grad,
                                int32_t grad_dtype, int64_t ldg, uint32_t* status, int sm_count, cudaStream_t stream) {
  DistillParams p = {};
  p.loss = loss, p.stats = stats, p.upstream = upstream, p.grad = grad, p.ldg = ldg, p.status = status;
  return launch(d, p, grad_dtype, sm_count, stream);
}

cudaError_t launch_distill_grad(const pvt_distill& d, const float* stats, const float* upstream, void* grad, int32_t grad_dtype,
                                int64_t ldg, uint32_t* status, int sm_count, cudaStream_t stream) {
  DistillParams p = {};
  p.stats = const_cast<float*>(stats), p.upstream = upstream, p.grad = grad, p.ldg = ldg, p.status = status;
  return launch(d, p, grad_dtype, sm_count, stream);
}

}  // namespace pvt
