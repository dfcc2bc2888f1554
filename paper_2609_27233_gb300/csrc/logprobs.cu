// Log probabilities of given tokens, entropy and the best alternatives of rows
// of logits, and the gradient of the first two with respect to the logits.
//
// With y = x / T, m = max x, s = sum_v exp((x_v - m) / T) and l = ln s:
//   logprob = (x_t - m) / T - l
//   H       = l - (1/s) sum_v exp((x_v - m) / T) (x_v - m) / T
//   p_v     = exp((x_v - m) / T - l)
//   d/dx_v  = (1/T) [ g (1[v = t] - p_v) - h p_v (ln p_v + H) ]
// for the upstream gradients g of logprob and h of H.  m and l are kept apart
// (the call's stats): their sum, the log-sum-exp, would lose the low bits of l
// where m is large.
#include <algorithm>
#include <cmath>

#include "logits.cuh"

namespace umim {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 8;        // vectors that a thread loads together: forward
constexpr int kGradUnroll = 4;    // and gradient
constexpr int kMaxCluster = 8;    // CTAs per row, at most

struct LogprobArgs {
  const void *logits;
  int32_t R, V;
  int64_t ld;
  const int32_t *n_dev;
  const int32_t *tokens;     // nullptr: no token, every row counts
  float inv_t, c;            // 1 / T, log2(e) / T
  float inv_low, c_low;      // what is left of 1 / T, and of c, relative to it, past their fp32 values
  int32_t n_top, slice;      // slice: elements of a row per CTA
  int32_t ahead;             // rows between one and that whose beginning its CTA brings into L2, or 0
  float *logprobs, *entropy;
  float2 *stats;
  int32_t *top_ids;
  float *top_logprobs;
  int32_t *status;
};

struct GradArgs {
  const void *logits;
  int32_t R, V;
  int64_t ld;
  const int32_t *n_dev;
  const int32_t *tokens;
  float inv_t, c;            // 1 / T, log2(e) / T
  int32_t parts, chunks;     // CTAs per row, chunks of a CTA
  const float2 *stats;
  const float *entropy, *g, *h;
  void *grad;
  int32_t *status;
};

__device__ __forceinline__ int rows_used(const int32_t *n_dev, int R) { return n_dev ? min(max(*n_dev, 0), R) : R; }

// A row's token; -1 leaves the row out, as does (with an error) one that is no token.
__device__ __forceinline__ int row_token(const int32_t *tokens, int r, int V, int32_t *status, bool report) {
  const int t = tokens[r];
  if (t >= 0 && t < V) return t;
  if (t != -1 && report) set_error(status, UMIM_ERR_INVALID_ARG);
  return -1;
}

// ---------------------------------------------------------------------------
// softmax statistics: a running maximum m, and s = sum 2^t, w = sum t 2^t over
// t = (x - m) c, c = log2(e) / T
// ---------------------------------------------------------------------------
struct Stats {
  float m, s, w;
};
__device__ __forceinline__ Stats no_stats() { return Stats{-INFINITY, 0.f, 0.f}; }

// s and w from their reference to `to`, which is not below it.  What underflows goes to 0, a NaN stays one.
__device__ __forceinline__ void rebase(Stats &a, float to, float c) {
  if (!(a.m == to)) {
    const float d = (a.m - to) * c, f = ex2(d), s = a.s;
    a.s = s * f;
    a.w = f > 0.f ? f * fmaf(s, d, a.w) : a.s;
    a.m = to;
  }
}

// the warp's statistics in every lane, at its maximum; top: the largest this lane has seen
__device__ __forceinline__ Stats warp_stats(Stats a, float top, float c) {
  rebase(a, warp_max(top), c);
  const float2 v = warp_sum2(make_float2(a.s, a.w));
  a.s = v.x;
  a.w = v.y;
  return a;
}

// 2^t is 0 from t = -150 on; where it is weighed with t, a t of -inf must not make that
// no number.  (bf16 elements are kept finite two at a time instead, which
// holds as long as |m c| < 2^24.)
constexpr float kLeastT = -1000.f;

// One thread's part: eight vectors at a time.  t is one FMA, x c + b with
// b = -m c rounded; the rounding r is common to a chunk and made good on its
// sums, so that t is as exact for large |m| as (x - m) c.  Where r itself is large
// (|m c| past 2^24, or no number) the chunk is read again and done the careful
// way.  NaN and +inf leave s as NaN on both.
//
// The reference m follows the maximum only when that has come 2^16 past it:
// until then the exponentials are as exact, and the sums far from overflowing.
constexpr float kSlack = 16.f;

template <class E>
struct Running {
  Stats st = no_stats();
  float top = -INFINITY;             // the maximum
  float b = 0.f, r = 0.f, rf = 1.f;

  // again(k): vector k of the chunk, read a second time
  template <class Again>
  __device__ __forceinline__ void add(const uint4 (&u)[kUnroll], uint32_t max_word, float c, Again again) {
    const float cm = E::to_float(E::word_max_bits(max_word));
    top = fmaxf(top, cm);
    if ((cm - st.m) * c > kSlack) {
      rebase(st, cm, c);
      b = -cm * c;
      r = fmaf(-cm, c, -b);
      rf = ex2(r);
      if (!(fabsf(r) <= 1.f)) b = NAN;   // the careful way
    }
    const float2 c2 = make_float2(c, c), b2 = make_float2(b, b);
    float2 s0 = make_float2(0.f, 0.f), s1 = s0, w0 = s0, w1 = s0;
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
#pragma unroll
      for (int i = 0; i < E::VEC / 2; ++i) {
        float2 x;
        if constexpr (E::kHasFinite)
          x = E::pair(E::finite_words(word(u[k], i)));
        else
          x = pair_of<E>(u[k], i);
        float2 t = __ffma2_rn(x, c2, b2);
        const float2 e = make_float2(ex2(t.x), ex2(t.y));
        if constexpr (!E::kHasFinite) t = make_float2(fmaxf(t.x, kLeastT), fmaxf(t.y, kLeastT));
        if (i & 1) {
          s1 = __fadd2_rn(s1, e);
          w1 = __ffma2_rn(e, t, w1);
        } else {
          s0 = __fadd2_rn(s0, e);
          w0 = __ffma2_rn(e, t, w0);
        }
      }
    s0 = __fadd2_rn(s0, s1);
    w0 = __fadd2_rn(w0, w1);
    const float s = s0.x + s0.y, w = w0.x + w0.y;
    if (!isnan(b)) {
      st.s = fmaf(rf, s, st.s);
      st.w = fmaf(rf, fmaf(r, s, w), st.w);
    } else {
      add_carefully(again, c);
    }
  }

  template <class Again>
  __device__ __forceinline__ void add_carefully(Again again, float c) {
    const float m0 = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll 1
    for (int k = 0; k < kUnroll; ++k) {
      const uint4 u = again(k);
#pragma unroll
      for (int i = 0; i < E::VEC / 2; ++i) {
        const float2 x = pair_of<E>(u, i);
        float t = (x.x - m0) * c;
        float e = ex2(t);
        st.s += e;
        st.w = fmaf(e, fmaxf(t, kLeastT), st.w);
        t = (x.y - m0) * c;
        e = ex2(t);
        st.s += e;
        st.w = fmaf(e, fmaxf(t, kLeastT), st.w);
      }
    }
  }
};

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
// One cluster of C CTAs per row, each on one of C contiguous parts, a chunk of 64 strips of
// 32 vectors after the other.  A warp takes eight strips of it side by side, a lane one vector
// of each: every logit is read once, by 16-byte loads, a warp's eight together while
// the others work on theirs.  (SPREAD: every eighth strip, so that all threads
// have some of a part that is no whole chunk; spread_pays has when.)
// (Half as many a chunk ahead of their use took 4 % longer for 4096 rows of 128256
// bf16 with 64 alternatives, asynchronous copies into buffers of the warp's own another
// 4 %.)
//
// The alternatives need no second pass over the row.  Beside the sums, the
// maximum of every segment of 32 consecutive elements goes to shared memory.
// In whatever way the row is divided into groups, the n-th largest of the groups'
// maxima is a bound for the n best elements.  The groups here are the 256
// that C threads each have read, whose maxima the threads hold anyway: a few
// rounds of counting give a threshold that n of them reach, and not many
// more.  The segments that reach it are read again (64 or 128 bytes each, from L2),
// and of a row's elements about 256 ln(256 / (256 - n)) pass it (21 for n = 20, 177
// for 128), which are ranked by counting.
//
// Equal values can make them more than 256.  The n best by (value, lowest id) lie in
// the n best segments by (maximum, lowest place): n segments before one that
// holds an element each have an element before it.  So bisections, by value and
// then by place, pick exactly n segments, and of their elements exactly n.
//
// What bounds it: without alternatives the one read of the logits (4096 rows of 128256
// bf16: 149 us, 7.0 TB/s, above the measured copy's rate); with them the
// instructions as well, 5.8 a logit for the pass and 1.4 (one alternative) to 2.8
// (128) for segments and search: 166 us with 20, 176 with 64, 186 with 128.  Rows that take the bisections cost four
// times that: 751 us with 64 alternatives where all but 12 are masked by the type's lowest value (327 of it the pass).
//
// All of it happens in shared memory and registers of the cluster: no
// workspace, no atomics on global memory, the same bits in every call.
constexpr int kSegment = 32;
constexpr float kPeaked = 1.03125f;   // s below this: the largest element has 97 % of the probability
template <class E>
__host__ __device__ constexpr int chunk_elems() {   // of a CTA's chunk
  return kUnroll * kWarps * 32 * E::VEC;
}

// While a CTA searches it reads nothing, so before that it has the beginning of the row that a CTA in
// its place is likely to take next brought into L2 (2.1 % less time for 4096 rows of 128256 bf16
// with 64 alternatives, 3.9 % for 2000 rows of 50257; with 16 KB 1.2 and 4.9 %, with 64 KB 2.7 % less
// and 3.1 % more).
constexpr int kAheadBytes = 32768;
constexpr int kCands = kThreads;     // candidates that are ranked, at most
constexpr int kListed = 2 * kThreads; // segments that reach the threshold, at most (else the exact way)

// Dynamic shared memory.
template <class E>
struct TopShared {
  uint64_t *merge;         // rank 0 of several: [C][merge_cap(n)] every CTA's candidates
  typename E::T *seg;      // [segments, up to a whole chunk] maximum of each
  static __host__ __device__ int padded(int slice) {
    return ceil_div(slice, chunk_elems<E>()) * (chunk_elems<E>() / kSegment);
  }
  // what a CTA tells rank 0: n at most, or the few more that the threshold let pass
  static __host__ __device__ int merge_cap(int n) { return n > 32 ? n : 32; }
  static size_t bytes(int slice, int n, int C) {
    return 8 * (size_t)(C > 1 ? C * merge_cap(n) : 0) + sizeof(typename E::T) * (size_t)padded(slice);
  }
  __device__ TopShared(uint8_t *p, int slice, int n, int C) {   // seg starts on 16 bytes: C is even where it counts
    merge = reinterpret_cast<uint64_t *>(p);
    seg = reinterpret_cast<typename E::T *>(merge + (C > 1 ? C * merge_cap(n) : 0));
  }
};

__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t key_of(uint64_t e) { return (uint32_t)(e >> 32); }
__device__ __forceinline__ uint32_t id_of(uint64_t e) { return ~(uint32_t)e; }
__device__ __forceinline__ uint64_t entry(uint32_t key, uint32_t id) { return ((uint64_t)key << 32) | (uint32_t)~id; }

// The bits of vector word w[j / 2] (16-bit elements) or w[j] that are element j.
template <class E>
__device__ __forceinline__ typename E::T element(const uint4 &u, int j) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  if constexpr (E::VEC == 8)
    return (typename E::T)(w[j / 2] >> (16 * (j & 1)));
  else
    return __uint_as_float(w[j]);
}

// the same where j is not known to the compiler
template <class E>
__device__ __forceinline__ typename E::T element_at(const uint4 &u, int j) {
  const int i = E::VEC == 8 ? j / 2 : j;
  const uint32_t w = i & 2 ? (i & 1 ? u.w : u.z) : (i & 1 ? u.y : u.x);
  if constexpr (E::VEC == 8)
    return (typename E::T)(w >> (16 * (j & 1)));
  else
    return __uint_as_float(w);
}

// bit j: element j is no smaller than the one of key `least` (none is NaN)
template <class E>
__device__ __forceinline__ uint32_t reach_mask(const uint4 &u, uint32_t least) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  uint32_t mask = 0;
  if constexpr (E::VEC == 8) {
    const uint32_t bits = E::from_key(least), both = bits | bits << 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) mask |= (E::reach_words(w[i], both) & 0x00020001u) << (2 * i);
    return (mask | mask >> 16) & 0xffu;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) mask |= (__uint_as_float(w[i]) >= E::from_key(least) ? 1u : 0u) << i;
    return mask;
  }
}

// the warp's values in descending order (a bitonic sort)
__device__ __forceinline__ uint64_t warp_sorted(uint64_t v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) {
      const uint64_t o = __shfl_xor_sync(0xffffffffu, v, j);
      const bool larger = ((lane & j) == 0) == ((lane & k) == 0);   // this lane keeps the larger one
      v = (v > o) == larger ? v : o;
    }
  return v;
}

// The n first of the CTA's entries by (key descending, id ascending), of which there are
// more: a key, and the largest id that is still in at that key.  lo: a key that
// more than n reach; hi: the largest; ids are below `ids`.  own(pred): how
// many of this thread's entries satisfy pred(key, id).
struct Cut {
  uint32_t key, id;
  __device__ bool in(uint32_t k, uint32_t i) const { return k > key || (k == key && i <= id); }
};
template <class Own>
__device__ Cut cut_at(int n, uint32_t lo, uint32_t hi, uint32_t ids, Own own) {
  __shared__ int part[2][kWarps];
  int turn = 0;
  const auto count = [&](auto pred) {   // over the CTA
    const int warp_sum = __reduce_add_sync(0xffffffffu, own(pred));
    if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = warp_sum;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) sum += part[turn][i];
    turn ^= 1;   // the next count's barrier is before these are written again
    return sum;
  };
  Cut c;
  while (lo < hi) {   // the largest key that n reach
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    if (count([&](uint32_t k, uint32_t) { return k >= mid; }) >= n)
      lo = mid;
    else
      hi = mid - 1;
  }
  c.key = lo;
  const int left = n - count([&](uint32_t k, uint32_t) { return k > c.key; });
  uint32_t a = 0, b = ids - 1;
  while (a < b) {     // the smallest id with `left` equal entries at or below it
    const uint32_t mid = (a + b) / 2;
    if (count([&](uint32_t k, uint32_t i) { return k == c.key && i <= mid; }) >= left)
      b = mid;
    else
      a = mid + 1;
  }
  c.id = a;
  __syncthreads();   // the last count has been read
  return c;
}

// The elements of row[beg, end) that reach `least`, in any order, to cand[]; where they
// are more than kCands, the n best.  hi: the largest key.  Returns how many.
// Neither NaN nor +inf is among them.
template <class E>
__device__ int gather_best(const typename E::T *seg, const typename E::T *row, int beg, int end, int n, uint32_t least,
                           uint32_t hi, uint64_t *cand, int32_t *status) {
  __shared__ int s_listed, s_held;
  __shared__ uint16_t list[kListed];
  const int tid = threadIdx.x, segs = ceil_div(end - beg, kSegment);

  using T = typename E::T;
  const float least_x = E::to_float(E::from_key(least));   // a bound in passing: x >= it as its key >= least
  // the segments that reach `least` and that `in` takes, to list[]; returns how many
  const auto list_segments = [&](auto in) {
    if (tid == 0) s_listed = 0;
    __syncthreads();
    for (int i = tid * E::VEC; i < segs; i += kThreads * E::VEC) {
      const uint4 u = *reinterpret_cast<const uint4 *>(seg + i);
      const uint32_t top = E::max_words(E::max_words(u.x, u.y), E::max_words(u.z, u.w));
      if (E::to_float(E::word_max_bits(top)) >= least_x)
        for (uint32_t hits = reach_mask<E>(u, least); hits; hits &= hits - 1) {
          const int j = __ffs(hits) - 1;
          if (in(element_at<E>(u, j), (uint32_t)(i + j))) {
            const int at = atomicAdd(&s_listed, 1);
            if (at < kListed) list[at] = (uint16_t)(i + j);
          }
        }
    }
    __syncthreads();
    return s_listed;
  };

  // the i-th vector of the listed segments, the first element's id to e
  constexpr int kVecs = kSegment / E::VEC;
  const auto load_listed = [&](int i, int &e) {
    int s = list[i / kVecs];
    if (!in_bounds(s, segs, status, kSiteLogprobSegment)) s = 0;
    e = beg + s * kSegment + (i % kVecs) * E::VEC;
    return load_raw<E>(row, e, end);
  };
  // The elements of listed segments that reach `least` and that `in` takes, to cand[]; returns how
  // many.  Three vectors a thread on their way at once (82.3 us for 4104 rows of 32000 bf16 with 128
  // alternatives, 85.4 by two; no difference for 64 and fewer).
  const auto gather = [&](int listed, auto in) {
    if (tid == 0) s_held = 0;
    __syncthreads();
    const auto take = [&](const uint4 &u, int e) {
      const uint32_t top = E::max_words(E::max_words(u.x, u.y), E::max_words(u.z, u.w));
      if (E::to_float(E::word_max_bits(top)) >= least_x)
        for (uint32_t hits = reach_mask<E>(u, least); hits; hits &= hits - 1) {
          const int j = __ffs(hits) - 1;
          const T x = element_at<E>(u, j);
          if (in(x, (uint32_t)(e + j))) {
            const int at = atomicAdd(&s_held, 1);
            if (at < kCands) cand[at] = entry(E::order_key(x), (uint32_t)(e + j));
          }
        }
    };
    constexpr int kAtOnce = 3;
    for (int i = tid; i < listed * kVecs; i += kAtOnce * kThreads) {
      uint4 u[kAtOnce];
      int e[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
        if (i + k * kThreads < listed * kVecs) u[k] = load_listed(i + k * kThreads, e[k]);
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
        if (i + k * kThreads < listed * kVecs) take(u[k], e[k]);
    }
    __syncthreads();
    return s_held;
  };
  const auto reaches = [](T, uint32_t) { return true; };
  const int listed = list_segments(reaches);
  if (listed <= kListed) {
    const int held = gather(listed, reaches);
    if (held <= kCands) return held;
  }
  // Many equal ones: n segments exactly, then n elements.  More than n segments are above
  // `least`, unless all of it lies in fewer.
  Cut cut{least, (uint32_t)segs};
  if (listed > n)
    cut = cut_at(n, least, hi, (uint32_t)segs, [&](auto pred) {
      int c = 0;
      for (int i = tid; i < segs; i += kThreads) {
        const uint32_t k = E::order_key(seg[i]);
        c += k >= least && pred(k, (uint32_t)i);
      }
      return c;
    });
  const int kept = list_segments([&](T x, uint32_t i) { return cut.in(E::order_key(x), i); });
  const Cut best = cut_at(n, cut.key, hi, (uint32_t)end, [&](auto pred) {
    int c = 0;
    for (int i = tid; i < kept * kVecs; i += kThreads) {
      int e;
      const uint4 u = load_listed(i, e);
#pragma unroll
      for (int j = 0; j < E::VEC; ++j) {
        const uint32_t k = E::order_key(element<E>(u, j));
        c += k >= cut.key && pred(k, (uint32_t)(e + j));
      }
    }
    return c;
  });
  return gather(kept, [&](T x, uint32_t i) { return best.in(E::order_key(x), i); });
}

// The n first of the M > n entries of from[], in any order, to cand[] (which may be from).
__device__ void keep_best(const uint64_t *from, int M, int n, uint32_t lo, uint32_t hi, int V, uint64_t *cand) {
  __shared__ int s_kept;
  if (threadIdx.x == 0) s_kept = 0;
  const Cut cut = cut_at(n, lo, hi, (uint32_t)V, [&](auto pred) {
    int c = 0;
    for (int i = threadIdx.x; i < M; i += kThreads) c += pred(key_of(from[i]), id_of(from[i]));
    return c;
  });
  constexpr int kHold = kMaxCluster * kMaxTop / kThreads;   // entries of a thread, at most
  uint64_t held[kHold];
#pragma unroll
  for (int k = 0; k < kHold; ++k) {
    const int i = threadIdx.x + k * kThreads;
    held[k] = i < M && cut.in(key_of(from[i]), id_of(from[i])) ? from[i] : 0;
  }
  __syncthreads();   // all of from has been read
#pragma unroll
  for (int k = 0; k < kHold; ++k)
    if (held[k] != 0) {
      const int at = atomicAdd(&s_kept, 1);
      cand[at] = held[k];
    }
  __syncthreads();
}

// What the warps of a cluster tell each other: their sums, and the least of their groups' maxima.
struct __align__(16) WarpPart {
  float m, s, w, least;
};

template <class E, bool TOP, bool SPREAD>
__global__ void __launch_bounds__(kThreads, 4) token_logprobs_kernel(LogprobArgs a) {
  extern __shared__ __align__(128) uint8_t dyn[];
  __shared__ WarpPart s_parts[kMaxCluster * kWarps];
  __shared__ uint32_t s_group[kThreads];
  __shared__ __align__(16) uint64_t s_cand[kCands];
  __shared__ int s_count[kMaxCluster];
  __shared__ float2 s_rest;
  griddep_wait();
  griddep_launch();
  const int C = (int)cluster_size(), rank = C > 1 ? (int)cluster_ctarank() : 0;
  const int r = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.V, n = TOP ? a.n_top : 0;
  if (r >= rows_used(a.n_dev, a.R)) return;
  const int token = a.tokens ? row_token(a.tokens, r, V, a.status, rank == 0 && tid == 0) : 0;
  if (token < 0) {   // left out
    if (rank == 0) {
      if (tid == 0) {
        if (a.logprobs) a.logprobs[r] = 0.f;
        if (a.entropy) a.entropy[r] = 0.f;
        if (a.stats) a.stats[r] = make_float2(0.f, 0.f);
      }
      for (int i = tid; i < n; i += kThreads) {
        a.top_ids[(int64_t)r * n + i] = -1;
        a.top_logprobs[(int64_t)r * n + i] = -INFINITY;
      }
    }
    return;
  }
  const typename E::T *row = static_cast<const typename E::T *>(a.logits) + (int64_t)r * a.ld;
  const int beg = min(rank * a.slice, V), end = min(beg + a.slice, V);
  const TopShared<E> sh(dyn, a.slice, n, C);
  if (C > 1) cluster_arrive();   // what is pushed to a CTA waits until it runs
  const bool writes = rank == 0 && tid == kThreads - 32;   // the row's numbers: a warp with little to search
  float x_t = 0.f;
  if (writes) x_t = E::to_float(row[token]);

  // ---- one pass over this CTA's part ----
  const float c = a.c;
  Running<E> run;
  // elements of a strip, from the warp's first to its next one, and from a chunk to the next
  constexpr int kStrip = 32 * E::VEC, kNext = SPREAD ? kWarps * kStrip : kStrip, kChunk = kUnroll * kWarps * kStrip;
  const int first = SPREAD ? warp * kStrip : warp * kUnroll * kStrip;
  const auto load = [&](uint4 (&v)[kUnroll], int e0) {   // the warp's strips from element e0 on
    if (e0 + (kUnroll - 1) * kNext + kStrip <= end) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        v[k] = __ldcs(reinterpret_cast<const uint4 *>(row + e0 + k * kNext + lane * E::VEC));
    } else {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) v[k] = load_raw<E>(row, e0 + k * kNext + lane * E::VEC, end);
    }
  };
  // where this lane's segment goes: the one of strip lane % 4 of each four that has the vector lane
  typename E::T *seg_at = sh.seg + (first + (lane & 3) * kNext) / kSegment + lane / (32 / E::VEC);
  const auto take = [&](const uint4 (&u)[kUnroll], int e0) {
    uint32_t top[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
      top[k] = E::max_words(E::max_words(u[k].x, u[k].y), E::max_words(u[k].z, u[k].w));
    if constexpr (TOP) {
      // The maxima of four neighbouring lanes' vectors, transposed: a lane ends up with
      // that of its four for vector lane % 4 of each four.
      static_assert(kUnroll % 4 == 0, "four vectors among four lanes");
      const bool odd = lane & 1, high = lane & 2;
#pragma unroll
      for (int g = 0; g < kUnroll; g += 4) {
        const uint32_t p =
            E::max_words(odd ? top[g + 1] : top[g], __shfl_xor_sync(0xffffffffu, odd ? top[g] : top[g + 1], 1));
        const uint32_t q =
            E::max_words(odd ? top[g + 3] : top[g + 2], __shfl_xor_sync(0xffffffffu, odd ? top[g + 2] : top[g + 3], 1));
        uint32_t m = E::max_words(high ? q : p, __shfl_xor_sync(0xffffffffu, high ? p : q, 2));
        if (E::VEC == 4) m = E::max_words(m, __shfl_xor_sync(0xffffffffu, m, 4));   // eight lanes make a segment
        if (E::VEC == 8 || !(lane & 4)) seg_at[g * kNext / kSegment] = E::word_max_bits(m);
      }
      seg_at += kChunk / kSegment;
    }
    uint32_t all = top[0];
#pragma unroll
    for (int k = 1; k < kUnroll; ++k) all = E::max_words(all, top[k]);
    run.add(u, all, c, [&](int k) { return load_raw<E>(row, e0 + k * kNext + lane * E::VEC, end); });
  };
  for (int e0 = beg + first; e0 < end; e0 += kChunk) {
    uint4 u[kUnroll];
    load(u, e0);
    take(u, e0);
  }

  if (TOP && a.ahead > 0 && tid == 0 && end >= E::VEC && r + a.ahead < rows_used(a.n_dev, a.R) &&
      (!a.tokens || a.tokens[r + a.ahead] >= 0))
    bulk_prefetch(row + (int64_t)a.ahead * a.ld, (uint32_t)min(end / E::VEC * 16, kAheadBytes));

  // ---- the row's sums, and a threshold for its alternatives ----
  {
    float group = run.top;   // the maximum of this thread's group: C threads that lie side by side
    for (int o = 1; o < C; o <<= 1) group = fmaxf(group, __shfl_xor_sync(0xffffffffu, group, o));
    const Stats ws = warp_stats(run.st, run.top, c);
    const WarpPart p{ws.m, ws.s, ws.w, -warp_max(-group)};
    const int place = rank * kWarps + warp;
    const uint32_t key = E::order_key(E::from_float(group));
    const int at = (rank * kThreads + tid) / C;   // the group's, among the row's 256
    if (C == 1) {
      if (lane == 0) s_parts[place] = p;
      if (TOP) s_group[at] = key;
      __syncthreads();
    } else {
      cluster_wait();
      if (lane < C) {
        const uint32_t to = peer_addr(&s_parts[place], (uint32_t)lane);
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to), "f"(p.m), "f"(p.s), "f"(p.w),
                     "f"(p.least)
                     : "memory");
      }
      // thread j of a group tells CTA j
      if (TOP)
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_addr(&s_group[at], (uint32_t)(tid % C))), "r"(key)
                     : "memory");
      cluster_sync_all();
    }
  }
  Stats all = no_stats();
  float least_group = INFINITY;
  for (int i = lane; i < C * kWarps; i += 32) {
    const WarpPart p = s_parts[i];
    Stats q{p.m, p.s, p.w};
    least_group = fminf(least_group, p.least);
    const float to = fmaxf(all.m, q.m);
    rebase(all, to, c);
    rebase(q, to, c);
    all.s += q.s;
    all.w += q.w;
  }
  all = warp_stats(all, all.m, c);
  // NaN and +inf have no place in the order, and a row that holds one has no alternatives
  const bool bad = !(all.s < INFINITY), empty = all.m == -INFINITY && !bad;

  // Where one element has nearly all of the probability, ln s and the entropy are as small as what the others
  // add to its 1, and a sum that holds the 1 has rounded that away.  (Equal largest ones make s 2 or more.)
  // So they are summed alone: every warp but that element's has, its other lanes have too, and its
  // own lane's elements are read again, by the whole warp.  (Summed with the 1, the entropy of such rows was off by
  // up to 7e-7, so it is 5e-8, and in proportion where it is smaller.)  A row like this costs its CTA about 1.5 us.  Where
  // every row is one, for random rows and for those, us: 4096 of 128256 bf16 with 64 alternatives 176 and 193, 8192 without
  // 288 and 307, 4104 of 32000 with 20 66 and 74, 16384 of 8000 with 128 271 and 296, 128 of 128256 with 5 14.3 and 14.7.
  const bool peaked = !bad && !empty && all.s < kPeaked;   // the same in all of a row's threads
  float rest = 0.f;
  if (peaked) {
    int at = 0;
    for (int i = lane; i < C * kWarps; i += 32)
      if (s_parts[i].m == all.m) at = i;
    at = __reduce_max_sync(0xffffffffu, at);
    if (at == rank * kWarps + warp) {
      const int owner = __ffs(__ballot_sync(0xffffffffu, run.top == all.m)) - 1;
      rebase(run.st, all.m, c);
      float2 v = lane == owner ? make_float2(0.f, 0.f) : make_float2(run.st.s, run.st.w);
#pragma unroll 1
      for (int q = lane; q < ceil_div(end - beg, kChunk) * kUnroll; q += 32) {   // its vectors
        const int e = beg + first + q / kUnroll * kChunk + q % kUnroll * kNext + owner * E::VEC;
        if (e >= end) continue;
        float x[E::VEC];
        unpack<E>(load_raw<E>(row, e, end), x);
#pragma unroll
        for (int j = 0; j < E::VEC; ++j) {
          const float t = (x[j] - all.m) * c, p = x[j] == all.m ? 0.f : ex2(t);
          v.x += p;
          v.y = fmaf(p, fmaxf(t, kLeastT), v.y);
        }
      }
      __syncwarp();
      v = warp_sum2(v);
      if (C == 1) {
        if (lane == 0) s_rest = v;
      } else if (lane < C) {
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(peer_addr(&s_rest, (uint32_t)lane)), "f"(v.x),
                     "f"(v.y)
                     : "memory");
      }
    }
    if (C > 1)
      cluster_sync_all();
    else
      __syncthreads();
    float2 v = make_float2(0.f, 0.f);
    for (int i = lane; i < C * kWarps; i += 32)
      if (i != at) {
        Stats q{s_parts[i].m, s_parts[i].s, s_parts[i].w};
        rebase(q, all.m, c);
        v.x += q.s;
        v.y += q.w;
      }
    v = warp_sum2(v);
    rest = v.x + s_rest.x;
    all.w = v.y + s_rest.y;
    all.s = 1.f + rest;
  }

  // The sums were taken with c, off by c_low of itself: ln s by c_low times the mean of (x - m) / T, to first order.  (The
  // entropy's two parts are off alike.)  And log probabilities are rounded once: x - m, then both parts of 1 / T by FMA.
  const float mean = kLn2 * (all.w / all.s), l0 = peaked ? log1pf(rest) : logf(all.s);
  const float m0 = empty ? 0.f : all.m, l = bad ? NAN : empty ? 0.f : fmaf(a.c_low, mean, l0);
  const auto log_prob = [&](float x) {
    const float d = x - m0;
    return d == -INFINITY ? d : fmaf(d, a.inv_t, fmaf(d, a.inv_low, -l));
  };
  if (writes) {
    if (a.logprobs) a.logprobs[r] = bad ? NAN : log_prob(x_t);
    if (a.entropy) a.entropy[r] = bad ? NAN : empty ? 0.f : l0 - mean;
    if (a.stats) a.stats[r] = bad ? make_float2(NAN, NAN) : make_float2(all.m, l);
  }

  int M = 0;   // the candidates, in s_cand of rank 0
  if constexpr (TOP) {
    if (!bad && !empty) {
      const uint32_t hi = E::order_key(E::from_float(all.m)), none = E::order_key(E::kNegInf);
      const float lg = -warp_max(-least_group);
      uint32_t least = max(E::order_key(E::from_float(lg)), none + 1);
      {   // largest_reached, until not many more than n reach it
        const uint32_t group = s_group[tid];
        const int most = min(n + n / 8 + 4, kThreads / 2 + 8);   // about 194 candidates, 256 being the limit
        uint32_t top = hi;
        while (least < top) {
          const uint32_t mid = least + (top - least + 1) / 2;
          const int reach = __syncthreads_count(group >= mid);
          if (reach >= n)
            least = mid;
          else
            top = mid - 1;
          if (reach >= n && reach <= most) break;
        }
      }
      M = gather_best<E>(sh.seg, row, beg, end, n, least, hi, s_cand, a.status);
      if (C > 1) {   // to rank 0
        const int cap = sh.merge_cap(n);
        if (M > cap) {
          keep_best(s_cand, M, n, least, hi, V, s_cand);
          M = n;
        }
        if (tid == 0)
          asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(peer_addr(&s_count[rank], 0)), "r"(M) : "memory");
        if (tid < M)
          asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(peer_addr(&sh.merge[rank * cap + tid], 0)),
                       "l"(s_cand[tid])
                       : "memory");
        cluster_sync_all();
        if (rank != 0) return;
        M = 0;
        for (int k = 0; k < C; ++k) M += s_count[k];
        const bool fit = M <= kCands;
        uint64_t *side_by_side = fit ? s_cand : sh.merge;   // in merge list k moves down to the end of list k - 1
        for (int k = 0, at = 0; k < C; ++k) {
          const int count = s_count[k];
          const uint64_t e = tid < count ? sh.merge[k * cap + tid] : 0;
          if (!fit) __syncthreads();
          if (tid < count) side_by_side[at + tid] = e;
          at += count;
        }
        __syncthreads();
        if (!fit) {
          keep_best(sh.merge, M, n, least, hi, V, s_cand);
          M = n;
        }
      }
    }
  }
  if (rank != 0) return;

  // ---- the alternatives in order ----
  if constexpr (TOP) {
    uint64_t mine;
    int place = 0;
    if (M <= kCands / 2) {   // an entry's place is how many come before it: P threads side by side count for it
      int P = 1;
      while (2 * P * M <= kThreads && P < 32) P *= 2;
      const int i = tid / P;
      mine = i < M ? s_cand[i] : 0;
#pragma unroll 8
      for (int k = tid % P; k < M; k += P) place += s_cand[k] > mine;
      for (int o = 1; o < P; o <<= 1) place += __shfl_xor_sync(0xffffffffu, place, o);
      if (tid % P != 0) mine = 0;
    } else {                 // every warp sorts its 32, then looks for its own in the other warps' lists
      mine = warp_sorted(tid < M ? s_cand[tid] : 0);
      __syncthreads();
      s_cand[tid] = mine;
      __syncthreads();
      int before[kWarps] = {};
#pragma unroll
      for (int step = 16; step > 0; step >>= 1)
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
          if (s_cand[w * 32 + before[w] + step - 1] > mine) before[w] += step;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) place += before[w] + (before[w] == 31 && s_cand[w * 32 + 31] > mine);
    }
    if (mine != 0 && place < n && in_bounds(place, n, a.status, kSiteLogprobRank)) {
      a.top_ids[(int64_t)r * n + place] = (int)id_of(mine);
      a.top_logprobs[(int64_t)r * n + place] = log_prob(E::to_float(E::from_key(key_of(mine))));
    }
    if (tid >= M && tid < n) {
      a.top_ids[(int64_t)r * n + tid] = -1;
      a.top_logprobs[(int64_t)r * n + tid] = bad ? NAN : -INFINITY;
    }
  }
}

// ---------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------
// Elementwise, bound by its one read and one write of every element.  A CTA takes
// some chunks of a row: 4 vectors a thread each, loaded together and ahead of the
// row's numbers.  With t = log2 p the element is p (A + B t), A = -(g + h H) / T and
// B = -h ln 2 / T; the token's own is -g expm1(ln p) / T + p (A + g / T + B t), exact
// where p is so near 1 that 1 - p would be nothing.
template <class E>
__global__ void __launch_bounds__(kThreads, 4) token_logprobs_grad_kernel(GradArgs a) {
  griddep_wait();
  griddep_launch();
  const int r = blockIdx.x / a.parts, V = a.V;
  if (r >= rows_used(a.n_dev, a.R)) return;
  const typename E::T *row = static_cast<const typename E::T *>(a.logits) + (int64_t)r * a.ld;
  typename E::T *out = static_cast<typename E::T *>(a.grad) + (int64_t)r * a.ld;
  constexpr int kStep = kThreads * E::VEC, kChunk = kGradUnroll * kStep;
  const int part = blockIdx.x % a.parts * a.chunks * kChunk, last = min(V, part + a.chunks * kChunk);
  int e0 = part + threadIdx.x * E::VEC;

  const int token = a.tokens ? row_token(a.tokens, r, V, a.status, threadIdx.x == 0) : 0;
  const float2 st = a.stats[r];
  const float g = a.g ? a.g[r] * a.inv_t : 0.f, h = a.h ? a.h[r] * a.inv_t : 0.f;
  const bool zero = token < 0 || st.x == -INFINITY;
  if (zero) {
    const float z[E::VEC] = {};
    for (; e0 < last; e0 += kStep) store_vec<E>(out, e0, V, z);
    return;
  }
  const float H = a.h ? a.entropy[r] : 0.f;
  // a row without a distribution has NaN for m: all of it is
  const float A = isnan(st.x) ? NAN : -g - h * H, B = -h * kLn2;
  const float2 A2 = make_float2(A, A), B2 = make_float2(B, B), nm2 = make_float2(-st.x, -st.x);
  const float2 c2 = make_float2(a.c, a.c), nl2 = make_float2(-st.y * kLog2e, -st.y * kLog2e);
  for (; e0 < last; e0 += kChunk) {
    uint4 u[kGradUnroll];
#pragma unroll
    for (int k = 0; k < kGradUnroll; ++k) {
      const int e = e0 + k * kStep;
      if (e + E::VEC <= V)
        u[k] = __ldcs(reinterpret_cast<const uint4 *>(row + e));
      else if (e < V)
        u[k] = load_raw<E>(row, e, V);
    }
#pragma unroll
    for (int k = 0; k < kGradUnroll; ++k) {
      const int e = e0 + k * kStep;
      if (e >= last) break;
      float d[E::VEC];
#pragma unroll
      for (int i = 0; i < E::VEC / 2; ++i) {
        float2 t = __ffma2_rn(__fadd2_rn(pair_of<E>(u[k], i), nm2), c2, nl2);
        t = make_float2(fmaxf(t.x, kLeastT), fmaxf(t.y, kLeastT));
        const float2 v = __fmul2_rn(make_float2(ex2(t.x), ex2(t.y)), __ffma2_rn(t, B2, A2));
        d[2 * i] = v.x;
        d[2 * i + 1] = v.y;
      }
      if (a.g && (unsigned)(token - e) < (unsigned)E::VEC) {
        float x[E::VEC];
        unpack<E>(u[k], x);
#pragma unroll
        for (int j = 0; j < E::VEC; ++j)
          if (e + j == token) {
            const float z = (x[j] - st.x) * a.inv_t - st.y, t = fmaxf(z * kLog2e, kLeastT);
            d[j] = -g * expm1f(z) + ex2(t) * fmaf(t, B, A + g);
          }
      }
      if (e + E::VEC <= V)
        __stcs(reinterpret_cast<uint4 *>(out + e), pack<E>(d));
      else
        store_vec<E>(out, e, V, d);
    }
  }
}

}  // namespace

namespace {

template <class E, bool TOP, bool SPREAD>
umim_status launch_logprobs(LogprobArgs a, int C, cudaStream_t stream) {
  // a whole row's segments and the largest merge: with the kernel's own 6 KB below the 48 KB that need no leave
  static_assert(sizeof(float) * (kMaxLogitVocab / kSegment) + 8 * kMaxCluster * kMaxTop <= 42 * 1024 &&
                    kMaxLogitVocab % chunk_elems<E>() == 0, "shared memory");
  const size_t smem = TOP ? TopShared<E>::bytes(a.slice, a.n_top, C) : 0;
  trace_mark(stream, "logprobs.rows");
  const cudaError_t e = launch_pdl_cluster(token_logprobs_kernel<E, TOP, SPREAD>, dim3((unsigned)a.R * (unsigned)C),
                                           dim3(kThreads), (unsigned)C, smem, stream, a);
  trace_mark(stream, nullptr);
  return e == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

// Whether to spread a part over all warps.  Side by side, its first warps have eight strips each and the
// others nothing: that is less to do where few warps are busy, but only the busy ones' threads make groups, and the search
// needs half as many groups again as alternatives, or its threshold is the part's lowest element.  Past
// half a chunk the warps' unequal shares cost more.  Measured spread / side by side, us, bf16: 32768 rows of 2000 with 5, 20
// and 64 alternatives 421 / 337, 443 / 372 and 506 / 1698; 8192 of 8000 with 20, 64 and 128: 99.7 / 95.0, 118 / 119 and 137 / 698;
// 5461 of 12000 with 5 and 20: 64.0 / 66.1 and 66.9 / 69.7; 4096 of 16000, nearly a chunk, with 64: 61.1 / 60.7.
template <class E>
bool spread_pays(int slice, int n_top) {
  const int busy = ceil_div(slice, chunk_elems<E>() / kWarps);
  return slice < chunk_elems<E>() && (2 * slice > chunk_elems<E>() || 3 * n_top > 2 * 32 * busy);
}

template <class E>
umim_status launch_type(const LogprobArgs &a, int C, cudaStream_t stream) {
  if (a.n_top == 0) return launch_logprobs<E, false, false>(a, C, stream);
  return spread_pays<E>(a.slice, a.n_top) ? launch_logprobs<E, true, true>(a, C, stream)
                                          : launch_logprobs<E, true, false>(a, C, stream);
}

// CTAs per row: rows are divided while that leaves at most three CTAs to an SM, or two with
// alternatives, and a part is still worth one (2048 elements).  Measured for 152 rows of 128256 bf16 with 20
// alternatives: 14.2 us by two CTAs a row, 20.1 by four, which are all the places that the SMs have, so that some
// clusters may wait for others; for 200 rows of 32000: 7.5 by one, 10.0 by two; without
// alternatives, 200 rows of 128256: 14.5 by two, 16.2 by one.
int cluster_for(int R, int V, int n_top, int num_sms) {
  int C = 1;
  while (C < kMaxCluster && (int64_t)R * 2 * C <= (n_top > 0 ? 2 : 3) * num_sms && V / (2 * C) >= 2048) C *= 2;
  return C;
}

}  // namespace

umim_status token_logprobs(const void *logits, int dtype, int R, int V, int64_t ld, const int32_t *n_dev,
                           const int32_t *tokens, float temperature, int n_top, float *logprobs, float *entropy,
                           float *stats, int32_t *top_ids, float *top_logprobs, int32_t *dev_status,
                           cudaStream_t stream, int num_sms) {
  const int C = cluster_for(R, V, n_top, num_sms);
  const int slice = ceil_div(ceil_div(V, C), kSegment) * kSegment;
  const int ahead = C == 1 ? 4 * num_sms : 0;   // as many CTAs run at once
  const double inv = 1.0 / (double)temperature, c = 1.4426950408889634 * inv;
  const LogprobArgs a{logits, R, V, ld, n_dev, tokens, (float)inv, (float)c, (float)(inv - (float)inv),
                      (float)(c / (float)c - 1.0), n_top, slice, ahead, logprobs, entropy,
                      reinterpret_cast<float2 *>(stats), top_ids, top_logprobs, dev_status};
  return dtype == UMIM_DTYPE_BF16   ? launch_type<ElemBf16>(a, C, stream)
         : dtype == UMIM_DTYPE_FP16 ? launch_type<ElemFp16>(a, C, stream)
                                    : launch_type<ElemFp32>(a, C, stream);
}

constexpr int kGradChunks = 4, kGradCtas = 16;

umim_status token_logprobs_grad(const void *logits, int dtype, int R, int V, int64_t ld, const int32_t *n_dev,
                                const int32_t *tokens, float temperature, const float *stats, const float *entropy,
                                const float *g, const float *h, void *grad, int32_t *dev_status, cudaStream_t stream,
                                int num_sms) {
  const int vec = 16 / (int)dtype_bytes(dtype);
  const int row_chunks = ceil_div(V, kGradUnroll * kThreads * vec);
  const int chunks = (int)std::clamp<int64_t>((int64_t)R * row_chunks / (kGradCtas * num_sms), 1, kGradChunks);
  const int parts = ceil_div(row_chunks, chunks);
  const GradArgs a{logits, R, V, ld, n_dev, tokens, 1.f / temperature, kLog2e / temperature, parts, chunks,
                   reinterpret_cast<const float2 *>(stats), entropy, g, h, grad, dev_status};
  auto *k = dtype == UMIM_DTYPE_BF16   ? token_logprobs_grad_kernel<ElemBf16>
            : dtype == UMIM_DTYPE_FP16 ? token_logprobs_grad_kernel<ElemFp16>
                                       : token_logprobs_grad_kernel<ElemFp32>;
  trace_mark(stream, "logprobs.grad");
  const cudaError_t e = launch_pdl(k, dim3((unsigned)R * (unsigned)parts), dim3(kThreads), 0, stream, a);
  trace_mark(stream, nullptr);
  return e == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

}  // namespace umim
