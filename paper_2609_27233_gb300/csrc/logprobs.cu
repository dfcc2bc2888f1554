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
constexpr int kUnroll = 4;        // vectors of a thread in flight, and one chunk more
constexpr int kMaxCluster = 8;    // CTAs per row, at most

struct LogprobArgs {
  const void *logits;
  int32_t R, V;
  int64_t ld;
  const int32_t *n_dev;
  const int32_t *tokens;     // nullptr: no token, every row counts
  float inv_t, c;            // 1 / T, log2(e) / T
  int32_t n_top, slice;      // slice: elements of a row per CTA
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
  int32_t parts;             // CTAs per row
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

// s and w from the reference `from` to `to` >= from.  What underflows goes to 0, a NaN stays one.
__device__ __forceinline__ void rebase(Stats &a, float to, float c) {
  if (!(a.m == to)) {
    const float d = (a.m - to) * c, f = ex2(d), s = a.s;
    a.s = s * f;
    a.w = f > 0.f ? f * fmaf(s, d, a.w) : a.s;
    a.m = to;
  }
}

// the warp's statistics in every lane
__device__ __forceinline__ Stats warp_stats(Stats a, float c) {
  rebase(a, warp_max(a.m), c);
  const float2 v = warp_sum2(make_float2(a.s, a.w));
  a.s = v.x;
  a.w = v.y;
  return a;
}

// One thread's part: four vectors at a time.  t is one FMA, x c + b with
// b = -m c rounded; the rounding r is common to a chunk and made good on its
// sums, so that t is as exact for large |m| as (x - m) c.  Where r itself is large,
// or a -inf is met (0 times -inf is no number), the sums come out as no
// numbers and the chunk is done again the careful way; only NaN and +inf are
// left as NaN by that.
template <class E>
struct Running {
  Stats st = no_stats();
  float b = 0.f, r = 0.f, rf = 1.f;

  // again(k): vector k of the chunk, read a second time
  template <class Again>
  __device__ __forceinline__ void add(const uint4 (&u)[kUnroll], uint32_t max_word, float c, Again again) {
    const float cm = E::to_float(E::word_max_bits(max_word));
    if (cm > st.m) {
      rebase(st, cm, c);
      b = -cm * c;
      r = fmaf(-cm, c, -b);
      rf = ex2(r);
      if (!(fabsf(r) <= 1.f)) b = NAN;   // |m c| past 2^24, or no number: the careful way
    }
    const float2 c2 = make_float2(c, c), b2 = make_float2(b, b);
    float2 s0 = make_float2(0.f, 0.f), s1 = s0, w0 = s0, w1 = s0;
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
#pragma unroll
      for (int i = 0; i < E::VEC / 2; ++i) {
        const float2 t = __ffma2_rn(pair_of<E>(u[k], i), c2, b2);
        const float2 e = make_float2(ex2(t.x), ex2(t.y));
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
    if (s < INFINITY && w > -INFINITY) {
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
        t = t < -1000.f ? -1000.f : t;   // 2^t is 0 from -150 on; a NaN passes
        float e = ex2(t);
        st.s += e;
        st.w = fmaf(e, t, st.w);
        t = (x.y - m0) * c;
        t = t < -1000.f ? -1000.f : t;
        e = ex2(t);
        st.s += e;
        st.w = fmaf(e, t, st.w);
      }
    }
  }
};

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
// One cluster of C CTAs per row, each on one of C contiguous parts.  A warp
// takes chunks of 4 x 32 vectors, a lane one vector of each 32: every logit is
// read once, by 16-byte loads a chunk ahead of their use.
//
// The alternatives need no second pass over the row.  Beside the sums, the
// maximum of every segment of 32 consecutive elements goes to shared memory.
// The n largest elements (by value, then by lowest id) lie in the n largest
// segments (by maximum, then by lowest place): n segments before one that holds an
// element each have an element before it.  So the segments' maxima are searched
// for a threshold that n of them reach, and the few segments at or above
// it are read again (64 or 128 bytes each, from L2).
//
// The threshold is taken over 256 groups of segments, one a thread, since the
// n-th largest of the groups' maxima is a bound too: then about
// 256 ln(256 / (256 - n)) elements pass it (21 for n = 20, 177 for 128), and a
// thread each ranks them by counting.  Equal values can make them many more;
// then the same bisections that gave the threshold pick exactly n segments, and
// exactly n of their elements.
//
// All of it happens in shared memory and registers of the cluster: no
// workspace, no atomics on global memory, the same bits in every call.
constexpr int kSegment = 32;

template <class E>
struct TopShared {
  typename E::T *seg;      // [segments] maximum of each
  uint16_t *list;          // [segments] those at or above the threshold
  uint64_t *cand;          // [32 n] elements at or above it: (key, ~id)
  uint64_t *merge;         // rank 0: [C][n] every CTA's best, descending
  static size_t bytes(int slice, int n, int C) {
    const size_t segs = (size_t)ceil_div(slice, kSegment);
    return 8 * ((size_t)kSegment * n + (C > 1 ? (size_t)C * n : 0)) + (sizeof(typename E::T) + 2) * segs;
  }
  __device__ TopShared(uint8_t *p, int slice, int n, int C) {
    const int segs = ceil_div(slice, kSegment);
    cand = reinterpret_cast<uint64_t *>(p);
    merge = cand + kSegment * n;
    seg = reinterpret_cast<typename E::T *>(merge + (C > 1 ? C * n : 0));
    list = reinterpret_cast<uint16_t *>(seg + segs);
  }
};

// The largest k in [lo, hi] that at least n entries reach (lo where fewer reach it);
// count(k): how many do, the same in every thread.
template <class Count>
__device__ uint32_t largest_reached(uint32_t lo, uint32_t hi, int n, Count count) {
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    if (count(mid) >= n)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// how many of M entries, held by the CTA's threads in turn, satisfy pred
template <class Pred>
__device__ int count_entries(int M, Pred pred) {
  int c = 0;
  for (int i = threadIdx.x; i - (int)threadIdx.x < M; i += kThreads) c += __syncthreads_count(i < M && pred(i));
  return c;
}

// Exactly the n first of M > n entries by (key descending, id ascending), as a key and the
// largest id that is still in at that key; ids are below `ids`.
struct Cut {
  uint32_t key, id;
  __device__ bool in(uint32_t k, uint32_t i) const { return k > key || (k == key && i <= id); }
};
template <class Key, class Id>
__device__ Cut cut_at(int M, int n, uint32_t lo, uint32_t hi, uint32_t ids, Key key, Id id) {
  Cut c;
  c.key = largest_reached(lo, hi, n, [&](uint32_t k) { return count_entries(M, [&](int i) { return key(i) >= k; }); });
  const int left = n - count_entries(M, [&](int i) { return key(i) > c.key; });
  // the smallest id with `left` equal entries at or below it
  uint32_t a = 0, b = ids - 1;
  while (a < b) {
    const uint32_t mid = (a + b) / 2;
    if (count_entries(M, [&](int i) { return key(i) == c.key && id(i) <= mid; }) >= left)
      b = mid;
    else
      a = mid + 1;
  }
  c.id = a;
  return c;
}

__device__ __forceinline__ uint32_t key_of(uint64_t e) { return (uint32_t)(e >> 32); }
__device__ __forceinline__ uint32_t id_of(uint64_t e) { return ~(uint32_t)e; }

// This CTA's n best elements of row[beg, end), best first, to sorted[]: (key, ~id); sorted[0, n) comes in as zeros.
// Neither NaN nor +inf is among them.
template <class E>
__device__ void best_of_slice(const TopShared<E> &sh, const typename E::T *row, int beg, int end, int n,
                              uint64_t *sorted, int32_t *status) {
  __shared__ uint32_t s_hi[kWarps], s_lo[kWarps];
  __shared__ int s_listed, s_held, s_kept;
  __shared__ uint64_t s_keep[kMaxTop];
  const int tid = threadIdx.x, segs = ceil_div(end - beg, kSegment);
  const uint32_t none = E::order_key(E::kNegInf);
  const auto seg_key = [&](int i) { return E::order_key(sh.seg[i]); };

  // a group of segments per thread; lanes start at different places of theirs (banks)
  const int G = ceil_div(segs, kThreads), g0 = min(tid * G, segs), gn = min(G, segs - g0);
  uint32_t group = none;
  for (int j = 0, k = gn > 0 ? tid % gn : 0; j < gn; ++j) {
    group = max(group, seg_key(g0 + k));
    k = k + 1 == gn ? 0 : k + 1;
  }
  {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, group), lo = __reduce_min_sync(0xffffffffu, group);
    if ((tid & 31) == 0) {
      s_hi[tid >> 5] = hi;
      s_lo[tid >> 5] = lo;
    }
    if (tid == 0) s_listed = s_held = s_kept = 0;
  }
  __syncthreads();
  uint32_t hi = s_hi[0], lo = s_lo[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) {
    hi = max(hi, s_hi[i]);
    lo = min(lo, s_lo[i]);
  }
  if (hi == none) return;   // nothing above -inf (the same in every thread)
  lo = max(lo, none + 1);
  const uint32_t least =
      largest_reached(lo, hi, n, [&](uint32_t k) { return __syncthreads_count(group >= k); });

  if (group >= least)
    for (int j = 0; j < gn; ++j)
      if (seg_key(g0 + j) >= least) sh.list[atomicAdd(&s_listed, 1)] = (uint16_t)(g0 + j);
  __syncthreads();
  const int listed = s_listed;

  // the elements at or above `from` of the listed segments that `in` takes
  constexpr int kVecs = kSegment / E::VEC;
  const auto gather = [&](uint32_t from, auto in) {
    for (int i = tid; i < listed * kVecs; i += kThreads) {
      const int seg = sh.list[i / kVecs];
      if (!in_bounds(seg, segs, status, kSiteLogprobSegment) || !in(seg)) continue;
      const int e = beg + seg * kSegment + (i % kVecs) * E::VEC;
      if (e >= end) continue;
      const uint4 u = load_raw<E>(row, e, end);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int j = 0; j < E::VEC; ++j) {
        typename E::T x;
        if constexpr (E::VEC == 8)
          x = (typename E::T)(w[j / 2] >> (16 * (j & 1)));
        else
          x = __uint_as_float(w[j]);
        const uint32_t k = E::order_key(x);
        if (k >= from && e + j < end) {
          const int at = atomicAdd(&s_held, 1);
          if (at < kSegment * n) sh.cand[at] = ((uint64_t)k << 32) | (uint32_t)~(uint32_t)(e + j);
        }
      }
    }
    __syncthreads();
  };
  gather(least, [](int) { return true; });
  if (s_held > kSegment * n) {   // many equal ones: n segments exactly
    const Cut cut = cut_at(listed, n, least, hi, (uint32_t)segs, [&](int i) { return seg_key(sh.list[i]); },
                           [&](int i) { return (uint32_t)sh.list[i]; });
    if (tid == 0) s_held = 0;
    __syncthreads();
    gather(cut.key, [&](int seg) { return cut.in(seg_key(seg), (uint32_t)seg); });
  }
  const uint64_t *best = sh.cand;
  int M = min(s_held, kSegment * n);
  if (M > kThreads) {            // more than a thread each: n elements exactly
    const Cut cut = cut_at(M, n, least, hi, (uint32_t)end, [&](int i) { return key_of(sh.cand[i]); },
                           [&](int i) { return id_of(sh.cand[i]); });
    for (int i = tid; i < M; i += kThreads)
      if (cut.in(key_of(sh.cand[i]), id_of(sh.cand[i]))) {
        const int at = atomicAdd(&s_kept, 1);
        if (in_bounds(at, kMaxTop, status, kSiteLogprobRank)) s_keep[at] = sh.cand[i];
      }
    __syncthreads();
    best = s_keep;
    M = s_kept;
  }
  if (tid < M) {
    const uint64_t mine = best[tid];
    int rank = 0;
    for (int i = 0; i < M; ++i) rank += best[i] > mine;
    if (rank < n) sorted[rank] = mine;
  }
}

template <class E, bool TOP>
__global__ void __launch_bounds__(kThreads, 4) token_logprobs_kernel(LogprobArgs a) {
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ Stats s_warp[kWarps], s_cta[kMaxCluster];
  __shared__ uint64_t s_sorted[kMaxTop];
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
  float x_t = 0.f;
  if (rank == 0 && tid == 0) x_t = E::to_float(row[token]);

  // ---- one pass over this CTA's part ----
  constexpr int kChunk = kUnroll * 32 * E::VEC;   // elements of a warp's chunk
  const float c = a.c;
  Running<E> run;
  uint4 u[kUnroll], next[kUnroll];
  const auto load = [&](uint4 (&v)[kUnroll], int e0) {   // chunk at element e0
    if (e0 + kChunk <= end) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        v[k] = __ldcs(reinterpret_cast<const uint4 *>(row + e0 + (k * 32 + lane) * E::VEC));
    } else if (e0 < end) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) v[k] = load_raw<E>(row, e0 + (k * 32 + lane) * E::VEC, end);
    }
  };
  int e0 = beg + warp * kChunk;
  load(next, e0);
  for (; e0 < end; e0 += kWarps * kChunk) {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) u[k] = next[k];
    load(next, e0 + kWarps * kChunk);
    uint32_t top[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
      top[k] = E::max_words(E::max_words(u[k].x, u[k].y), E::max_words(u[k].z, u[k].w));
    if constexpr (TOP) {
      // The maxima of four neighbouring lanes' vectors, transposed: a lane ends up with
      // that of its four for vector lane % 4.
      static_assert(kUnroll == 4, "four vectors among four lanes");
      const bool odd = lane & 1, high = lane & 2;
      uint32_t p = E::max_words(odd ? top[1] : top[0], __shfl_xor_sync(0xffffffffu, odd ? top[0] : top[1], 1));
      uint32_t q = E::max_words(odd ? top[3] : top[2], __shfl_xor_sync(0xffffffffu, odd ? top[2] : top[3], 1));
      uint32_t v = E::max_words(high ? q : p, __shfl_xor_sync(0xffffffffu, high ? p : q, 2));
      const int vec = (lane & 3) * 32 + (lane & ~3);   // the first of the four in the chunk
      int at = (e0 - beg + vec * E::VEC) / kSegment;
      if (E::VEC == 4) v = E::max_words(v, __shfl_xor_sync(0xffffffffu, v, 4));   // eight lanes make a segment
      if ((E::VEC == 8 || !(lane & 4)) && at < ceil_div(end - beg, kSegment)) sh.seg[at] = E::word_max_bits(v);
    }
    run.add(u, E::max_words(E::max_words(top[0], top[1]), E::max_words(top[2], top[3])), c,
            [&](int k) { return load_raw<E>(row, e0 + (k * 32 + lane) * E::VEC, end); });
  }

  // ---- the CTA's sums and alternatives ----
  const Stats ws = warp_stats(run.st, c);
  if (lane == 0) s_warp[warp] = ws;
  __syncthreads();
  Stats cta = lane < kWarps ? s_warp[lane] : no_stats();
  cta = warp_stats(cta, c);
  if constexpr (TOP) {
    for (int i = tid; i < n; i += kThreads) s_sorted[i] = 0;
    // NaN and +inf have no place in the order, and a row that holds one has no alternatives
    if (cta.s < INFINITY) best_of_slice<E>(sh, row, beg, end, n, s_sorted, a.status);
    __syncthreads();
  }
  if (C > 1) {   // to rank 0
    cluster_sync_all();   // every CTA of the cluster runs
    if (tid == 0) {
      const uint32_t to = peer_addr(&s_cta[rank], 0);
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(cta.m) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4), "f"(cta.s) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 8), "f"(cta.w) : "memory");
    }
    for (int i = tid; i < n; i += kThreads)
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(peer_addr(&sh.merge[rank * n + i], 0)), "l"(s_sorted[i])
                   : "memory");
    cluster_sync_all();
    if (rank != 0) return;
    cta = lane < C ? s_cta[lane] : no_stats();
    cta = warp_stats(cta, c);
    if constexpr (TOP) {   // every entry's place among the C lists
      for (int i = tid; i < n; i += kThreads) s_sorted[i] = 0;
      __syncthreads();
      for (int i = tid; i < C * n; i += kThreads) {
        const uint64_t mine = sh.merge[i];
        int place = i % n;
        for (int l = 0; l < C && mine; ++l) {
          if (l == i / n) continue;
          int lo = 0, hi = n;   // entries of list l before mine
          while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (sh.merge[l * n + mid] > mine)
              lo = mid + 1;
            else
              hi = mid;
          }
          place += lo;
        }
        if (mine && place < n) s_sorted[place] = mine;
      }
      __syncthreads();
    }
  }

  // ---- outputs ----
  const bool bad = !(cta.s < INFINITY), empty = cta.m == -INFINITY && !bad;
  const float m0 = empty ? 0.f : cta.m, l = bad ? NAN : empty ? 0.f : logf(cta.s);
  if (tid == 0) {
    if (a.logprobs) a.logprobs[r] = bad ? NAN : (x_t - m0) * a.inv_t - l;
    if (a.entropy) a.entropy[r] = bad ? NAN : empty ? 0.f : l - kLn2 * (cta.w / cta.s);
    if (a.stats) a.stats[r] = bad ? make_float2(NAN, NAN) : make_float2(cta.m, l);
  }
  for (int i = tid; i < n; i += kThreads) {
    const uint64_t e = bad ? 0 : s_sorted[i];
    a.top_ids[(int64_t)r * n + i] = e ? (int)id_of(e) : -1;
    a.top_logprobs[(int64_t)r * n + i] =
        bad ? NAN : e ? (E::to_float(E::from_key(key_of(e))) - m0) * a.inv_t - l : -INFINITY;
  }
}

// ---------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------
// Elementwise, bound by its one read and one write of every element.  A CTA takes
// kGradChunks chunks of a row: 4 vectors a thread, loaded together and ahead of the
// row's numbers.  With t = log2 p the element is p (A + B t), A = -(g + h H) / T and
// B = -h ln 2 / T; the token's own is -g expm1(ln p) / T + p (A + g / T + B t), exact
// where p is so near 1 that 1 - p would be nothing.
constexpr int kGradChunks = 2;

template <class E>
__global__ void __launch_bounds__(kThreads, 4) token_logprobs_grad_kernel(GradArgs a) {
  griddep_wait();
  griddep_launch();
  const int r = blockIdx.x / a.parts, V = a.V;
  if (r >= rows_used(a.n_dev, a.R)) return;
  const typename E::T *row = static_cast<const typename E::T *>(a.logits) + (int64_t)r * a.ld;
  typename E::T *out = static_cast<typename E::T *>(a.grad) + (int64_t)r * a.ld;
  constexpr int kStep = kThreads * E::VEC, kChunk = kUnroll * kStep;
  int e0 = (blockIdx.x % a.parts) * (kGradChunks * kChunk) + threadIdx.x * E::VEC;
  const int last = min(V, (int)(blockIdx.x % a.parts + 1) * (kGradChunks * kChunk));

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
    uint4 u[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int e = e0 + k * kStep;
      if (e + E::VEC <= V)
        u[k] = __ldcs(reinterpret_cast<const uint4 *>(row + e));
      else if (e < V)
        u[k] = load_raw<E>(row, e, V);
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int e = e0 + k * kStep;
      if (e >= last) break;
      float d[E::VEC];
#pragma unroll
      for (int i = 0; i < E::VEC / 2; ++i) {
        float2 t = __ffma2_rn(__fadd2_rn(pair_of<E>(u[k], i), nm2), c2, nl2);
        t = make_float2(fmaxf(t.x, -1000.f), fmaxf(t.y, -1000.f));   // of -inf: 0 times it would be no number
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
            const float z = (x[j] - st.x) * a.inv_t - st.y, t = fmaxf(z * kLog2e, -1000.f);
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

template <class E, bool TOP>
umim_status launch_logprobs(LogprobArgs a, int C, cudaStream_t stream) {
  const size_t smem = TOP ? TopShared<E>::bytes(a.slice, a.n_top, C) : 0;
  if (TOP && !allow_smem(token_logprobs_kernel<E, TOP>, TopShared<E>::bytes(kMaxLogitVocab, kMaxTop, kMaxCluster)))
    return UMIM_ERR_CUDA;
  trace_mark(stream, "logprobs.rows");
  const cudaError_t e = launch_pdl_cluster(token_logprobs_kernel<E, TOP>, dim3((unsigned)a.R * (unsigned)C),
                                           dim3(kThreads), (unsigned)C, smem, stream, a);
  trace_mark(stream, nullptr);
  return e == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

// CTAs per row: enough that the SMs hold four each, where a part is still worth a CTA (2048 elements).
int cluster_for(int R, int V, int num_sms) {
  int C = 1;
  while (C < kMaxCluster && (int64_t)R * C < 4 * num_sms && V / (2 * C) >= 2048) C *= 2;
  return C;
}

}  // namespace

umim_status token_logprobs(const void *logits, int dtype, int R, int V, int64_t ld, const int32_t *n_dev,
                           const int32_t *tokens, float temperature, int n_top, float *logprobs, float *entropy,
                           float *stats, int32_t *top_ids, float *top_logprobs, int32_t *dev_status,
                           cudaStream_t stream, int num_sms) {
  const int C = cluster_for(R, V, num_sms);
  const int slice = ceil_div(ceil_div(V, C), kSegment) * kSegment;
  const LogprobArgs a{logits, R, V, ld, n_dev, tokens, 1.f / temperature, kLog2e / temperature, n_top, slice,
                      logprobs, entropy, reinterpret_cast<float2 *>(stats), top_ids, top_logprobs, dev_status};
  if (n_top > 0)
    return dtype == UMIM_DTYPE_BF16   ? launch_logprobs<ElemBf16, true>(a, C, stream)
           : dtype == UMIM_DTYPE_FP16 ? launch_logprobs<ElemFp16, true>(a, C, stream)
                                      : launch_logprobs<ElemFp32, true>(a, C, stream);
  return dtype == UMIM_DTYPE_BF16   ? launch_logprobs<ElemBf16, false>(a, C, stream)
         : dtype == UMIM_DTYPE_FP16 ? launch_logprobs<ElemFp16, false>(a, C, stream)
                                    : launch_logprobs<ElemFp32, false>(a, C, stream);
}

umim_status token_logprobs_grad(const void *logits, int dtype, int R, int V, int64_t ld, const int32_t *n_dev,
                                const int32_t *tokens, float temperature, const float *stats, const float *entropy,
                                const float *g, const float *h, void *grad, int32_t *dev_status, cudaStream_t stream) {
  const int vec = 16 / (int)dtype_bytes(dtype);
  const int parts = ceil_div(V, kGradChunks * kUnroll * kThreads * vec);
  const GradArgs a{logits, R, V, ld, n_dev, tokens, 1.f / temperature, kLog2e / temperature, parts,
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
