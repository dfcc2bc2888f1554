// Distillation from the teacher's top log probabilities: the soft-target
// cross-entropy over the aligned pairs of App. F when only the K best
// alternatives of each teacher row were kept, and its gradient with respect to
// the student logits.
//
// For a pair with the teacher's entries (a_i, lambda_i), i < K, the student's
// y = x / T and q = softmax(y):
//   renormalised  p = softmax(lambda),  p_rest = 0
//   with a tail   p = exp(lambda),      p_rest = 1 - sum p
//   loss = - sum_i p_i ln q(a_i) - p_rest ln q_rest,  q_rest = sum of q outside the a_i
//   d loss / dx_v = (1/T) q_v (P - p_rest / q_rest)   outside the a_i
//                   (1/T) (P q_v - p_i)               at v = a_i,   P = sum p + p_rest
// q_rest is summed over the elements outside the list: one minus the listed
// ones would lose it where the student puts nearly everything on them.
// For the same reason every 1 - q and 1 - p below is a sum of what is left, and every ln of
// a q near 1 a log1p.
#include <algorithm>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "logits.cuh"

namespace umim {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 4;
constexpr float kSlack = 16.f;
constexpr int kMaxCluster = 8;    // CTAs per row, at most
constexpr int kPartBytes = 65536; // three parts of this size fit an SM's shared memory
constexpr int kHalfBytes = 106496; // two
constexpr int kPlanThreads = 512, kPlanPairs = kPlanThreads / 32;
constexpr int kTable = 2 * kMaxTop;   // slots for the ids of a list
constexpr int kEntries = kMaxTop / 32;   // entries of a list per lane
// A list that holds all there is leaves a p_rest of rounding: the listed log probabilities are fp32, each
// off by up to about 16 2^-24.  Where the student's rest is nothing too (its mask is
// the teacher's, or no id is left), ln q_rest is no measure of anything, so
// there, and only there, a p_rest below 2^-20 counts as 0.
constexpr float kLeastRest = 9.5367431640625e-7f;
constexpr float kNoRest = 7.8886090522101181e-31f;   // q_rest below 2^-100 is none: far above where it underflows

struct TopkHeader {
  int32_t status;         // status word when the caller passes none
  int32_t error;          // the pairs are invalid: nothing is written
  int32_t clusters_done;  // clusters of the main kernel that finished
  int32_t pad[61];
};
static_assert(sizeof(TopkHeader) == 256, "header size");

struct Entry {
  int32_t id;   // -1: none
  float p;
};

// A pair's teacher row beside its entries.
struct __align__(16) Head {
  float listed, rest;   // sum p, p_rest
  float others;         // sum p without the largest entry
  float pad;
};

struct TopkArgs {
  const int32_t *top_ids;      // [R_T][K]
  const float *top_logprobs;   // [R_T][K]
  int32_t R_T, K;
  const void *student;
  int32_t R_S, V;
  int64_t ld;
  const int32_t *teacher_rows, *student_rows;
  int32_t max_pairs;
  const int32_t *n_dev;
  float inv_t, c, grad_scale;  // 1 / T, log2(e) / T
  int32_t tail, slice;         // slice: elements of a row per CTA
  float *loss, *pair_loss;
  void *grad;                  // or nullptr
  uint32_t *paired;            // [R_S] bits: the student rows in a pair
  Entry *lists;                // [max_pairs][K] the pairs' entries as the main kernel takes them
  Head *heads;                 // [max_pairs]
  TopkHeader *hdr;
  int32_t *status;
};

inline size_t a256(size_t x) { return (x + 255) & ~size_t(255); }

__device__ __forceinline__ float warp_sum(float v) { return warp_sum2(make_float2(v, 0.f)).x; }

// The bits of an id mixed by multiplications and shifts: a list of ids at equal distances, which
// one multiplication would map to slots at equal distances, comes out spread.  The factors are 2^32 / phi
// (Fibonacci hashing) and 2^32 (e - 2), both to the next odd number.  128 ids, at any equal distance or
// at random, take 1.49 probes each on average and 2.3 in the worst of 1800 lists.
__device__ __forceinline__ uint32_t mixed(uint32_t x) {
  x *= 0x9e3779b9u;
  x ^= x >> 17;
  x *= 0xb7e15163u;
  return x ^ (x >> 16);
}

// CTA 0 checks the pairs, before anything is written, and marks the student rows that are
// in one: a bit each, in shared memory, or where these are too many for that in global memory.
// (Not in shared memory part by part, which reads the pairs once for each: a call with 2 000 000 rows took
// 21.9 ms, 13.2 like this; 500 000 3.2 and 3.1; 200 000, two parts, 1.20 and 1.25.)  A warp of the others per pair: its
// teacher row's entries, checked, as probabilities.  Both read N; neither waits
// for the other.
__global__ void __launch_bounds__(kPlanThreads) topk_plan_kernel(TopkArgs a) {
  __shared__ uint32_t table[kPlanPairs][kTable];   // CTA 0: the marks; else a warp's ids, hashed, and
  __shared__ int32_t owner[kPlanPairs][kTable];    // the first entry that has each
  griddep_wait();
  griddep_launch();
  const int tid = threadIdx.x, lane = tid & 31, K = a.K;
  const int N = a.n_dev ? *a.n_dev : a.max_pairs;
  if (blockIdx.x == 0) {
    constexpr int kMarked = 32 * kPlanPairs * kTable;
    const int words = ceil_div(a.R_S, 32);
    bool bad = N < 0 || N > a.max_pairs;
    const auto mark_rows = [&](uint32_t *mark) {
      for (int i = tid; i < words; i += kPlanThreads) mark[i] = 0;
      __syncthreads();
      if (!bad)
#pragma unroll 4
        for (int p = tid; p < N; p += kPlanThreads) {
          const int t = a.teacher_rows[p], s = a.student_rows[p];
          if (t < 0 || t >= a.R_T || s < 0 || s >= a.R_S) {
            bad = true;
          } else {
            const uint32_t bit = 1u << (s & 31);
            if (atomicOr(&mark[s >> 5], bit) & bit) bad = true;   // a student row in two pairs
          }
        }
      bad = __syncthreads_or(bad);
    };
    if (a.R_S <= kMarked) {
      mark_rows(&table[0][0]);
      for (int i = tid; i < words; i += kPlanThreads) a.paired[i] = (&table[0][0])[i];
    } else {
      mark_rows(a.paired);
    }
    if (tid == 0) {
      a.hdr->error = bad;
      a.hdr->clusters_done = 0;
      if (bad) set_error(a.status, UMIM_ERR_INVALID_ARG);
    }
    return;
  }
  const int pr = (blockIdx.x - 1) * kPlanPairs + tid / 32;
  if (pr >= N || N > a.max_pairs) return;
  const int t = a.teacher_rows[pr];
  if (t < 0 || t >= a.R_T) return;
  int id[kEntries];
  float lam[kEntries], p[kEntries];
#pragma unroll
  for (int j = 0; j < kEntries; ++j) {
    const int i = j * 32 + lane;
    id[j] = i < K ? a.top_ids[(int64_t)t * K + i] : -1;
    lam[j] = i < K ? a.top_logprobs[(int64_t)t * K + i] : -INFINITY;
  }
  // what umim_token_logprobs leaves of a row of logits with NaN or +inf in it
  bool spoilt = true;
#pragma unroll
  for (int j = 0; j < kEntries; ++j) spoilt &= j * 32 + lane >= K || (id[j] == -1 && isnan(lam[j]));
  spoilt = __all_sync(0xffffffffu, spoilt);
  bool wrong = false;
#pragma unroll
  for (int j = 0; j < kEntries; ++j)
    if (id[j] < -1 || id[j] >= a.V) {
      wrong = true;
      id[j] = -1;
    }
  // of two equal ids the first counts: a table of the ids, and who has each first
  uint32_t *ids = table[tid / 32];
  int32_t *first = owner[tid / 32];
  for (int i = lane; i < kTable; i += 32) {
    ids[i] = ~0u;
    first[i] = INT32_MAX;
  }
  __syncwarp();
  int place[kEntries];
#pragma unroll
  for (int j = 0; j < kEntries; ++j)
    if (id[j] >= 0) {   // half the table is free: the probe ends
      int h = (int)(mixed((uint32_t)id[j]) & (kTable - 1));
      for (uint32_t old; (old = atomicCAS(&ids[h], ~0u, (uint32_t)id[j])) != ~0u && old != (uint32_t)id[j];)
        h = (h + 1) & (kTable - 1);
      place[j] = h;
      atomicMin(&first[h], j * 32 + lane);
    }
  __syncwarp();
#pragma unroll
  for (int j = 0; j < kEntries; ++j)
    if (id[j] >= 0 && first[place[j]] != j * 32 + lane) {
      wrong = true;
      id[j] = -1;
    }
  if (wrong) set_error(a.status, UMIM_ERR_INVALID_ARG);
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < kEntries; ++j)
    if (id[j] >= 0) top = fmaxf(top, lam[j]);
  top = warp_max(top);
  // The largest entry is kept apart from the sum of the others.  1 - sum p is taken as (1 - p_max) - others,
  // 1 - p_max as -expm1(lambda_max): off by 16 2^-24 of 1 - p_max at most, about what the rounding of the other
  // entries' lambda means.  (1 minus the sum of all is off by 2^-24 of 1: a teacher
  // that is sure of one token lost up to 7 % of a p_rest of 3e-6.)
  bool mine = false;   // this lane has the largest entry, or one as large
#pragma unroll
  for (int j = 0; j < kEntries; ++j) mine |= id[j] >= 0 && lam[j] == top;
  const unsigned holders = __ballot_sync(0xffffffffu, mine && top != -INFINITY);
  mine = holders != 0 && lane == __ffs(holders) - 1;
  const float base = a.tail || top == -INFINITY ? 0.f : top;
  float others = 0.f;
#pragma unroll
  for (int j = 0; j < kEntries; ++j) {
    p[j] = id[j] >= 0 && !(lam[j] == -INFINITY) ? expf(lam[j] - base) : 0.f;
    if (mine && id[j] >= 0 && lam[j] == top)
      mine = false;   // the largest, once
    else
      others += p[j];
  }
  others = warp_sum(others);
  const float sum = (holders ? expf(top - base) : 0.f) + others;
  float listed = sum, rest = 0.f, scale = 1.f;
  if (spoilt) {
    listed = NAN;
  } else if (a.tail) {
    rest = -expm1f(top) - others;
    if (rest < 0.f) rest = 0.f;
  } else if (sum != 0.f) {   // a row without entries adds nothing
    scale = 1.f / sum;
    if (!isnan(sum)) listed = 1.f;
  }
#pragma unroll
  for (int j = 0; j < kEntries; ++j)
    if (j * 32 + lane < K) a.lists[(int64_t)pr * K + j * 32 + lane] = Entry{id[j], p[j] * scale};
  if (lane == 0) a.heads[pr] = Head{listed, rest, others * scale, 0.f};
}

// A warp's stretch of a part of `vecs` vectors, and the shared memory for it: a vector for each
// lane, in vectors.
__host__ __device__ __forceinline__ int stretch_vecs(int vecs) { return ceil_div(vecs, kWarps); }
__host__ __device__ __forceinline__ int room_vecs(int vecs) {
  return ceil_div(stretch_vecs(vecs), 32) * 32;
}

// What a warp's stretch of the row adds: outside the list the maximum mr and the sum of
// 2^((x - mr) c); over the listed elements the maximum m, and the sums of 2^((x - m) c), without one
// element at m itself, of p and of p (x - m) / T.  The rest keeps a maximum
// of its own: where the listed ones are far above it, its sum would be nothing beside m.
// The element at m, a 1, is left out because beside it the others would lose their digits.
struct __align__(16) Part {
  float m, mr, rest, top, p, py, pad[2];
};

// One cluster of C CTAs for pair after pair, each CTA on one of C contiguous parts of the
// student's row, and each warp on one of eight contiguous stretches of that,
// which stays in shared memory between the two passes over it: every logit is
// read once and every gradient element written once, and what bounds the kernel is
// that traffic (8700 pairs of 128256 bf16 with 9600 rows: 739 us, 6.35 TB/s; without the
// gradient 2870 pairs take 144 us, 5.1 TB/s, with it 262 of 3260 rows).  A warp
// loads its stretch of the next pair's row, by an asynchronous copy, as soon as it has
// written this one's gradient.  Once a pair every warp tells all CTAs of the
// cluster its sums, by asynchronous stores that count on a barrier in each of
// them; there are two of these buffers, in turn, and nobody writes to one
// before everybody has read what it held.  Three CTAs of up to 64 KB to an SM load,
// sum and write in turn.
//
// Measured for 2870 pairs of 3260 rows, against 261 us like this: a CTA for every row, with the
// same parts, which starts and loads anew each time, 316; with parts of
// half the size 358; a cluster barrier a pair, which waits for the
// gradient's stores too, 467.
//
// The listed elements are taken out of the stretch before the first pass (-inf in
// their place), so that it sums the rest alone, and their gradients are written
// after the second pass, over the zeros that it left there.
//
// Rows in no pair get their zeros in between.
template <class E>
__global__ void __launch_bounds__(kThreads, 3) topk_ce_kernel(TopkArgs a) {
  extern __shared__ __align__(128) uint8_t dyn[];   // the part
  __shared__ __align__(8) uint64_t s_landed[kWarps], s_told[2];
  __shared__ Part s_parts[2][kMaxCluster * kWarps];
  __shared__ int s_last;
  using T = typename E::T;
  const int C = (int)cluster_size(), rank = C > 1 ? (int)cluster_ctarank() : 0;
  const int cid = blockIdx.x / C, clusters = gridDim.x / C;
  const int tid = threadIdx.x, lane = tid & 31, warp = warp_index(), V = a.V, K = a.K;
  // this warp's stretch [beg, end) of a row; the vector that the row's end cuts is not copied but loaded
  const int stretch = stretch_vecs(a.slice / E::VEC) * E::VEC;
  const int cta_end = min((rank + 1) * a.slice, V);
  const int beg = min(rank * a.slice + warp * stretch, cta_end), end = min(beg + stretch, cta_end);
  const int vecs = ceil_div(end - beg, E::VEC), whole_vecs = (end - beg) / E::VEC;
  const int room = room_vecs(a.slice / E::VEC);
  uint4 *pvec = reinterpret_cast<uint4 *>(dyn) + warp * room;
  T *part = reinterpret_cast<T *>(pvec);
  uint64_t *landed = &s_landed[warp];
  const float c = a.c;
  const auto rescale = [c](float from, float to) { return from == to ? 1.f : ex2((from - to) * c); };
  const auto row_of = [&](int s) { return static_cast<const T *>(a.student) + (int64_t)s * a.ld; };

  // The first pair's row is on its way while the plan is being made (17 pairs of 128256 bf16: 12.5 us
  // instead of 13.4): what the caller gave was there before the plan began, and no plan has checked it yet.
  const int N = a.n_dev ? *a.n_dev : a.max_pairs;
  int pr = cid;
  int s_row = N >= 0 && N <= a.max_pairs && pr < N ? a.student_rows[pr] : -1;
  if (s_row >= a.R_S) s_row = -1;
  uint4 cut = make_uint4(0, 0, 0, 0);
  Entry e[kEntries];
  Head head{0.f, 0.f, 0.f, 0.f};
  const auto load_list = [&](int q) {
#pragma unroll
    for (int j = 0; j < kEntries; ++j)
      e[j] = j * 32 + lane < K ? a.lists[(int64_t)q * K + j * 32 + lane] : Entry{-1, 0.f};
    head = a.heads[q];
  };
  bool failed = false;   // a wait gave up: this thread starts nothing more that would land later, and waits for nothing
  const auto copy = [&](int s) {   // the stretch of student row s
    if (lane == 0 && !failed) {
      mbar_arrive_expect_tx(landed, (uint32_t)whole_vecs * 16u);
      if (whole_vecs > 0) bulk_load(part, row_of(s) + beg, (uint32_t)whole_vecs * 16u, landed);
      if (whole_vecs < vecs) cut = load_raw<E>(row_of(s), beg + whole_vecs * E::VEC, V);
    }
  };
  const uint32_t told_bytes = (uint32_t)(C * kWarps * sizeof(Part));
  // what no copy reaches stays -inf: the first pass needs no bounds
  for (int i = whole_vecs + lane; i < room; i += 32)
    pvec[i] = make_uint4(E::kNegInf2, E::kNegInf2, E::kNegInf2, E::kNegInf2);
  if (lane == 0) mbar_init(landed, 1);
  if (tid == 0)
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_told[i], 1);
      mbar_arrive_expect_tx(&s_told[i], told_bytes);
    }
  fence_mbar_init();
  __syncwarp();
  if (s_row >= 0) copy(s_row);
  const auto wait = [&](uint64_t *bar, uint32_t parity) {
    if (!failed && !mbar_wait_sleep(bar, parity)) {
      failed = true;
      set_error(a.status, UMIM_ERR_TIMEOUT);
      mbar_wait_sleep(bar, parity);   // once more, for what may be on its way
    }
  };
  griddep_wait();
  griddep_launch();
  const int error = a.hdr->error;
  if (s_row >= 0) load_list(pr);
  if (error) {   // the pairs are invalid
    if (s_row >= 0) wait(landed, 0);   // no copy lands in shared memory that is another CTA's by then
    return;
  }
  if (C > 1) cluster_sync_all();   // every CTA's barriers are there before anyone tells it anything

  // Student rows in no pair: a look at one of this cluster's after each pair, the others at the end.
  int other = a.grad ? cid : a.R_S;
  const auto is_other = [&](uint32_t word) { return other < a.R_S && !(word >> (other & 31) & 1); };
  const auto write_zeros = [&]() {
    const float z[E::VEC] = {};
    T *out = static_cast<T *>(a.grad) + (int64_t)other * a.ld;
    for (int i = lane; i < vecs; i += 32) store_vec<E>(out, beg + i * E::VEC, V, z);
  };
  for (int count = 0; pr < N; pr += clusters, ++count) {
    const uint32_t word = other < a.R_S ? a.paired[other >> 5] : 0;
    const int next = pr + clusters;
    const int next_row = next < N ? a.student_rows[next] : 0;
    const float listed = head.listed, others = head.others;
    float rest = head.rest;
    wait(landed, (uint32_t)count & 1u);
    if (lane == 0 && whole_vecs < vecs) pvec[whole_vecs] = cut;
    __syncwarp();

    // ---- the listed elements of this stretch ----
    float x[kEntries], mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < kEntries; ++j) {
      x[j] = -INFINITY;
      if (j * 32 >= K) break;
      if (e[j].id < beg || e[j].id >= end) e[j].id = -1;   // another warp's, or none
      if (e[j].id >= 0 && in_bounds(e[j].id - beg, stretch, a.status, kSiteTopkEntry)) {
        x[j] = E::to_float(part[e[j].id - beg]);
        part[e[j].id - beg] = E::kNegInf;
      }
      mx = fmaxf(mx, x[j]);
    }
    __syncwarp();

    // ---- the rest's maximum and sum ----
    // t = log2 e^((x - m) / T) is one FMA, x c + b with b = -m c rounded; the rounding r is made
    // good on a round's sum.  m follows the maximum when that has come 2^16 past it.
    float m = -INFINITY, top = -INFINITY, s = 0.f, b = 0.f, rf = 1.f;
    const auto sum_vecs = [&](auto many, int i0) {   // vectors i0, i0 + 32, ...
      constexpr int U = decltype(many)::value;
      uint4 u[U];
#pragma unroll
      for (int k = 0; k < U; ++k) u[k] = pvec[i0 + k * 32];
      uint32_t w = E::max_words(E::max_words(u[0].x, u[0].y), E::max_words(u[0].z, u[0].w));
#pragma unroll
      for (int k = 1; k < U; ++k)
        w = E::max_words(w, E::max_words(E::max_words(u[k].x, u[k].y), E::max_words(u[k].z, u[k].w)));
      const float cm = E::to_float(E::word_max_bits(w));
      top = fmaxf(top, cm);
      if ((cm - m) * c > kSlack) {
        s *= ex2((m - cm) * c);
        m = cm;
        b = -m * c;
        const float r = fmaf(-m, c, -b);
        rf = ex2(r);
        if (!(fabsf(r) <= 1.f)) b = NAN;   // |m c| past 2^24, or no number
      }
      const float2 c2 = make_float2(c, c), b2 = make_float2(b, b);
      float2 s0 = make_float2(0.f, 0.f), s1 = s0;
      if (!isnan(b)) {
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
          for (int i = 0; i < E::VEC / 2; ++i) {
            const float2 t = __ffma2_rn(pair_of<E>(u[k], i), c2, b2);
            const float2 q = make_float2(ex2(t.x), ex2(t.y));
            if (i & 1)
              s1 = __fadd2_rn(s1, q);
            else
              s0 = __fadd2_rn(s0, q);
          }
        s0 = __fadd2_rn(s0, s1);
        s = fmaf(rf, s0.x + s0.y, s);
      } else {
#pragma unroll 1
        for (int k = 0; k < U; ++k) {
          const uint4 v = pvec[i0 + k * 32];
#pragma unroll
          for (int i = 0; i < E::VEC / 2; ++i) {
            const float2 x2 = pair_of<E>(v, i);
            s += ex2((x2.x - m) * c) + ex2((x2.y - m) * c);
          }
        }
      }
    };
    int i0 = lane;
    for (; i0 - lane + (kUnroll - 1) * 32 < vecs; i0 += kUnroll * 32)
      sum_vecs(std::integral_constant<int, kUnroll>(), i0);
    for (; i0 - lane < vecs; i0 += 32) sum_vecs(std::integral_constant<int, 1>(), i0);
    Part mine;
    mine.mr = warp_max(top);
    mine.m = warp_max(mx);
    {
      const float m0 = mine.m == -INFINITY ? 0.f : mine.m;
      float top = 0.f, p = 0.f, py = 0.f;
      int at_m = 0;
#pragma unroll
      for (int j = 0; j < kEntries; ++j)
        if (j * 32 < K && e[j].id >= 0) {
          const float y = x[j] - m0;
          if (x[j] == mine.m && mine.m != -INFINITY) {
            ++at_m;
            top += y;   // nothing, or NaN for +inf
          } else {
            top += ex2(y * c);
          }
          p += e[j].p;
          if (e[j].p != 0.f) py = fmaf(e[j].p, y * a.inv_t, py);
        }
      const float2 u = warp_sum2(make_float2(s * rescale(m, mine.mr), top)), v = warp_sum2(make_float2(p, py));
      mine.rest = u.x;
      at_m = __reduce_add_sync(0xffffffffu, at_m);
      mine.top = u.y + (float)max(at_m - 1, 0);
      mine.p = v.x;
      mine.py = v.y;
    }

    // ---- to every CTA of the cluster, and the row's from all of its warps ----
    const int turn = count & 1;
    const Part *parts = s_parts[turn];
    if (C > 1) {
      if (lane < C && !failed) {
        const uint32_t to = peer_addr(&s_parts[turn][rank * kWarps + warp], (uint32_t)lane);
        const uint32_t bar = peer_addr(&s_told[turn], (uint32_t)lane);
        st_async16(to, make_float4(mine.m, mine.mr, mine.rest, mine.top), bar);
        st_async16(to + 16, make_float4(mine.p, mine.py, 0.f, 0.f), bar);
      }
      __syncwarp();
      wait(&s_told[turn], (uint32_t)(count >> 1) & 1u);
      if (tid == 0 && !failed) mbar_arrive_expect_tx(&s_told[turn], told_bytes);   // for the pair after the next
    } else {
      if (lane == 0) s_parts[turn][warp] = mine;
      __syncthreads();
    }
    float all_ml = -INFINITY, all_mr = -INFINITY;
    for (int i = lane; i < C * kWarps; i += 32) {
      all_ml = fmaxf(all_ml, parts[i].m);
      all_mr = fmaxf(all_mr, parts[i].mr);
    }
    all_ml = warp_max(all_ml);
    all_mr = warp_max(all_mr);
    const float all_m = fmaxf(all_ml, all_mr);
    float all_rest = 0.f, all_top = 0.f, all_py = 0.f, at_ml = 0.f;
    for (int i = lane; i < C * kWarps; i += 32) {
      const Part q = parts[i];
      all_rest += q.rest * rescale(q.mr, all_mr);
      if (q.m == all_ml) {
        all_top += q.top;
        at_ml += 1.f;
      } else {
        all_top += (q.top + 1.f) * rescale(q.m, all_ml);
      }
      all_py += q.py + (q.p != 0.f && q.m != all_m && q.m != -INFINITY ? q.p * ((q.m - all_m) * a.inv_t) : 0.f);
    }
    {
      const float2 u = warp_sum2(make_float2(all_rest, all_top)), v = warp_sum2(make_float2(all_py, at_ml));
      all_rest = u.x;
      all_top = all_ml == -INFINITY ? u.y : u.y + (v.y - 1.f);
      all_py = v.x;
    }
    // The row's sum at its maximum: what is listed and the rest.  Where the maximum is a listed element, Z is
    // 1 + beside; with q = 1 / Z of that element, 1 - q is beside / Z and -ln q is log1p(beside), to
    // their own digits however near 1 q is.
    const float m0 = all_m == -INFINITY ? 0.f : all_m;
    const float down = rescale(all_mr, all_m);   // from the rest's maximum to the row's
    const float sum_rest = all_rest * down;
    const float sum_listed = all_ml == -INFINITY ? all_top : (1.f + all_top) * rescale(all_ml, all_m);
    const bool best_listed = all_ml == all_m && all_ml != -INFINITY;
    const float beside = all_top + sum_rest, Z = best_listed ? 1.f + beside : sum_listed + sum_rest;
    const bool empty = all_m == -INFINITY && Z == 0.f, no_rest = sum_rest / Z < kNoRest;
    if (rest < kLeastRest && no_rest) rest = 0.f;
    const float whole = rest > 0.f ? 1.f : listed;   // P
    if (rank == 0 && tid == 0 && in_bounds(pr, a.max_pairs, a.status, kSiteTopkPair)) {
      // sum p (ln Z - y) + p_rest (ln Z - ln of the rest's sum)
      const float lz = best_listed ? log1pf(beside) : logf(Z);
      float loss = (listed != 0.f ? listed * lz : 0.f) - all_py;
      if (rest > 0.f)
        loss += all_rest == 0.f ? INFINITY
                                : rest * (no_rest ? lz - logf(all_rest) + (all_m - all_mr) * a.inv_t
                                                  : log1pf(sum_listed / sum_rest));
      if (empty) loss = whole != 0.f ? INFINITY : 0.f;
      a.pair_loss[pr] = isnan(Z) || isnan(whole) ? NAN : loss;
    }

    // ---- the gradient ----
    if (a.grad && in_bounds(s_row, a.R_S, a.status, kSiteTopkStudentRow)) {
      const float per = empty ? 0.f : 1.f / Z, g = empty ? 0.f : a.grad_scale * a.inv_t / (float)N;
      // Outside: 2^((x - mr) c), over the rest's sum, times P q_rest - p_rest; where the rest has most of the row,
      // that is sum p - P q_listed, both of them small.
      const float pull = sum_rest > sum_listed ? listed - whole * (sum_listed * per) : whole * (sum_rest * per) - rest;
      const float coef = all_rest > 0.f ? g * pull / all_rest : 0.f * Z * whole;   // NaN stays one
      const float mr = all_mr == -INFINITY ? 0.f : all_mr, bias = -mr * c, r = fmaf(-mr, c, -bias);
      const bool exact = fabsf(r) <= 1.f;   // as above
      const float fcoef = coef * ex2(r);
      const float2 fcoef2 = make_float2(fcoef, fcoef), coef2 = make_float2(coef, coef);
      const float2 c2 = make_float2(c, c), b2 = make_float2(bias, bias), nmr2 = make_float2(-mr, -mr);
      T *out = static_cast<T *>(a.grad) + (int64_t)s_row * a.ld;
      const auto gradient = [&](const uint4 &u, float (&f)[E::VEC]) {
#pragma unroll
        for (int j = 0; j < E::VEC / 2; ++j) {
          const float2 t = __ffma2_rn(pair_of<E>(u, j), c2, b2);
          const float2 d = __fmul2_rn(make_float2(ex2(t.x), ex2(t.y)), fcoef2);
          f[2 * j] = d.x;
          f[2 * j + 1] = d.y;
        }
      };
      const auto careful = [&](const uint4 &u, float (&f)[E::VEC]) {
#pragma unroll
        for (int j = 0; j < E::VEC / 2; ++j) {
          const float2 t = __fmul2_rn(__fadd2_rn(pair_of<E>(u, j), nmr2), c2);
          const float2 d = __fmul2_rn(make_float2(ex2(t.x), ex2(t.y)), coef2);
          f[2 * j] = d.x;
          f[2 * j + 1] = d.y;
        }
      };
      uint4 *to = reinterpret_cast<uint4 *>(out + beg);
      float f[E::VEC];
      if (exact) {
#pragma unroll 4
        for (int i = lane; i < whole_vecs; i += 32) {
          gradient(pvec[i], f);
          __stcs(to + i, pack<E>(f));
        }
      } else {
        for (int i = lane; i < whole_vecs; i += 32) {
          careful(pvec[i], f);
          __stcs(to + i, pack<E>(f));
        }
      }
      if (lane == 0 && whole_vecs < vecs) {
        careful(pvec[whole_vecs], f);
        store_vec<E>(out, beg + whole_vecs * E::VEC, V, f);
      }
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kEntries; ++j)
        if (j * 32 < K && e[j].id >= 0) {
          // P q - p; where q is above one half, (P - p) - P (1 - q) instead, and where p is too (it is the
          // largest then), P - p is what the others and the rest add up to
          const float d = x[j] == all_m && beside < 1.f
                              ? (e[j].p > 0.5f * whole ? others + rest : whole - e[j].p) - whole * (beside * per)
                              : whole * (ex2((x[j] - m0) * c) * per) - e[j].p;
          out[e[j].id] = E::from_float(g * d);
        }
    }
    // ---- the next pair's ----
    s_row = next_row;
    if (next < N) {
      fence_proxy_async_smem();   // what the lanes wrote here comes before the copy
      __syncwarp();
      copy(s_row);
      load_list(next);
    }
    if (is_other(word)) write_zeros();
    if (other < a.R_S) other += clusters;
  }
  for (; other < a.R_S; other += clusters)
    if (is_other(a.paired[other >> 5])) write_zeros();

  if (C > 1) cluster_sync_all();   // no CTA leaves while one may still tell it anything
  // ---- the loss: the last cluster sums the per-pair losses in pair order ----
  if (rank != 0) return;
  __syncthreads();
  if (tid == 0) {
    s_last = 0;
    if (arrive_is_last(&a.hdr->clusters_done, clusters)) s_last = 1;
  }
  __syncthreads();
  if (!s_last) return;
  __shared__ double dsum[kWarps];
  const int per = (N + kThreads - 1) / kThreads;
  double acc = 0.0;
  for (int i = 0; i < per; ++i)
    if (tid * per + i < N) acc += (double)__ldcg(a.pair_loss + tid * per + i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
  if (lane == 0) dsum[warp] = acc;
  __syncthreads();
  if (tid == 0) {
    double t = 0.0;
    for (int i = 0; i < kWarps; ++i) t += dsum[i];
    a.loss[0] = N > 0 ? (float)(t / (double)N) : 0.f;
  }
}

// elements of a row per CTA: whole vectors of every type
int slice_of(int V, int C) { return ceil_div(ceil_div(V, C), 8) * 8; }

// its shared memory
size_t part_bytes(int V, int C, int esize) {
  return (size_t)room_vecs(slice_of(V, C) / (16 / esize)) * kWarps * 16;
}

// CTAs per row: as many as it takes for three parts to fit an SM, or two where no cluster is large enough
// for that; and for few rows more, while that leaves an SM to each and a part is still worth a CTA
// (2048 elements).  Measured for 57 rows of 32000 bf16: 11.1 us by two CTAs a row, 14.2 by four
// and eight; for 1500 of 151936 bf16: 160 by five, 166 by six, 201 by eight, three parts fitting
// in each case; for 700 of 151936 fp32: 155 by six, two parts fitting as by seven, 172, and eight, 164.
int cluster_for(int R, int V, int esize, int num_sms) {
  const auto fitting = [&](int bytes) {
    int C = 1;
    while (C < kMaxCluster && part_bytes(V, C, esize) > (size_t)bytes) ++C;
    return C;
  };
  int C = fitting(kPartBytes);
  if (part_bytes(V, C, esize) > (size_t)kPartBytes) C = fitting(kHalfBytes);
  while (C < kMaxCluster && (int64_t)R * 2 * C <= num_sms && V / (2 * C) >= 2048) C = std::min(2 * C, kMaxCluster);
  return C;
}

// Clusters of C CTAs of `bytes` shared memory that the device holds at once, looked up once per
// device, type and configuration.  Not 3 x SMs / C: a GPU cluster's SMs need not be a
// multiple of C, and a cluster that has to wait for another to end doubles the time.
template <class E>
int resident_clusters(int C, size_t bytes, int num_sms) {
  struct Known {
    int dev, C, n;
    size_t bytes;
  };
  static Known known[64];
  static int n_known = 0;
  static std::mutex mu;
  int dev = 0;
  cudaGetDevice(&dev);
  std::lock_guard<std::mutex> lock(mu);
  for (int i = 0; i < n_known; ++i)
    if (known[i].dev == dev && known[i].C == C && known[i].bytes == bytes) return known[i].n;
  // before the first launch of any configuration here; the largest size, so that none finds a smaller limit
  if (!allow_smem(topk_ce_kernel<E>, std::max(part_bytes(kMaxLogitVocab, kMaxCluster, (int)sizeof(typename E::T)),
                                              (size_t)kPartBytes)))
    return 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(C * std::max(1, num_sms / C)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = bytes;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, topk_ce_kernel<E>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    n = 0;
  }
  if (n > 0 && n_known < 64) known[n_known++] = Known{dev, C, n, bytes};
  return n;
}

template <class E>
umim_status launch_topk_ce(TopkArgs a, cudaStream_t stream, int num_sms) {
  constexpr int esize = sizeof(typename E::T);
  const int C = cluster_for(std::max(a.R_S, 1), a.V, esize, num_sms);
  const size_t bytes = part_bytes(a.V, C, esize);
  a.slice = slice_of(a.V, C);
  const int resident = resident_clusters<E>(C, bytes, num_sms);
  if (resident < 1) return UMIM_ERR_CUDA;
  const int clusters = std::min(std::max(a.R_S, 1), resident);
  trace_mark(stream, "distill.topk_ce");
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)clusters * (unsigned)C);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  // Where a cluster has few pairs it starts while the plan is being made: 18.7 us instead of 21.7 for 108
  // pairs of 128256 bf16, 31.5 instead of 34.5 for 220, 27.5 instead of 30.0 for 456 of 50257.  Where it
  // has many it must not: some clusters find their SMs taken by the plan, come late and end last, 56.2
  // instead of 54.5 for 448 pairs of 128256, 301 instead of 245 for 2870 of as many rows.
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = (int64_t)a.R_S <= 2 * (int64_t)resident ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, topk_ce_kernel<E>, a);
  trace_mark(stream, nullptr);
  return e == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

}  // namespace

size_t distill_topk_ce_workspace_bytes(int R_S, int max_pairs) {
  const size_t P = (size_t)std::max(max_pairs, 1);
  return sizeof(TopkHeader) + a256(sizeof(uint32_t) * ((size_t)R_S / 32 + 1)) + a256(sizeof(float) * P) +
         a256(sizeof(Head) * P) + a256(sizeof(Entry) * kMaxTop * P);
}

umim_status distill_topk_ce(const int32_t *top_ids, const float *top_logprobs, int R_T, int K, const void *student,
                            int dtype, int R_S, int V, int64_t ld, const int32_t *teacher_rows,
                            const int32_t *student_rows, int max_pairs, const int32_t *n_dev, float temperature,
                            int tail, float grad_scale, float *loss, float *pair_loss, void *grad, void *ws,
                            int32_t *dev_status, cudaStream_t stream, int num_sms) {
  char *p = static_cast<char *>(ws);
  TopkHeader *hdr = reinterpret_cast<TopkHeader *>(p);
  p += sizeof(TopkHeader);
  const auto take = [&p](size_t bytes) {
    char *q = p;
    p += a256(bytes);
    return q;
  };
  const size_t P = (size_t)std::max(max_pairs, 1);
  TopkArgs a;
  a.top_ids = top_ids;
  a.top_logprobs = top_logprobs;
  a.R_T = R_T;
  a.K = K;
  a.student = student;
  a.R_S = R_S;
  a.V = V;
  a.ld = ld;
  a.teacher_rows = teacher_rows;
  a.student_rows = student_rows;
  a.max_pairs = max_pairs;
  a.n_dev = n_dev;
  a.inv_t = 1.f / temperature;
  a.c = kLog2e / temperature;
  a.grad_scale = grad_scale;
  a.tail = tail;
  a.loss = loss;
  a.grad = grad;
  a.paired = reinterpret_cast<uint32_t *>(take(sizeof(uint32_t) * ((size_t)R_S / 32 + 1)));
  float *ws_pair_loss = reinterpret_cast<float *>(take(sizeof(float) * P));
  a.pair_loss = pair_loss ? pair_loss : ws_pair_loss;
  a.heads = reinterpret_cast<Head *>(take(sizeof(Head) * P));
  a.lists = reinterpret_cast<Entry *>(take(sizeof(Entry) * kMaxTop * P));
  a.hdr = hdr;
  a.status = dev_status ? dev_status : &hdr->status;
  trace_mark(stream, "distill.topk_plan");
  const unsigned plan_ctas = 1 + (unsigned)ceil_div(max_pairs, kPlanPairs);
  if (launch_pdl(topk_plan_kernel, dim3(plan_ctas), dim3(kPlanThreads), 0, stream, a) != cudaSuccess)
    return UMIM_ERR_CUDA;
  return dtype == UMIM_DTYPE_BF16   ? launch_topk_ce<ElemBf16>(a, stream, num_sms)
         : dtype == UMIM_DTYPE_FP16 ? launch_topk_ce<ElemFp16>(a, stream, num_sms)
                                    : launch_topk_ce<ElemFp32>(a, stream, num_sms);
}

}  // namespace umim
