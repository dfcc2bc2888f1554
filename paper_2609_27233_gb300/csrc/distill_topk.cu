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
#include <algorithm>
#include <cmath>

#include "logits.cuh"

namespace umim {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 4;
constexpr int kMaxCluster = 8;    // CTAs per row, at most
constexpr int kPartBytes = 65536; // three parts of this size fit an SM's shared memory
constexpr int kPlanThreads = 1024;
// The listed log probabilities are fp32: their exponentials are off by up to
// about 16 2^-24 each, relatively, so 1 - sum p below 2^-20 is rounding, and
// its logarithm's partner q_rest may be 0 where the list holds all there is.
constexpr float kLeastRest = 9.5367431640625e-7f;

struct TopkHeader {
  int32_t status;     // status word when the caller passes none
  int32_t error;      // the pairs are invalid: nothing is written
  int32_t n_pairs;    // N
  int32_t rows_done;  // rows that the main kernel has finished
  int32_t pad[60];
};
static_assert(sizeof(TopkHeader) == 256, "header size");

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
  int32_t *row_pair;           // [R_S] pair of each student row, -1 if none
  TopkHeader *hdr;
  int32_t *status;
};

inline size_t a256(size_t x) { return (x + 255) & ~size_t(255); }

// One CTA: the pair of every student row; the pairs are checked before anything is written.
__global__ void __launch_bounds__(kPlanThreads) topk_plan_kernel(TopkArgs a) {
  griddep_wait();
  griddep_launch();
  const int tid = threadIdx.x;
  __shared__ int bad;
  const int N = a.n_dev ? *a.n_dev : a.max_pairs;
  if (tid == 0) bad = N < 0 || N > a.max_pairs;
  for (int r = tid; r < a.R_S; r += kPlanThreads) a.row_pair[r] = -1;
  __syncthreads();
  if (!bad)
    for (int p = tid; p < N; p += kPlanThreads) {
      const int t = a.teacher_rows[p], s = a.student_rows[p];
      if (t < 0 || t >= a.R_T || s < 0 || s >= a.R_S || atomicCAS(&a.row_pair[s], -1, p) != -1) bad = 1;
    }
  __syncthreads();
  if (tid == 0) {
    a.hdr->error = bad;
    a.hdr->n_pairs = N;
    a.hdr->rows_done = 0;
    if (bad) set_error(a.status, UMIM_ERR_INVALID_ARG);
  }
}

// sum / maximum over the CTA's first K <= kMaxTop threads' values (the others pass the neutral one)
__device__ __forceinline__ float cta_sum(float v, float *part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  float r = part[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) r += part[i];
  return r;
}
__device__ __forceinline__ float cta_max(float v, float *part) {
  v = warp_max(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  float r = part[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) r = fmaxf(r, part[i]);
  return r;
}

// What a CTA's part of the row adds: outside the list the maximum mr and the sum of
// 2^((x - mr) c); the maximum m of the whole part, and over the listed
// elements the sums of 2^((x - m) c), p and p (x - m) / T.  The rest keeps a maximum
// of its own: where the listed ones are far above it, its sum would be nothing beside m.
struct Part {
  float m, mr, rest, top, p, py;
};

// One cluster of C CTAs per student row, each on one of C contiguous parts, which
// it holds in shared memory between the two passes over it: every logit is read
// once, by one asynchronous copy per part, and every gradient element written
// once.  What bounds it is that traffic; with three CTAs to an SM one loads
// while another sums or writes.
//
// The listed elements are taken out of the part before the first pass (-inf in
// their place), so that it sums the rest alone, and their gradients are written
// after the second pass, over the zeros that it left there.
template <class E>
__global__ void __launch_bounds__(kThreads, 3) topk_ce_kernel(TopkArgs a) {
  extern __shared__ __align__(128) uint8_t dyn[];   // the part
  __shared__ __align__(8) uint64_t landed;
  __shared__ int s_id[kMaxTop];
  __shared__ float s_part[kWarps];
  __shared__ float2 s_stat[kWarps];
  __shared__ Part s_parts[kMaxCluster];
  __shared__ int s_last;
  griddep_wait();
  griddep_launch();
  const int C = (int)cluster_size(), rank = C > 1 ? (int)cluster_ctarank() : 0;
  const int r = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31, V = a.V, K = a.K;
  if (a.hdr->error) return;
  const int N = a.hdr->n_pairs, pr = r < a.R_S ? a.row_pair[r] : -1;   // no student rows: one CTA, for the loss
  using T = typename E::T;
  const T *row = static_cast<const T *>(a.student) + (int64_t)r * a.ld;
  T *out = a.grad && r < a.R_S ? static_cast<T *>(a.grad) + (int64_t)r * a.ld : nullptr;
  const int beg = min(rank * a.slice, V), end = min(beg + a.slice, V), n = end - beg;
  const int vecs = ceil_div(n, E::VEC), whole_vecs = n / E::VEC;
  T *part = reinterpret_cast<T *>(dyn);
  const uint4 *pvec = reinterpret_cast<const uint4 *>(dyn);
  if (pr < 0) {
    const float z[E::VEC] = {};
    if (out)
      for (int i = tid; i < vecs; i += kThreads) store_vec<E>(out, beg + i * E::VEC, V, z);
  } else {
    // ---- the part, and meanwhile the list: thread i < K has entry i ----
    if (tid == 0) {
      mbar_init(&landed, 1);
      fence_mbar_init();
      mbar_arrive_expect_tx(&landed, (uint32_t)whole_vecs * 16u);
      if (whole_vecs > 0) bulk_load(dyn, row + beg, (uint32_t)whole_vecs * 16u, &landed);
    }
    if (tid < vecs - whole_vecs) {   // the vector that the row's end cuts
      const uint4 u = load_raw<E>(row, beg + whole_vecs * E::VEC, V);
      *reinterpret_cast<uint4 *>(part + whole_vecs * E::VEC) = u;
    }
    const int tr = in_bounds(a.teacher_rows[pr], a.R_T, a.status, kSiteTopkTeacherRow) ? a.teacher_rows[pr] : 0;
    int id = -1;
    float lam = -INFINITY;
    if (tid < K) {
      id = a.top_ids[(int64_t)tr * K + tid];
      lam = a.top_logprobs[(int64_t)tr * K + tid];
      if (id < -1 || id >= V) {
        if (rank == 0) set_error(a.status, UMIM_ERR_INVALID_ARG);
        id = -1;
      }
      s_id[tid] = id;
    }
    __syncthreads();
    if (id >= 0) {
      for (int j = 0; j < tid; ++j)
        if (s_id[j] == id) id = -2;   // a repeated id: the first entry counts
      if (id == -2 && rank == 0) set_error(a.status, UMIM_ERR_INVALID_ARG);
    }
    float p, rest = 0.f, whole;   // p_i, p_rest, P
    if (a.tail) {
      p = id >= 0 ? expf(lam) : 0.f;
      whole = cta_sum(p, s_part);
      rest = 1.f - whole;
      if (rest < kLeastRest) rest = 0.f;
      whole += rest;
    } else {
      const float top = cta_max(id >= 0 ? lam : -INFINITY, s_part);
      p = id >= 0 && !(lam == -INFINITY) ? expf(lam - top) : 0.f;
      const float sum = cta_sum(p, s_part);
      p = sum == 0.f ? 0.f : p / sum;   // a row without entries adds nothing
      whole = sum == 0.f ? 0.f : 1.f;
    }
    if (!mbar_wait_sleep(&landed, 0)) set_error(a.status, UMIM_ERR_TIMEOUT);
    const bool mine = id >= beg && id < end;
    float x = -INFINITY;
    if (mine && in_bounds(id - beg, n, a.status, kSiteTopkEntry)) {
      x = E::to_float(part[id - beg]);
      part[id - beg] = E::kNegInf;
    }
    __syncthreads();

    // ---- the rest's maximum and sum ----
    const float c = a.c;
    float m = -INFINITY, s = 0.f;
    for (int i0 = tid; i0 < vecs; i0 += kUnroll * kThreads) {
      uint4 u[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        u[k] = i0 + k * kThreads < vecs ? pvec[i0 + k * kThreads]
                                        : make_uint4(E::kNegInf2, E::kNegInf2, E::kNegInf2, E::kNegInf2);
      uint32_t top = E::kNegInf2;
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        top = E::max_words(top, E::max_words(E::max_words(u[k].x, u[k].y), E::max_words(u[k].z, u[k].w)));
      const float cm = E::to_float(E::word_max_bits(top));
      if (cm > m) {
        s *= ex2((m - cm) * c);
        m = cm;
      }
      const float nm = m == -INFINITY ? 0.f : -m;
      const float2 nm2 = make_float2(nm, nm), c2 = make_float2(c, c);
      float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
#pragma unroll
        for (int i = 0; i < E::VEC / 2; ++i) {
          const float2 t = __fmul2_rn(__fadd2_rn(pair_of<E>(u[k], i), nm2), c2);
          const float2 e = make_float2(ex2(t.x), ex2(t.y));
          if (i & 1)
            s1 = __fadd2_rn(s1, e);
          else
            s0 = __fadd2_rn(s0, e);
        }
      s0 = __fadd2_rn(s0, s1);
      s += s0.x + s0.y;
    }
    const auto rescale = [c](float from, float to) { return from == to ? 1.f : ex2((from - to) * c); };
    Part mypart;
    {
      const float wm = warp_max(m);
      const float sum = warp_sum2(make_float2(s * rescale(m, wm), 0.f)).x;
      if (lane == 0) s_stat[tid >> 5] = make_float2(wm, sum);
      mypart.m = cta_max(x, s_part);   // the listed elements'
      const float2 w = lane < kWarps ? s_stat[lane] : make_float2(-INFINITY, 0.f);
      mypart.mr = warp_max(w.x);
      mypart.rest = warp_sum2(make_float2(w.y * rescale(w.x, mypart.mr), 0.f)).x;
      mypart.m = fmaxf(mypart.m, mypart.mr);
    }
    {
      const float m0 = mypart.m == -INFINITY ? 0.f : mypart.m;
      const float y = x - m0;
      mypart.top = cta_sum(mine ? ex2(y * c) : 0.f, s_part);
      mypart.p = cta_sum(mine ? p : 0.f, s_part);
      mypart.py = cta_sum(mine && p != 0.f ? p * (y * a.inv_t) : 0.f, s_part);
    }
    // ---- the row's, in every CTA ----
    Part all = mypart;
    if (C > 1) {
      cluster_sync_all();   // every CTA of the cluster runs
      if (tid < C) {
        const uint32_t to = peer_addr(&s_parts[rank], (uint32_t)tid);
        const float v[6] = {mypart.m, mypart.mr, mypart.rest, mypart.top, mypart.p, mypart.py};
#pragma unroll
        for (int i = 0; i < 6; ++i)
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4 * i), "f"(v[i]) : "memory");
      }
      cluster_sync_all();
      for (int k = 0; k < C; ++k) {
        all.m = fmaxf(all.m, s_parts[k].m);
        all.mr = fmaxf(all.mr, s_parts[k].mr);
      }
      all.rest = all.top = all.py = 0.f;
      for (int k = 0; k < C; ++k) {
        const Part q = s_parts[k];
        all.rest += q.rest * rescale(q.mr, all.mr);
        all.top += q.top * rescale(q.m, all.m);
        all.py += q.py + (q.p != 0.f && q.m != all.m && q.m != -INFINITY ? q.p * ((q.m - all.m) * a.inv_t) : 0.f);
      }
    }
    const float m0 = all.m == -INFINITY ? 0.f : all.m;
    const float down = rescale(all.mr, all.m);   // from the rest's maximum to the row's
    const float Z = all.rest * down + all.top;
    const bool empty = all.m == -INFINITY && Z == 0.f;
    if (rank == 0 && tid == 0 && in_bounds(pr, a.max_pairs, a.status, kSiteTopkPair)) {
      // sum p (ln Z - y) + p_rest (ln Z - ln of the rest's sum)
      const float lz = logf(Z), listed = whole - rest;
      float loss = (listed != 0.f ? listed * lz : 0.f) - all.py;
      if (rest > 0.f)
        loss += all.rest == 0.f ? INFINITY : rest * (lz - logf(all.rest) + (all.m - all.mr) * a.inv_t);
      if (empty) loss = whole != 0.f ? INFINITY : 0.f;
      a.pair_loss[pr] = isnan(Z) ? NAN : loss;
    }
    // ---- the gradient ----
    if (out) {
      const float g = a.grad_scale * a.inv_t / (float)N;
      // outside: 2^((x - mr) c) times this
      const float q = whole * (down / Z);
      const float coef = empty ? 0.f : g * (rest > 0.f && all.rest > 0.f ? q - rest / all.rest : q);
      const float nmr = all.mr == -INFINITY ? 0.f : -all.mr;
      const float2 coef2 = make_float2(coef, coef), nm2 = make_float2(nmr, nmr), c2 = make_float2(c, c);
      T *o = out + beg;
#pragma unroll 4
      for (int i = tid; i < vecs; i += kThreads) {
        const uint4 u = pvec[i];
        float f[E::VEC];
#pragma unroll
        for (int j = 0; j < E::VEC / 2; ++j) {
          const float2 t = __fmul2_rn(__fadd2_rn(pair_of<E>(u, j), nm2), c2);
          const float2 d = __fmul2_rn(make_float2(ex2(t.x), ex2(t.y)), coef2);
          f[2 * j] = d.x;
          f[2 * j + 1] = d.y;
        }
        if (i < whole_vecs)
          __stcs(reinterpret_cast<uint4 *>(o + i * E::VEC), pack<E>(f));
        else
          store_vec<E>(o, i * E::VEC, n, f);
      }
      __syncthreads();
      if (mine) out[id] = E::from_float(empty ? 0.f : g * (whole * (ex2((x - m0) * c) / Z) - p));
    }
  }
  if (rank != 0) return;
  // ---- the loss: the last CTA sums the per-pair losses in pair order ----
  __syncthreads();
  if (tid == 0) s_last = arrive_is_last(&a.hdr->rows_done, (int)gridDim.x / C);
  __syncthreads();
  if (!s_last) return;
  __shared__ double dsum[kThreads / 32];
  const int per = (N + kThreads - 1) / kThreads;
  double acc = 0.0;
  for (int i = 0; i < per; ++i)
    if (tid * per + i < N) acc += (double)__ldcg(a.pair_loss + tid * per + i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
  if ((tid & 31) == 0) dsum[tid >> 5] = acc;
  __syncthreads();
  if (tid == 0) {
    double t = 0.0;
    for (int i = 0; i < kThreads / 32; ++i) t += dsum[i];
    a.loss[0] = N > 0 ? (float)(t / (double)N) : 0.f;
  }
}

// elements of a row per CTA: whole vectors of every type
int slice_of(int V, int C) { return ceil_div(ceil_div(V, C), 8) * 8; }

// CTAs per row: as many as it takes for three parts to fit an SM, and for few rows more, so
// that the SMs hold three CTAs each, where a part is still worth a CTA (2048 elements).
int cluster_for(int R, int V, int esize, int num_sms) {
  int C = 1;
  while (C < kMaxCluster && (slice_of(V, C) * esize > kPartBytes ||
                             ((int64_t)R * C < 3 * num_sms && V / (2 * C) >= 2048)))
    C *= 2;
  return C;
}

}  // namespace

size_t distill_topk_ce_workspace_bytes(int R_S, int max_pairs) {
  return sizeof(TopkHeader) + a256(sizeof(int32_t) * (size_t)std::max(R_S, 1)) +
         a256(sizeof(float) * (size_t)std::max(max_pairs, 1));
}

umim_status distill_topk_ce(const int32_t *top_ids, const float *top_logprobs, int R_T, int K, const void *student,
                            int dtype, int R_S, int V, int64_t ld, const int32_t *teacher_rows,
                            const int32_t *student_rows, int max_pairs, const int32_t *n_dev, float temperature,
                            int tail, float grad_scale, float *loss, float *pair_loss, void *grad, void *ws,
                            int32_t *dev_status, cudaStream_t stream, int num_sms) {
  char *p = static_cast<char *>(ws);
  TopkHeader *hdr = reinterpret_cast<TopkHeader *>(p);
  p += sizeof(TopkHeader);
  int32_t *row_pair = reinterpret_cast<int32_t *>(p);
  p += a256(sizeof(int32_t) * (size_t)std::max(R_S, 1));
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
  a.pair_loss = pair_loss ? pair_loss : reinterpret_cast<float *>(p);
  a.grad = grad;
  a.row_pair = row_pair;
  a.hdr = hdr;
  a.status = dev_status ? dev_status : &hdr->status;
  trace_mark(stream, "distill.topk_plan");
  if (launch_pdl(topk_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a) != cudaSuccess) return UMIM_ERR_CUDA;
  auto *k = dtype == UMIM_DTYPE_BF16   ? topk_ce_kernel<ElemBf16>
            : dtype == UMIM_DTYPE_FP16 ? topk_ce_kernel<ElemFp16>
                                       : topk_ce_kernel<ElemFp32>;
  const int esize = (int)dtype_bytes(dtype);
  const int C = cluster_for(std::max(R_S, 1), V, esize, num_sms);
  a.slice = slice_of(V, C);
  if (!allow_smem(k, (size_t)slice_of(kMaxLogitVocab, kMaxCluster) * 4)) return UMIM_ERR_CUDA;
  trace_mark(stream, "distill.topk_ce");
  const cudaError_t e = launch_pdl_cluster(k, dim3((unsigned)std::max(R_S, 1) * (unsigned)C), dim3(kThreads),
                                           (unsigned)C, (size_t)a.slice * esize, stream, a);
  trace_mark(stream, nullptr);
  return e == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

}  // namespace umim
