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

constexpr int kThreads = 256;
constexpr int kPlanThreads = 1024;
// The listed log probabilities are fp32: their exponentials are off by up to
// about 16 2^-24 each, relatively, so 1 - sum p below 2^-20 is rounding, and
// its logarithm's partner q_rest may be 0 where the list holds all there is.
constexpr float kLeastRest = 9.5367431640625e-7f;

struct TopkHeader {
  int32_t status;     // status word when the caller passes none
  int32_t error;      // the pairs are invalid: nothing is written
  int32_t n_pairs;    // N
  int32_t ctas_done;  // CTAs of the main kernel that finished
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
  float inv_t, grad_scale;
  int32_t tail;
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
    a.hdr->ctas_done = 0;
    if (bad) set_error(a.status, UMIM_ERR_INVALID_ARG);
  }
}

template <class F>
__device__ float block_reduce(float v, F op) {
  __shared__ float part[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  float r = part[0];
  for (int i = 1; i < kThreads / 32; ++i) r = op(r, part[i]);
  return r;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }

// One CTA per student row: the list, the row's maximum and sums, the gradient.
template <class E>
__global__ void __launch_bounds__(kThreads) topk_ce_kernel(TopkArgs a) {
  griddep_wait();
  __shared__ uint32_t listed[kMaxLogitVocab / 32];   // a bit per vocabulary entry: in the teacher's list
  __shared__ int s_id[kMaxTop];
  __shared__ int s_last;
  const int r = blockIdx.x, tid = threadIdx.x, V = a.V, K = a.K;
  if (a.hdr->error) return;
  const int N = a.hdr->n_pairs, pr = r < a.R_S ? a.row_pair[r] : -1;   // no student rows: one CTA, for the loss
  const typename E::T *row = static_cast<const typename E::T *>(a.student) + (int64_t)r * a.ld;
  typename E::T *out = a.grad && r < a.R_S ? static_cast<typename E::T *>(a.grad) + (int64_t)r * a.ld : nullptr;
  if (pr < 0) {
    float z[E::VEC] = {};
    if (out)
      for (int e = tid * E::VEC; e < V; e += kThreads * E::VEC) store_vec<E>(out, e, V, z);
  } else {
    // thread i < K holds entry i
    const int tr = in_bounds(a.teacher_rows[pr], a.R_T, a.status, kSiteTopkTeacherRow) ? a.teacher_rows[pr] : 0;
    for (int i = tid; i < (V + 31) / 32; i += kThreads) listed[i] = 0;
    int id = -1;
    float lam = -INFINITY, x = 0.f;
    if (tid < K) {
      id = a.top_ids[(int64_t)tr * K + tid];
      if (id < -1 || id >= V) {
        set_error(a.status, UMIM_ERR_INVALID_ARG);
        id = -1;
      }
      s_id[tid] = id;
    }
    __syncthreads();
    if (id >= 0) {
      for (int j = 0; j < tid; ++j)
        if (s_id[j] == id) id = -2;   // a repeated id: the first entry counts
      if (id < 0) set_error(a.status, UMIM_ERR_INVALID_ARG);
    }
    if (id >= 0) {
      lam = a.top_logprobs[(int64_t)tr * K + tid];
      x = E::to_float(row[id]);
      atomicOr(&listed[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    float p, rest = 0.f, whole;
    if (a.tail) {
      p = id >= 0 ? expf(lam) : 0.f;
      whole = block_reduce(p, add);
      rest = 1.f - whole;
      if (rest < kLeastRest) rest = 0.f;
      whole += rest;
    } else {
      const float top = block_reduce(lam, fmaxf);
      p = id >= 0 && !(lam == -INFINITY) ? expf(lam - top) : 0.f;
      const float sum = block_reduce(p, add);
      p = sum == 0.f ? 0.f : p / sum;   // a row without entries adds nothing
      whole = sum == 0.f ? 0.f : 1.f;
    }
    float m = -INFINITY;
    for (int v = tid; v < V; v += kThreads) m = fmaxf(m, E::to_float(row[v]));
    m = block_reduce(m, fmaxf);
    const float m0 = m == -INFINITY ? 0.f : m;
    float zr = 0.f;
    for (int v = tid; v < V; v += kThreads)
      if (!((listed[v >> 5] >> (v & 31)) & 1)) zr += expf((E::to_float(row[v]) - m0) * a.inv_t);
    zr = block_reduce(zr, add);
    const float y = (x - m0) * a.inv_t;
    const float Z = zr + block_reduce(id >= 0 ? expf(y) : 0.f, add);
    const bool empty = m == -INFINITY && Z == 0.f;
    const float lz = logf(Z);
    float part = p != 0.f ? -p * (empty ? -INFINITY : y - lz) : 0.f;
    if (tid == 0 && rest > 0.f) part -= rest * (empty ? -INFINITY : logf(zr) - lz);
    part = block_reduce(part, add);
    if (tid == 0 && in_bounds(pr, a.max_pairs, a.status, kSiteTopkPair)) a.pair_loss[pr] = part;
    if (out) {
      const float c = a.grad_scale * a.inv_t / (float)N;
      const float out_c = empty ? 0.f : c * (rest > 0.f && zr > 0.f ? whole / Z - rest / zr : whole / Z);
      for (int e = tid * E::VEC; e < V; e += kThreads * E::VEC) {
        float f[E::VEC];
        load_vec<E>(row, e, V, 0.f, f);
#pragma unroll
        for (int j = 0; j < E::VEC; ++j) f[j] = empty ? 0.f : out_c * expf((f[j] - m0) * a.inv_t);
        store_vec<E>(out, e, V, f);
      }
      __syncthreads();
      if (id >= 0 && in_bounds(id, V, a.status, kSiteTopkEntry))
        out[id] = E::from_float(empty ? 0.f : c * (whole * expf(y) / Z - p));
    }
  }
  // ---- the loss: the last CTA sums the per-pair losses in pair order ----
  __syncthreads();
  if (tid == 0) s_last = arrive_is_last(&a.hdr->ctas_done, (int)gridDim.x);
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
  trace_mark(stream, "distill.topk_ce");
  const cudaError_t e = launch_pdl(k, dim3((unsigned)std::max(R_S, 1)), dim3(kThreads), 0, stream, a);
  trace_mark(stream, nullptr);
  return e == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

}  // namespace umim
