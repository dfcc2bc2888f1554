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

constexpr int kThreads = 256;

struct LogprobArgs {
  const void *logits;
  int32_t R, V;
  int64_t ld;
  const int32_t *n_dev;
  const int32_t *tokens;     // nullptr: no token, every row counts
  float inv_t;
  int32_t n_top;
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
  float inv_t;
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

// One CTA per row: the maximum, the sums, then one search for each alternative.
template <class E>
__global__ void __launch_bounds__(kThreads) token_logprobs_kernel(LogprobArgs a) {
  griddep_wait();
  const int r = blockIdx.x, tid = threadIdx.x, V = a.V;
  if (r >= rows_used(a.n_dev, a.R)) return;
  const int token = a.tokens ? row_token(a.tokens, r, V, a.status, tid == 0) : 0;
  if (token < 0) {
    if (tid == 0) {
      if (a.logprobs) a.logprobs[r] = 0.f;
      if (a.entropy) a.entropy[r] = 0.f;
      if (a.stats) a.stats[r] = make_float2(0.f, 0.f);
    }
    for (int i = tid; i < a.n_top; i += kThreads) {
      a.top_ids[(int64_t)r * a.n_top + i] = -1;
      a.top_logprobs[(int64_t)r * a.n_top + i] = -INFINITY;
    }
    return;
  }
  const typename E::T *row = static_cast<const typename E::T *>(a.logits) + (int64_t)r * a.ld;
  float m = -INFINITY;
  for (int v = tid; v < V; v += kThreads) m = fmaxf(m, E::to_float(row[v]));
  m = block_reduce(m, fmaxf);
  const float m0 = m == -INFINITY ? 0.f : m;
  float s = 0.f, w = 0.f;
  for (int v = tid; v < V; v += kThreads) {
    const float y = (E::to_float(row[v]) - m0) * a.inv_t, e = expf(y);
    s += e;
    if (!(e == 0.f)) w += e * y;
  }
  s = block_reduce(s, add);
  w = block_reduce(w, add);
  const bool bad = !(s < INFINITY), empty = m == -INFINITY && !bad;
  const float l = bad ? NAN : empty ? 0.f : logf(s);
  if (tid == 0) {
    const float y = (E::to_float(row[token]) - m0) * a.inv_t;
    if (a.logprobs) a.logprobs[r] = bad ? NAN : y - l;
    if (a.entropy) a.entropy[r] = bad ? NAN : empty ? 0.f : l - w / s;
    if (a.stats) a.stats[r] = bad ? make_float2(NAN, NAN) : make_float2(m, l);
  }
  // the alternatives: each the largest (value, lowest id) after the one before
  float last = INFINITY;
  int last_id = -1;
  for (int i = 0; i < a.n_top; ++i) {
    float best = -INFINITY;
    int id = INT32_MAX;
    for (int v = tid; v < V && !bad; v += kThreads) {
      const float x = E::to_float(row[v]);
      const bool after = x < last || (x == last && v > last_id);
      if (after && x > best) {
        best = x;
        id = v;
      }
    }
    const float top = block_reduce(best, fmaxf);
    // ids are below 2^24: exact as floats
    const float low = block_reduce(best == top && id != INT32_MAX ? (float)id : 1e9f, fminf);
    last = top;
    last_id = (int)low;
    if (tid == 0) {
      const bool none = top == -INFINITY;
      a.top_ids[(int64_t)r * a.n_top + i] = none ? -1 : last_id;
      a.top_logprobs[(int64_t)r * a.n_top + i] = bad ? NAN : none ? -INFINITY : (top - m0) * a.inv_t - l;
    }
  }
}

// One CTA per row, a vector per thread and step.
template <class E>
__global__ void __launch_bounds__(kThreads) token_logprobs_grad_kernel(GradArgs a) {
  griddep_wait();
  const int r = blockIdx.x, V = a.V;
  if (r >= rows_used(a.n_dev, a.R)) return;
  const typename E::T *row = static_cast<const typename E::T *>(a.logits) + (int64_t)r * a.ld;
  typename E::T *out = static_cast<typename E::T *>(a.grad) + (int64_t)r * a.ld;
  const int token = a.tokens ? row_token(a.tokens, r, V, a.status, threadIdx.x == 0) : 0;
  const float2 st = a.stats[r];
  const bool zero = token < 0 || st.x == -INFINITY;
  const float g = a.g ? a.g[r] * a.inv_t : 0.f, h = a.h ? a.h[r] * a.inv_t : 0.f, H = a.h ? a.entropy[r] : 0.f;
  for (int e = threadIdx.x * E::VEC; e < V; e += kThreads * E::VEC) {
    float x[E::VEC], d[E::VEC];
    if (zero) {
#pragma unroll
      for (int j = 0; j < E::VEC; ++j) d[j] = 0.f;
    } else {
      load_vec<E>(row, e, V, 0.f, x);
#pragma unroll
      for (int j = 0; j < E::VEC; ++j) {
        const float z = (x[j] - st.x) * a.inv_t - st.y, p = expf(z);
        d[j] = -p * g;
        if (a.g && e + j == token) d[j] = -expm1f(z) * g;
        if (!(p == 0.f)) d[j] -= h * p * (z + H);
      }
    }
    store_vec<E>(out, e, V, d);
  }
}

template <class Args>
umim_status launch_rows(void (*kern)(Args), const Args &a, int R, const char *label, cudaStream_t stream) {
  trace_mark(stream, label);
  const cudaError_t e = launch_pdl(kern, dim3((unsigned)R), dim3(kThreads), 0, stream, a);
  trace_mark(stream, nullptr);
  return e == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

}  // namespace

umim_status token_logprobs(const void *logits, int dtype, int R, int V, int64_t ld, const int32_t *n_dev,
                           const int32_t *tokens, float temperature, int n_top, float *logprobs, float *entropy,
                           float *stats, int32_t *top_ids, float *top_logprobs, int32_t *dev_status,
                           cudaStream_t stream, int num_sms) {
  LogprobArgs a{logits, R, V, ld, n_dev, tokens, 1.f / temperature, n_top, logprobs, entropy,
                reinterpret_cast<float2 *>(stats), top_ids, top_logprobs, dev_status};
  auto *k = dtype == UMIM_DTYPE_BF16   ? token_logprobs_kernel<ElemBf16>
            : dtype == UMIM_DTYPE_FP16 ? token_logprobs_kernel<ElemFp16>
                                       : token_logprobs_kernel<ElemFp32>;
  return launch_rows(k, a, R, "logprobs.rows", stream);
}

umim_status token_logprobs_grad(const void *logits, int dtype, int R, int V, int64_t ld, const int32_t *n_dev,
                                const int32_t *tokens, float temperature, const float *stats, const float *entropy,
                                const float *g, const float *h, void *grad, int32_t *dev_status, cudaStream_t stream,
                                int num_sms) {
  GradArgs a{logits, R, V, ld, n_dev, tokens, 1.f / temperature, reinterpret_cast<const float2 *>(stats), entropy,
             g, h, grad, dev_status};
  auto *k = dtype == UMIM_DTYPE_BF16   ? token_logprobs_grad_kernel<ElemBf16>
            : dtype == UMIM_DTYPE_FP16 ? token_logprobs_grad_kernel<ElemFp16>
                                       : token_logprobs_grad_kernel<ElemFp32>;
  return launch_rows(k, a, R, "logprobs.grad", stream);
}

}  // namespace umim
