// What the decode attention kernels share: the split of a batch's pages over the
// warps of a persistent grid, the partial results that it leaves in the workspace
// and the kernel that merges them (attention.cu describes both).
#pragma once

#include <algorithm>

#include "common.cuh"

namespace umim {

using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                   const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                   CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                   CUtensorMapFloatOOBfill);
EncodeTiledFn get_encode_tiled();

constexpr int kAttnWarps = 12;        // warps of a decode CTA (one CTA an SM)
constexpr int kPlanThreadsA = 1024;
constexpr int kSmemPlanBatch = 4096;   // sequences whose prefix sum a decode CTA keeps in shared memory

struct AttnPlan {
  int32_t W;          // pages per warp
  int32_t total;      // (segment, page) pairs (attention_pages.cu)
  int32_t pad[62];
};

struct AttnWs {
  AttnPlan *plan;
  int32_t *pref;      // [B + 1] pages before sequence b (of one KV head)
  float2 *part_ml;    // [pieces][16]      (m in log2 units, l)
  float *part_acc;    // [pieces][16][D]
};

inline size_t a256(size_t x) { return (x + 255) & ~size_t(255); }

inline size_t attn_ws_bytes(int B, int Hkv, int D, int total_warps) {
  const size_t nseg = (size_t)B * Hkv;
  const size_t pieces = nseg + total_warps;
  size_t b = a256(sizeof(AttnPlan)) + a256(sizeof(int32_t) * (B + 1));
  b += a256(sizeof(float2) * pieces * 16);
  b += a256(sizeof(float) * pieces * 16 * D);
  return b;
}

inline AttnWs attn_carve(void *ws, int B, int Hkv, int D, int total_warps) {
  const size_t nseg = (size_t)B * Hkv;
  const size_t pieces = nseg + total_warps;
  char *p = static_cast<char *>(ws);
  AttnWs w;
  w.plan = reinterpret_cast<AttnPlan *>(p);
  p += a256(sizeof(AttnPlan));
  w.pref = reinterpret_cast<int32_t *>(p);
  p += a256(sizeof(int32_t) * (B + 1));
  w.part_ml = reinterpret_cast<float2 *>(p);
  p += a256(sizeof(float2) * pieces * 16);
  w.part_acc = reinterpret_cast<float *>(p);
  return w;
}

// ---------------------------------------------------------------------------
// plan
// ---------------------------------------------------------------------------
// Exclusive prefix sum of every sequence's pages into pref[0 .. B] by a block of
// T threads; returns the total (every thread).  A length outside the block
// table counts as 0 and is recorded when `report` is set.
template <int T>
__device__ int plan_prefix(const int32_t *seq_lens, int B, int max_pages, int32_t *pref, bool report,
                           int32_t *status) {
  static_assert(T <= 1024, "one warp scans the warps' sums");
  __shared__ int s_sum[32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int carry = 0;
  for (int b0 = 0; b0 < B; b0 += T) {
    const int b = b0 + threadIdx.x;
    int n = 0;
    if (b < B) {
      int L = seq_lens[b];
      if (L < 0 || (int64_t)L > (int64_t)max_pages * kPageSize) {
        if (report) set_error(status, UMIM_ERR_INVALID_ARG);
        L = 0;
      }
      n = ceil_div(L, kPageSize);
    }
    int x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) s_sum[w] = x;
    __syncthreads();
    int v = lane < T / 32 ? s_sum[lane] : 0;   // every warp scans the warps' sums
#pragma unroll
    for (int o = 1; o < T / 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += y;
    }
    const int before = w ? __shfl_sync(0xffffffffu, v, w - 1) : 0;
    if (b < B) pref[b] = carry + before + x - n;
    carry += __shfl_sync(0xffffffffu, v, T / 32 - 1);
    __syncthreads();
  }
  if (threadIdx.x == 0) pref[B] = carry;
  __syncthreads();
  return carry;
}

// more than kSmemPlanBatch sequences: the prefix sum in a kernel of its own (one block)
static __global__ void __launch_bounds__(kPlanThreadsA)
    attn_plan_kernel(const int32_t *seq_lens, int B, int max_pages, AttnWs ws, int32_t *status) {
  griddep_wait();
  plan_prefix<kPlanThreadsA>(seq_lens, B, max_pages, ws.pref, true, status);
}

// ---------------------------------------------------------------------------
// combine: WPR warps per (b, query head) row, 256 threads per CTA.  The warps
// of a row split its segment's pieces, each merges its share in one pass with
// a running maximum, and (WPR > 1) the warps' (m, l, acc) are merged through
// shared memory.  WPR grows with the pieces per segment (few, long sequences
// split into many pieces).
// ---------------------------------------------------------------------------
constexpr int kCombineThreads = 256;

// Merges n partial results, those that warp `sub` of `step` takes, into a running (M, l, o);
// a lane holds E columns of o.  ml(i), acc(i): where result i's (m, l) and this lane's columns are.
template <int E, typename Ml, typename Acc>
__device__ __forceinline__ void merge_pieces(int n, int sub, int step, float &M, float &l, float (&o)[E], Ml ml_of, Acc acc_of) {
  // pieces whose loads are in flight together: one at a time, a row of 76 pieces
  // (long context, 16.4 us with eight warps a row) waits for memory ten times over;
  // four at a time 8.3 us
  constexpr int U = 4;
  for (int pc = sub; pc < n; pc += U * step) {
    float2 ml[U];
    float av[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      ml[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int e = 0; e < E; ++e) av[u][e] = 0.f;
      if (pc + u * step < n) {
        ml[u] = *ml_of(pc + u * step);
        const float *src = acc_of(pc + u * step);
        if constexpr (E == 4) {
          const float4 f = *reinterpret_cast<const float4 *>(src);
          av[u][0] = f.x, av[u][1] = f.y, av[u][2] = f.z, av[u][3] = f.w;
        } else {
          const float2 f = *reinterpret_cast<const float2 *>(src);
          av[u][0] = f.x, av[u][1] = f.y;
        }
      }
    }
    float nm = M;
#pragma unroll
    for (int u = 0; u < U; ++u) nm = fmaxf(nm, ml[u].x);
    // (a piece whose scores are all NaN has no maximum either, but a NaN sum: weighted, not skipped)
    const float from = nm == -INFINITY ? 0.f : nm;
    const float c_old = exp2f(M - from);
    l *= c_old;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= c_old;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float c = exp2f(ml[u].x - from);   // 0 for an absent or empty piece
      l = fmaf(ml[u].y, c, l);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(av[u][e], c, o[e]);
    }
    M = nm;
  }
}

// the same for `n` consecutive pieces of 16 rows from row `first` on
template <int E>
__device__ __forceinline__ void merge_rows(const AttnWs &ws, int64_t first, int n, int sub, int step, float &M, float &l,
                                           float (&o)[E]) {
  const float2 *ml = ws.part_ml + first;
  const float *acc = ws.part_acc + first * (32 * E) + (threadIdx.x & 31) * E;
  merge_pieces<E>(n, sub, step, M, l, o, [&](int i) { return ml + (int64_t)i * 16; },
                  [&](int i) { return acc + (int64_t)i * (16 * 32 * E); });
}

template <int D, int WPR>
__global__ void __launch_bounds__(kCombineThreads)
    attn_combine_kernel(AttnWs ws, int B, int Hq, int Hkv, int G, __nv_bfloat16 *out) {
  constexpr int E = D / 32;
  constexpr int RPB = kCombineThreads / 32 / WPR;   // rows per CTA
  __shared__ float s_m[kCombineThreads / 32], s_l[kCombineThreads / 32];
  __shared__ float s_acc[WPR > 1 ? kCombineThreads / 32 : 1][D];
  griddep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row_g = blockIdx.x * RPB + warp / WPR, sub = warp % WPR;
  const bool live = row_g < B * Hq;
  const int b = live ? row_g / Hq : 0, h = live ? row_g % Hq : 0;
  const int seg = b * Hkv + h / G, row = h % G;
  // the segment's pieces: seg + w for the warps w whose ranges meet its positions
  int p0 = 0, p1 = 0;
  if (live) {
    const int first = ws.pref[b], n = ws.pref[b + 1] - first, W = ws.plan->W;
    const int o = Hkv * first + h / G * n;
    if (n > 0) {
      p0 = seg + o / W;
      p1 = seg + (o + n - 1) / W + 1;
    }
  }
  float M = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  merge_rows<E>(ws, (int64_t)p0 * 16 + row, p1 - p0, sub, WPR, M, l, o);
  if constexpr (WPR > 1) {
    if (lane == 0) {
      s_m[warp] = M;
      s_l[warp] = l;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_acc[warp][lane * E + e] = o[e];
    __syncthreads();
    if (sub != 0) return;
    float Mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < WPR; ++w) Mx = fmaxf(Mx, s_m[warp + w]);
    l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    if (Mx == -INFINITY) Mx = 0.f;
#pragma unroll
    for (int w = 0; w < WPR; ++w) {
      const float c = exp2f(s_m[warp + w] - Mx);
      l += c * s_l[warp + w];
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += c * s_acc[warp + w][lane * E + e];
    }
  }
  if (!live) return;
  const float inv = p1 > p0 ? 1.f / l : 0.f;   // (no entries: zeros)
  __nv_bfloat16 *dst = out + ((int64_t)b * Hq + h) * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = __float2bfloat16_rn(o[e] * inv);
}

// warps that merge a row: about half the pieces that a segment has
inline int combine_warps(int per_seg) { return per_seg >= 16 ? 8 : per_seg >= 8 ? 4 : per_seg >= 4 ? 2 : 1; }

}  // namespace umim
