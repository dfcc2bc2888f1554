// What the kernels of attention over the 8-bit cache and over shared prefixes
// have in common: their arguments, workspace, and the plan of the prefixes.
#pragma once

#include "attention.cuh"

namespace umim {

constexpr int kSharedMaxBatch = 4096;   // sequences and prefixes whose prefix sums lie in shared memory
constexpr int kSharedMaxPrefixes = 512;

struct PagesArgs {
  const __nv_bfloat16 *q;
  const int32_t *block_table, *seq_lens;
  const int32_t *prefix_table, *prefix_lens, *prefix_offsets;   // shared prefixes only
  int32_t B, Hq, Hkv, G, max_pages, n_pages, layer, n_layers;
  int32_t n_prefixes, max_prefix_pages;
  int32_t smem_plan;
  int32_t most_rows;   // prefixes of more rows (sequence, query head of one KV head) are the tensor cores' (attention_prefix.cu)
  float scale_log2;
  int32_t *status;
};

// a cache of either kind
struct CacheView {
  void *values, *scales;   // scales null: bf16
  int n_layers, n_pages, n_kv_heads;
};

// Where a prefix's work and rows are: exclusive sums over the prefixes, and the
// offsets made to increase.  [n + 1] each.
struct PrefixPlan {
  int32_t *first;    // first sequence
  int32_t *blocks;   // blocks of 16 rows; for the tensor cores, segments of one or two tiles of 128 rows
  int32_t *pages;    // page visits of one KV head (pages x blocks); for the tensor cores, key tiles x row tiles
};

// ---------------------------------------------------------------------------
// prefixes with many rows, on the tensor cores
// ---------------------------------------------------------------------------
constexpr int kTcRows = 128, kTcKeys = 128;
// Where that kernel runs, prefixes of more rows than this are its: a tile of 128 rows and 128 entries costs
// 16 to 23 ns of the GPU however many of the rows are there, eight pages 8 to 12 ns for every 16 rows here.
constexpr int kTcMinRows = 16;

__host__ __device__ inline int tile_sequences(int G) { return kTcRows / G; }   // whole sequences a tile of rows

// Whether it runs at all: it takes 4 us of its own, so when a batch of equal groups, their prefixes as long as the
// table is wide, would save as much (in ns: 1 a page and 16 rows, 1.5 for 8-bit pages, half for D = 64, against twice
// that a page and 128 rows).  16-bit, 8 heads, D = 128: 16 sequences of 4 query heads a KV head behind 3000 entries take 17.5 us
// either way, 24 take 19.0 with it and 21.5 without, 64 behind 500 entries 19.7 and 18.4, 64 behind 12000 38 and 110.
inline bool tc_pays(int B, int n, int G, int Hkv, int D, bool narrow, int max_prefix_pages) {
  if ((int64_t)B * G <= kTcMinRows) return false;
  const int64_t rows = ((int64_t)B * G + n - 1) / n, saved = (rows + 15) / 16 - 2 * ((rows + kTcRows - 1) / kTcRows);
  return (int64_t)Hkv * max_prefix_pages * n * saved * (narrow ? 3 : 2) * D > 2 * 4000 * 128;
}

// segments at most (of one KV head): pairs of row tiles, and a single one a prefix
inline int64_t tc_max_segments(int B, int n, int G) {
  return B / (2 * tile_sequences(G)) + std::min<int64_t>(n, (int64_t)B * G / (kTcMinRows + 1)) + 1;
}

// CTAs of the pages' kernel, `ctas` for all.  Both kernels run at once where each has a fair part of the
// work, the CTAs that this one leaves unused making room for the other's: 64 sequences behind 16384
// entries, 16384 of their own, 32/8 heads, D = 128: 51.4 -> 45.1 us on the device.  Below an
// eighth they run one after the other on the whole GPU: few CTAs take their time over many
// short sequences (64 of one page each beside 16384 entries: 41 -> 52 us).  A key tile of a row tile takes an SM
// about as long as 12 (16 bits) or 15 pages of 16 rows.
__device__ __forceinline__ int pages_ctas(int ctas, int64_t pages, int64_t tiles, bool narrow) {
  const int64_t all = pages + tiles * (narrow ? 15 : 12);
  if (pages * 8 <= all || pages * 10 >= all * 9) return ctas;   // (no work at all too)
  return (int)((ctas * pages + all / 2) / all);
}

// the key tiles of a prefix for its row tiles, 0 where its rows are too few for the tensor cores' kernel
__device__ __forceinline__ int2 tc_work(const PagesArgs &a, int sequences, int len) {
  const int tiles = sequences * a.G > a.most_rows ? ceil_div(sequences, tile_sequences(a.G)) : 0;
  return make_int2((tiles + 1) / 2, tiles * ceil_div(len, kTcKeys));
}
// the page visits of the rest
__device__ __forceinline__ int2 pages_work(const PagesArgs &a, int sequences, int len) {
  const int rows = sequences * a.G, nb = rows > a.most_rows ? 0 : ceil_div(rows, 16);
  return make_int2(nb, nb * ceil_div(len, kPageSize));
}

struct PagesWs {
  AttnWs at;
  PrefixPlan pre, tc;
  int32_t *tc_W;         // key tiles x row tiles of a CTA
  float2 *tc_ml;         // [pieces][128]
  float *tc_acc;         // [pieces][D / 8][128][8]
};

// Where column c of a row of a tensor-core kernel's piece is.  A warp there holds a row
// a lane and stores eight columns of its 32 rows at once, a kilobyte in one piece; the
// combine kernel reads whole 32-byte sectors.  (Rows of D columns one behind another
// took 32 lines a store: 4 us of a call of 37.)
template <int D>
__host__ __device__ __forceinline__ int64_t tc_acc_at(int64_t piece, int row, int c) {
  return piece * (kTcRows * D) + (c / 8) * (kTcRows * 8) + row * 8 + c % 8;
}

// segments of a batch: (sequence, KV head), and (prefix, KV head, block of rows) at most
inline size_t max_segments(int B, int n, int G, int Hkv) {
  return (size_t)Hkv * (B + (n > 0 ? (size_t)n + (size_t)B * G / 16 : 0));
}

// n = 0: no prefixes.  With base null the sizes only; returns the bytes.
inline size_t pages_carve(void *base, PagesWs *ws, int B, int n, int G, int Hkv, int D, int num_sms) {
  char *p = static_cast<char *>(base);
  size_t bytes = 0;
  auto take = [&](size_t b) {
    char *r = p + bytes;
    bytes += a256(b);
    return r;
  };
  const size_t pieces = max_segments(B, n, G, Hkv) + (size_t)std::max(1, num_sms) * kAttnWarps;
  PagesWs w{};
  w.at.plan = reinterpret_cast<AttnPlan *>(take(sizeof(AttnPlan)));
  w.at.pref = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * ((size_t)B + 1)));
  w.at.part_ml = reinterpret_cast<float2 *>(take(sizeof(float2) * pieces * 16));
  w.at.part_acc = reinterpret_cast<float *>(take(sizeof(float) * pieces * 16 * D));
  if (n > 0) {
    const size_t b = sizeof(int32_t) * ((size_t)n + 1);
    for (PrefixPlan *x : {&w.pre, &w.tc}) {
      x->first = reinterpret_cast<int32_t *>(take(b));
      x->blocks = reinterpret_cast<int32_t *>(take(b));
      x->pages = reinterpret_cast<int32_t *>(take(b));
    }
    w.tc_W = reinterpret_cast<int32_t *>(take(sizeof(int32_t)));
    if ((int64_t)B * G > kTcMinRows) {
      const size_t tc = 2 * ((size_t)Hkv * tc_max_segments(B, n, G) + std::max(1, num_sms));
      w.tc_ml = reinterpret_cast<float2 *>(take(sizeof(float2) * tc * kTcRows));
      w.tc_acc = reinterpret_cast<float *>(take(sizeof(float) * tc * kTcRows * D));
    }
  }
  if (ws) *ws = w;
  return bytes;
}

// ---------------------------------------------------------------------------
// plan
// ---------------------------------------------------------------------------
// The plan of the prefixes, by a CTA's first warp (a barrier follows at the
// caller's).  Offsets that decrease or leave [0, B] count as the largest before
// them, a length outside the table as 0; both are recorded when `report` is set.
// work(rows' sequences, entries): (blocks, page visits); the result is the sum of other's second.
template <typename Work, typename Other>
__device__ __forceinline__ int plan_prefixes(const PagesArgs &a, const PrefixPlan &p, bool report, Work work, Other other) {
  const int lane = threadIdx.x & 31, n = a.n_prefixes;
  int most = 0, pages = 0, blocks = 0, rest = 0;
  for (int i0 = 0; i0 <= n; i0 += 32) {
    const int i = i0 + lane;
    int o = i <= n ? (a.prefix_offsets ? a.prefix_offsets[i] : i * a.B) : 0;   // (no offsets: one prefix for all)
    if (o < 0 || o > a.B) {
      if (report) set_error(a.status, UMIM_ERR_INVALID_ARG);
      o = 0;
    }
    int x = o;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) x = max(x, __shfl_up_sync(0xffffffffu, x, d));   // (lanes below d: their own)
    x = max(x, most);
    if (report && i <= n && x != o) set_error(a.status, UMIM_ERR_INVALID_ARG);
    if (i <= n) p.first[i] = x;
    most = __shfl_sync(0xffffffffu, x, 31);
  }
  __syncwarp();
  for (int i0 = 0; i0 <= n; i0 += 32) {
    const int i = i0 + lane;
    int2 w = make_int2(0, 0);
    if (i < n) {
      const int L = a.prefix_lens[i];
      if (L < 0 || (int64_t)L > (int64_t)a.max_prefix_pages * kPageSize) {
        if (report) set_error(a.status, UMIM_ERR_INVALID_ARG);
      } else if (L > 0) {
        w = work(p.first[i + 1] - p.first[i], L);
        rest += other(p.first[i + 1] - p.first[i], L).y;
      }
    }
    int xb = w.x, xp = w.y;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int yb = __shfl_up_sync(0xffffffffu, xb, d), yp = __shfl_up_sync(0xffffffffu, xp, d);
      if (lane >= d) xb += yb, xp += yp;
    }
    if (i <= n) {
      p.blocks[i] = blocks + xb - w.x;
      p.pages[i] = pages + xp - w.y;
    }
    blocks += __shfl_sync(0xffffffffu, xb, 31);
    pages += __shfl_sync(0xffffffffu, xp, 31);
  }
  return __reduce_add_sync(0xffffffffu, rest);
}

// the last i in [0, n) with at[i] * times <= x
__device__ __forceinline__ int last_at_most(const int32_t *at, int n, int times, int x) {
  int l = 0, h = n;
  while (h - l > 1) {
    const int m = (l + h) >> 1;
    if (at[m] * times <= x) l = m;
    else h = m;
  }
  return l;
}

// a plan in shared memory: [3][n + 1] from `mem` on
__device__ __forceinline__ PrefixPlan plan_at(int32_t *mem, int n) {
  return PrefixPlan{mem, mem + (n + 1), mem + 2 * (n + 1)};
}

bool prefix_tc_launch(const CacheView &kv, int D, const PagesArgs &a, const PagesWs &ws, cudaStream_t stream, int num_sms);

}  // namespace umim
