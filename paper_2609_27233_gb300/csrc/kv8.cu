// The 8-bit paged cache: rows of K and V quantised as they are written (a
// prompt's, a step's new entries, a step with merges) and read back.
//
// A row is one head's K or V of one entry, D bf16 values: largest magnitude,
// scale code, D e4m3 codes (kv8.cuh has the rounding).  Bytes bound the calls on
// many rows: 2 D read and D + 1 written a row.  D / 16 lanes hold a row, 16
// values each (32 bytes and 16), so a warp takes 4 (D = 128)
// or 8 rows at once; the largest magnitude is a maximum of the bf16 bit patterns,
// which order as the magnitudes do, over packed pairs and then over the row's lanes.
// Scaling by a power of two is exact in fp32, so a value is rounded once.
#include <algorithm>

#include <cuda_fp16.h>

#include "kv8.cuh"

namespace umim {
namespace {

constexpr int kRowThreads = 256;
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 4;    // rows in flight a group of lanes
constexpr int kMaxCluster = 8;    // CTAs per sequence (portable cluster size)
// Heads of K and V that a warp takes of its rows.  Two: 32768 rows of 8 heads, D = 128, written in 31.8 us
// (6.3 TB/s; one 38.8, four 33.1), 65536 read in 62.9 (6.4 TB/s; one 77, four 62.6).
constexpr int kRowHeads = 2;

template <int D>
constexpr int kRowLanes = D / 16;   // lanes of a row
template <int D>
constexpr int kWarpRows = 32 / kRowLanes<D>;

struct Row {   // a lane's 16 values of a row, packed bf16 pairs
  uint32_t x[8];
};

__device__ __forceinline__ uint4 ld_row_v4(const void *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// A lane's 32 bytes in one access where rows start on 32-byte boundaries, else in two: rows a
// multiple of 16 bytes apart are all that a call asks for.
template <bool WIDE>
__device__ __forceinline__ void load_row(const uint16_t *p, Row &r) {
  if constexpr (WIDE) {
    asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r.x[0]), "=r"(r.x[1]), "=r"(r.x[2]), "=r"(r.x[3]), "=r"(r.x[4]), "=r"(r.x[5]), "=r"(r.x[6]),
                   "=r"(r.x[7])
                 : "l"(p));
    return;
  }
  const uint4 a = ld_row_v4(p), b = ld_row_v4(p + 8);
  r.x[0] = a.x, r.x[1] = a.y, r.x[2] = a.z, r.x[3] = a.w;
  r.x[4] = b.x, r.x[5] = b.y, r.x[6] = b.z, r.x[7] = b.w;
}

template <bool WIDE>
__device__ __forceinline__ void store_row(uint16_t *p, const uint32_t (&x)[8]) {
  if constexpr (WIDE) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x[0]), "r"(x[1]), "r"(x[2]),
                 "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4 *>(p)[0] = make_uint4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<uint4 *>(p)[1] = make_uint4(x[4], x[5], x[6], x[7]);
  }
}

// The row's codes (16 of this lane) and its scale code.  Every lane of the warp takes part.
template <int D>
__device__ __forceinline__ uint4 quantise(Row &r, uint32_t &code) {
  auto reduce = [](uint32_t m) {   // over the row's lanes, then over the pair
#pragma unroll
    for (int o = 1; o < kRowLanes<D>; o <<= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
    return max(m & 0xffff, m >> 16);
  };
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = __vmaxu2(m, r.x[i] & 0x7fff7fff);
  m = reduce(m);
  constexpr uint32_t kInf = 0x7f80;   // bf16 patterns from here on are infinite or NaN
  if (__any_sync(0xffffffffu, m > kKv8Top)) {
    // Those have no part in the scale, and all become NaN: the conversion would make the
    // largest number of an infinity.  Finite numbers above the largest that is stored become that.
    // (Selected value by value below: a call of 32 us took 36.)
    uint32_t f = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t a = r.x[i] & 0x7fff, b = r.x[i] >> 16 & 0x7fff;
      f = __vmaxu2(f, (a < kInf ? a : 0) | (b < kInf ? b : 0) << 16);
      r.x[i] = (r.x[i] & 0x80008000u) | (a < kInf ? min(a, kKv8Top) : 0x7fffu) | (b < kInf ? min(b, kKv8Top) : 0x7fffu) << 16;
    }
    m = reduce(f);
  }
  code = kv8_scale_code(m);
  const float inv = __uint_as_float((254u - code) << 23);   // 2^-(code - 127), a normal number
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t h[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t x = r.x[2 * i + j];
      h[j] = e4m3x2_of(__uint_as_float(x << 16) * inv, __uint_as_float(x & 0xffff0000u) * inv);
    }
    w[i] = h[0] | h[1] << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Row (layer, page, K|V, head, slot) of a cache: its number, which is the scale's
// offset; the values are at D times that.
__device__ __forceinline__ int64_t row_of(int layer, int n_pages, int page, int kv_head, int Hkv, int slot) {
  return (((int64_t)layer * n_pages + page) * (2 * Hkv) + kv_head) * kPageSize + slot;
}

// ---------------------------------------------------------------------------
// prompts' rows, or one row a sequence: written, and read back
// ---------------------------------------------------------------------------
struct RowsArgs {
  uint8_t *values, *scales;
  int32_t n_layers, n_pages, n_kv_heads, layer;
  const int32_t *block_table;
  int32_t max_pages;
  const int32_t *start;      // [B] the entry that a sequence's first row is
  const int32_t *cu_rows;    // [B + 1], or nullptr: one row a sequence
  int32_t B, T;
  uint16_t *k, *v;           // read by a write, written by a read
  int64_t stride;            // elements from one row's heads to the next row's
  uint64_t per_part;         // 2^34 / parts, rounded up: a division by the parts of a row is a product
  int32_t *status;
};

// The page and slot of row t, page -1 for a row that has none: outside every
// sequence (left as it is), or at an entry that the table does not hold (reported).
// The warp's rows are t0 .. t0 + 7 at most; every lane takes part.
__device__ __forceinline__ int2 place_of(const RowsArgs &a, int t0, int t) {
  int b = t, in = 0;
  if (a.cu_rows != nullptr) {
    // the last sequence that starts at or before t0: 32 probes a step
    int lo = 0, n = a.B;
    while (n > 1) {
      const int step = (n + 31) / 32, at = (int)(threadIdx.x & 31) * step;
      const int hit = __popc(__ballot_sync(0xffffffffu, at < n && a.cu_rows[lo + at] <= t0));
      if (hit == 0) break;
      lo += (hit - 1) * step;
      n = min(step, n - (hit - 1) * step);
    }
    b = lo;
    while (b + 1 < a.B && a.cu_rows[b + 1] <= t) ++b;
    const int first = a.cu_rows[b];
    if (first < 0 || t < first || t >= a.cu_rows[b + 1]) return make_int2(-1, 0);
    in = t - first;
  }
  if (t >= a.T) return make_int2(-1, 0);
  // (in 32 bits: a table has less than 2^27 pages, and there are 2^24 rows at most)
  const int start = a.start[b];
  const uint32_t entry = (uint32_t)start + in;
  int page = -1;
  if (start >= 0 && entry < (uint32_t)a.max_pages * kPageSize) page = a.block_table[(uint32_t)b * a.max_pages + entry / kPageSize];
  if ((uint32_t)page >= (uint32_t)a.n_pages) {
    set_error(a.status, UMIM_ERR_INVALID_ARG);
    page = -1;
  }
  return make_int2(page, (int)(entry % kPageSize));
}

// offsets that do not start at 0 or that decrease, or rows that are not there
__device__ __forceinline__ void check_rows(const RowsArgs &a) {
  if (a.cu_rows == nullptr) return;
  bool bad = threadIdx.x == 0 && (a.cu_rows[0] != 0 || a.cu_rows[a.B] > a.T);
  for (int b = threadIdx.x; b < a.B; b += blockDim.x) bad = bad || a.cu_rows[b + 1] < a.cu_rows[b];
  if (bad) set_error(a.status, UMIM_ERR_INVALID_ARG);
}

// One warp: kWarpRows consecutive rows of U heads of K and V, whose loads are in flight while the
// rows' pages are looked up.
template <int D, bool WIDE>
__global__ void __launch_bounds__(kRowThreads) kv8_write_kernel(RowsArgs a) {
  constexpr int U = kRowHeads;
  griddep_wait();
  if (blockIdx.x == 0) check_rows(a);
  const int lane = threadIdx.x & 31, heads = 2 * a.n_kv_heads, parts = ceil_div(heads, U);
  const int task = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  const int block = (int)(task * a.per_part >> 34);   // task / parts: task < 2^22 * parts, so that its error stays below 1 / parts
  const int t0 = block * kWarpRows<D>, h0 = (task - block * parts) * U;
  if (t0 >= a.T) return;
  const int t = t0 + lane / kRowLanes<D>, col = lane % kRowLanes<D> * 16;
  Row r[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = h0 + u;
    if (t < a.T && h < heads)
      load_row<WIDE>((h < a.n_kv_heads ? a.k + h * D : a.v + (h - a.n_kv_heads) * D) + t * a.stride + col, r[u]);
    else
      r[u] = Row{};
  }
  const int2 at = place_of(a, t0, t);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t code;
    const uint4 w = quantise<D>(r[u], code);
    const int h = h0 + u;
    if (at.x < 0 || h >= heads) continue;
    const int64_t row = row_of(a.layer, a.n_pages, at.x, h, a.n_kv_heads, at.y);
    if (!in_bounds(row, (int64_t)a.n_layers * a.n_pages * heads * kPageSize, a.status, kSiteKv8Dst)) continue;
    *reinterpret_cast<uint4 *>(a.values + row * D + col) = w;
    if (col == 0) a.scales[row] = (uint8_t)code;
  }
}

template <int D, bool WIDE>
__global__ void __launch_bounds__(kRowThreads) kv8_read_kernel(RowsArgs a) {
  constexpr int U = kRowHeads;
  griddep_wait();
  if (blockIdx.x == 0) check_rows(a);
  const int lane = threadIdx.x & 31, heads = 2 * a.n_kv_heads, parts = ceil_div(heads, U);
  const int task = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  const int block = (int)(task * a.per_part >> 34);   // task / parts: task < 2^22 * parts, so that its error stays below 1 / parts
  const int t0 = block * kWarpRows<D>, h0 = (task - block * parts) * U;
  if (t0 >= a.T) return;
  const int t = t0 + lane / kRowLanes<D>, col = lane % kRowLanes<D> * 16;
  const int2 at = place_of(a, t0, t);
  if (at.x < 0) return;
  uint4 w[U];
  uint32_t code[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = h0 + u;
    w[u] = make_uint4(0, 0, 0, 0);
    code[u] = 127;
    if (h >= heads) continue;
    const int64_t row = row_of(a.layer, a.n_pages, at.x, h, a.n_kv_heads, at.y);
    if (!in_bounds(row, (int64_t)a.n_layers * a.n_pages * heads * kPageSize, a.status, kSiteKv8Src)) continue;
    w[u] = ld_row_v4(a.values + row * D + col);
    code[u] = a.scales[row];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = h0 + u;
    if (h >= heads) continue;
    const float s = e8m0_value(code[u]);
    const uint32_t in[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
    uint32_t out[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t f = f16x2_of_e4m3x2(in[i / 2] >> (i & 1) * 16);
      const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&f));
      // exact: four significant bits, and 2^-109 <= |x| <= 240 * 2^120 for what a write makes
      const __nv_bfloat162 y = __floats2bfloat162_rn(x.x * s, x.y * s);
      out[i] = *reinterpret_cast<const uint32_t *>(&y);
    }
    uint16_t *p = (h < a.n_kv_heads ? a.k + h * D : a.v + (h - a.n_kv_heads) * D) + t * a.stride + col;
    store_row<WIDE>(p, out);
  }
}

// ---------------------------------------------------------------------------
// one entry for every sequence in all layers, appended or in place of a merged suffix
// ---------------------------------------------------------------------------
// A cluster a sequence, as for the 16-bit cache (append.cu): every CTA reads the
// length, the merge and the page and takes the same decision, and after a cluster
// barrier writes its share of the (layer, K|V, head) rows; rank 0 records
// the page, the released page and the length.  The new entry's rows are loaded
// before any of that is known: most sequences do not merge, and the chain of
// length, page and rows is what a step of few rows waits for.
struct AppendArgs {
  uint8_t *values, *scales;
  int32_t n_layers, n_pages, n_kv_heads;
  int32_t *block_table;
  int32_t max_pages;
  int32_t *seq_lens;
  const uint16_t *new_k, *new_v;   // [B][n_layers][Hkv][D]
  const int32_t *new_pages;        // [B] or nullptr
  const int32_t *merge_k;          // [B] or nullptr (append only)
  const int32_t *merge_row;        // [B]
  int32_t n_rows;                  // rows of the surrogate arrays
  const uint16_t *sur_k, *sur_v;   // [n_rows][n_layers][Hkv][D]
  int32_t *released;               // [B] or nullptr
  int32_t *status;
};

template <int D>
__global__ void __launch_bounds__(kAppendThreads) kv8_append_kernel(AppendArgs a, int C) {
  griddep_wait();
  constexpr int kGroups = kAppendThreads / kRowLanes<D>;   // rows that a CTA holds at once
  const int b = blockIdx.x / C, rank = blockIdx.x % C;
  const int group = threadIdx.x / kRowLanes<D>, col = threadIdx.x % kRowLanes<D> * 16;
  const int Hkv = a.n_kv_heads, total = a.n_layers * 2 * Hkv;   // rows, ordered [layer][K|V][head]
  const int per_step = kGroups * C;
  auto load = [&](const uint16_t *k, const uint16_t *v, int src, int r0, Row (&r)[kAppendRows]) {
#pragma unroll
    for (int u = 0; u < kAppendRows; ++u) {
      const int i = r0 + u * per_step;
      r[u] = Row{};
      if (i < total) {
        const int layer = i / (2 * Hkv), kv = (i / Hkv) & 1, h = i % Hkv;
        load_row<false>((kv ? v : k) + (((int64_t)src * a.n_layers + layer) * Hkv + h) * D + col, r[u]);
      }
    }
  };
  Row r[kAppendRows];
  const int first = rank * kGroups + group;
  load(a.new_k, a.new_v, b, first, r);

  __shared__ int s_page, s_slot, s_row, s_L, s_k;
  if (threadIdx.x == 0) {
    const int L = a.seq_lens[b];
    const int k = a.merge_k ? a.merge_k[b] : 0;
    bool ok = L >= 0 && (int64_t)L < (int64_t)a.max_pages * kPageSize && k >= 0 && k <= 16 && k <= L + 1;
    int page_L = -1;
    if (ok) {
      if (L % kPageSize == 0) page_L = a.new_pages ? a.new_pages[b] : -1;
      else page_L = a.block_table[(int64_t)b * a.max_pages + L / kPageSize];
      ok = page_L >= 0 && page_L < a.n_pages;
    }
    int slot = L, page = page_L, row = -1;
    if (ok && k > 0) {
      row = a.merge_row ? a.merge_row[b] : -1;
      slot = L + 1 - k;
      page = slot / kPageSize == L / kPageSize ? page_L : a.block_table[(int64_t)b * a.max_pages + slot / kPageSize];
      ok = row >= 0 && row < a.n_rows && page >= 0 && page < a.n_pages;
    }
    if (!ok) {
      if (rank == 0) set_error(a.status, UMIM_ERR_INVALID_ARG);
      page = -1;
    }
    s_page = page;
    s_slot = slot;
    s_row = row;
    s_L = L;
    s_k = k;
  }
  __syncthreads();
  cluster_sync_all();   // every CTA of this sequence has read L, k and the pages
  const int page = s_page, slot = s_slot, row = s_row, L = s_L, k = s_k;
  if (page < 0) return;   // this sequence is left unchanged

  if (k > 0) load(a.sur_k, a.sur_v, row, first, r);
  for (int r0 = rank * kGroups; r0 < total; r0 += per_step * kAppendRows) {   // the same steps in every lane
    if (r0 != rank * kGroups) load(k > 0 ? a.sur_k : a.new_k, k > 0 ? a.sur_v : a.new_v, k > 0 ? row : b, r0 + group, r);
#pragma unroll
    for (int u = 0; u < kAppendRows; ++u) {
      uint32_t code;
      const uint4 w = quantise<D>(r[u], code);
      const int i = r0 + group + u * per_step;
      if (i >= total) continue;
      const int64_t to = row_of(i / (2 * Hkv), a.n_pages, page, i % (2 * Hkv), Hkv, slot % kPageSize);
      if (!in_bounds(to, (int64_t)total * a.n_pages * kPageSize, a.status, kSiteKv8Dst)) continue;
      *reinterpret_cast<uint4 *>(a.values + to * D + col) = w;
      if (col == 0) a.scales[to] = (uint8_t)code;
    }
  }
  if (rank == 0 && threadIdx.x == 0) {
    int32_t *bt = a.block_table + (int64_t)b * a.max_pages;
    if (L % kPageSize == 0) bt[L / kPageSize] = a.new_pages[b];   // the append opened this page
    const int Ln = k > 0 ? slot + 1 : L + 1;
    const int had = (L + 1 + kPageSize - 1) / kPageSize, keep = (Ln + kPageSize - 1) / kPageSize;
    int rel = -1;
    if (keep < had) {   // k <= 16: at most one page
      rel = bt[keep];
      bt[keep] = -1;
    }
    if (a.released) a.released[b] = rel;
    a.seq_lens[b] = Ln;
  }
}

template <int D, bool WRITE>
umim_status launch_rows(RowsArgs a, cudaStream_t stream) {
  const bool wide = reinterpret_cast<uintptr_t>(a.k) % 32 == 0 && reinterpret_cast<uintptr_t>(a.v) % 32 == 0 && a.stride % 16 == 0;
  auto kern = WRITE ? (wide ? kv8_write_kernel<D, true> : kv8_write_kernel<D, false>)
                    : (wide ? kv8_read_kernel<D, true> : kv8_read_kernel<D, false>);
  const int parts = ceil_div(2 * a.n_kv_heads, kRowHeads);   // of a row: warps that share it, 64 at most
  a.per_part = ((uint64_t(1) << 34) + parts - 1) / parts;
  const int64_t warps = (int64_t)ceil_div(a.T, kWarpRows<D>) * parts;
  const int64_t blocks = (warps + kRowThreads / 32 - 1) / (kRowThreads / 32);
  trace_mark(stream, WRITE ? "kv8.write" : "kv8.read");
  const cudaError_t e = launch_pdl(kern, dim3((unsigned)blocks), dim3(kRowThreads), 0, stream, a);
  trace_mark(stream, nullptr);
  return e == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

}  // namespace

umim_status kv8_rows(bool write, const umim_paged_kv8 *kv, int layer, const int32_t *block_table, int max_pages,
                     const int32_t *start, const int32_t *cu_rows, int B, void *k, void *v, int T, int64_t stride,
                     int32_t *status, cudaStream_t stream) {
  RowsArgs a{};
  a.values = static_cast<uint8_t *>(kv->values);
  a.scales = static_cast<uint8_t *>(kv->scales);
  a.n_layers = kv->n_layers;
  a.n_pages = kv->n_pages;
  a.n_kv_heads = kv->n_kv_heads;
  a.layer = layer;
  a.block_table = block_table;
  a.max_pages = max_pages;
  a.start = start;
  a.cu_rows = cu_rows;
  a.B = B;
  a.T = T;
  a.k = static_cast<uint16_t *>(k);
  a.v = static_cast<uint16_t *>(v);
  a.stride = stride;
  a.status = status;
  if (kv->head_dim == 128) return write ? launch_rows<128, true>(a, stream) : launch_rows<128, false>(a, stream);
  return write ? launch_rows<64, true>(a, stream) : launch_rows<64, false>(a, stream);
}

umim_status kv8_append_merge(const umim_paged_kv8 *kv, int32_t *block_table, int32_t max_pages, int32_t *seq_lens,
                             int32_t B, const void *new_k, const void *new_v, const int32_t *new_pages,
                             const int32_t *merge_k, const int32_t *merge_row, int32_t n_rows, const void *sur_k,
                             const void *sur_v, int32_t *released, int32_t *status, cudaStream_t stream) {
  AppendArgs a{};
  a.values = static_cast<uint8_t *>(kv->values);
  a.scales = static_cast<uint8_t *>(kv->scales);
  a.n_layers = kv->n_layers;
  a.n_pages = kv->n_pages;
  a.n_kv_heads = kv->n_kv_heads;
  a.block_table = block_table;
  a.max_pages = max_pages;
  a.seq_lens = seq_lens;
  a.new_k = static_cast<const uint16_t *>(new_k);
  a.new_v = static_cast<const uint16_t *>(new_v);
  a.new_pages = new_pages;
  a.merge_k = merge_k;
  a.merge_row = merge_row;
  a.n_rows = n_rows;
  a.sur_k = static_cast<const uint16_t *>(sur_k);
  a.sur_v = static_cast<const uint16_t *>(sur_v);
  a.released = released;
  a.status = status;
  // CTAs per sequence: enough that a group of lanes has about kAppendRows rows
  const int per_cta = kAppendThreads / (kv->head_dim / 16) * kAppendRows;
  const int C = std::min(kMaxCluster, std::max(1, ceil_div(kv->n_layers * 2 * kv->n_kv_heads, per_cta)));
  auto kern = kv->head_dim == 128 ? kv8_append_kernel<128> : kv8_append_kernel<64>;
  trace_mark(stream, "kv8.append_merge");
  const cudaError_t e =
      launch_pdl_cluster(kern, dim3((unsigned)(B * C)), dim3(kAppendThreads), (unsigned)C, 0, stream, a, C);
  trace_mark(stream, nullptr);
  return e == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

}  // namespace umim
