// Attention of many query rows over a shared prefix, on the 5th-generation tensor
// cores: the part of umim_decode_attention_shared that is no longer bound by the
// cache's bytes.  The rows (sequence, query head) of a group that share a KV head
// are the rows of a matrix Q, and
//     S = Q K^T,   P = exp2(scale S - m),   O = P V,   l = sum P
// over a range of the prefix's entries is one partial result (m, l, O) a row,
// which the combine kernel (attention_pages.cu) joins with the row's others.
//
// What bounds it: not the tensor cores (10 us of 25 in the case below, alone on the GPU) and not HBM, but what a slot's
// tile goes through one step after the other: S, its way to the softmax warps, the
// softmax, P V, and the next S, some 4000 cycles in 16 bits, with two slots in turn to
// cover it.  64 sequences x 4 query heads a KV head behind 16384 entries, 8 KV heads, D = 128,
// 16 bits: a call of 45.1 us on the device, 51.4 where the own entries' kernel does not run beside this one but
// before it, 40.1 without the softmax; five 8-bit prefixes of 12000, 120 sequences: 87.2, without the softmax 73.7,
// without the conversions 76.8, without both 61.4.
//
// Work: a row tile is 128 rows (whole sequences), a key tile 128 entries (8 pages).  A
// segment is a pair of row tiles, or a single one, of a prefix and KV head;
// (segment, key tile) pairs are flattened, weighted by their row tiles, and every
// CTA of a persistent grid takes an equal contiguous range.  A CTA holds two slots,
// each with S and O in tensor memory, four softmax warps (a thread a row) and an
// issuing warp: the pair's row tiles over the same key tiles, or one row tile's even
// and odd key tiles.  The slots take turns on the tensor cores (one's O += P V and
// next S while the other's softmax runs), as two heads do in prefill.cu.
//
// P is taken as a bf16 number and a bf16 remainder, two products with V each (17
// significant bits; one bf16 P would cost as much as the output's own rounding):
// 512 + 1024 cycles of tensor cores a tile of 128 x 128 x 128.  P lies over the S
// that it came from (16 columns of S: 8 of P, 8 of its remainder).  K and V are
// read from the pages as they lie: K is K-major, V MN-major (64 columns of the head
// dimension x 8 entries a swizzle atom), so nothing is transposed.
//
// 16-bit pages: two 128-byte boxes of 16 rows each for K and for V, straight into
// the operands' place.  The last page is loaded from row n - 16 on where it holds n <
// 16 entries: TMA reads rows before the first as zeros, so that nothing behind the
// prefix's end is ever read; S is masked there.
//
// 8-bit pages: eight warps read e4m3 rows and make fp16 operands of them, code * 2^(e - E + 7) with E the largest e of the
// page's 16 rows: 57344 at most, and multiples of 2^-24, so off by 2^-40 of the page's largest
// at most; rows with e below E - 31 become zeros, which is 2^-31 of it at most.  (Converting
// to value * 2^e in bf16 took twice the instructions, and they bound the kernel.)  Rows that hold nothing but
// zeros count for no largest e, whatever scale they are stored with, and pages that are not there neither.  q
// becomes fp16 in place, below 2^15 by a power of two a row.  With r the row's and the page's
// powers of two times the scale, and F the page's largest exponent of V's rows,
//     w = 2^(r s + F - n + 7),   O = sum w v',   l = sum 2^(r s - m),   out = 2^(n - m - 14) O / l,
// n the running maximum of r s + F over rows of V that hold something, and m that of r s: the weights that
// multiply V are at most 2^15 and are one fp16 number each (2^-12 of themselves).  l has a maximum of its own, since a page may hold most of the weight and
// hardly any of the output: V's scales lie up to 2^220 apart.  A page's part of l is the sum of its w times 2^-(m + F - n + 7);
// in a tile with a page whose w of a weight of 1 would be below 2^-26 (so that its fp16 weights are all 0), or with
// a row of V of zeros, whose w may be any number, the exponentials are taken once more against m.
#include <cuda_fp16.h>

#include "attention_pages.cuh"
#include "kv8.cuh"
#include "tmem.cuh"

namespace umim {
namespace {

constexpr uint32_t kTcTmemCols = 512;   // S of the slots at 0 and 128, O at 256 and 384
constexpr int kTcStages = 2;            // K and V rings
constexpr int kAhead = 3;               // 8-bit: key tiles on their way into L2 ahead of their loads (1 % of a call)

// shared memory (bytes, every piece but the plan 1024-aligned)
template <int D>
struct TcSmem {
  static constexpr int kTile = 128 * D * 2;               // Q of a slot, K, V: D / 64 atoms of [128 rows][128 B]
  static constexpr int kK = 2 * kTile;
  static constexpr int kV = kK + kTcStages * kTile;
  static constexpr int kPlan = kV + kTcStages * kTile;
  static constexpr int kMost = kPlan + 12 * (kSharedMaxPrefixes + 1) + 1024;
};
// warps 0 and 3 copies, 1-2 products, from 4 on softmax, then the 8-bit values
constexpr int kSoftmax = 4, kConverters = 8;
// Softmax warps of a slot's 32 rows: two, with half the keys each, take 1600 cycles a tile in
// place of 2800.  8-bit pages: one, since the converters need registers too (with 28
// warps the 72 registers a thread spill into a cache that the operands leave no room for).
template <int BITS>
constexpr int kHalves = BITS == 8 ? 1 : 2;
template <int BITS>
constexpr int kConvert = kSoftmax + 8 * kHalves<BITS>;
template <int BITS>
constexpr int kTcThreads = 32 * (BITS == 8 ? kConvert<BITS> + kConverters : kConvert<BITS>);
// one CTA's part of a segment
struct TcUnit {
  int i, g, tile;     // prefix, KV head, first row tile
  bool two;           // a pair of row tiles
  int seg;            // segment, over all
  int len;            // the prefix's entries
  int t0, t1;         // key tiles
};

// The unit at position x of [x, end), and where the next one starts; false behind the last.
__device__ __forceinline__ bool unit_at(const PagesArgs &a, const PrefixPlan &p, int &x, int end, TcUnit &u) {
  while (x < end) {
    u.i = last_at_most(p.pages, a.n_prefixes, a.Hkv, x);
    const int work = p.pages[u.i + 1] - p.pages[u.i], ns = p.blocks[u.i + 1] - p.blocks[u.i];
    u.len = a.prefix_lens[u.i];
    const int keys = ceil_div(u.len, kTcKeys), tiles = work / keys;
    int r = x - a.Hkv * p.pages[u.i];
    u.g = r / work;
    r -= u.g * work;
    const int s = r / (2 * keys);
    u.tile = 2 * s;
    u.two = 2 * s + 1 < tiles;
    u.seg = a.Hkv * p.blocks[u.i] + u.g * ns + s;
    const int width = u.two ? 2 : 1, at = x - (r - 2 * s * keys), stop = min(end, at + keys * width);
    u.t0 = ceil_div(x - at, width);
    u.t1 = min(keys, ceil_div(stop - at, width));
    x = stop;
    if (u.t0 < u.t1) return true;
  }
  return false;
}

// Loads that stay where they are written, ahead of their use: the compiler moves plain ones to it.
__device__ __forceinline__ int ld_early(const int32_t *p) {
  int v;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ld_early_v2(const uint8_t *p) {
  uint2 v;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t ld_early_u8(const uint8_t *p) {
  uint16_t v;
  asm volatile("ld.global.u8 %0, [%1];" : "=h"(v) : "l"(p));
  return v;
}

// two fp32 numbers as fp16, those beyond its range as its largest
__device__ __forceinline__ uint32_t half2_within(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// a tile's 32 columns from x on whose positions lie in [lo, hi)
__device__ __forceinline__ uint32_t columns_in(int x, int lo, int hi) {
  lo = max(lo - x, 0), hi = min(hi - x, 32);
  return hi > lo ? (~0u >> (32 - (hi - lo))) << lo : 0u;
}

__device__ __forceinline__ void st_global_v8(float *p, float a, float b, float c, float d, float e, float f, float g, float h) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(a), "f"(b), "f"(c), "f"(d),
               "f"(e), "f"(f), "f"(g), "f"(h)
               : "memory");
}

// D x 128 keys, MN-major in 128-byte swizzle atoms of 64 columns x 8 keys: 1024 bytes to
// the next 8 keys, kTcKeys * 128 to the next 64 columns
__device__ __forceinline__ uint64_t sw128_mnmajor_desc(uint32_t smem_addr) {
  return sw128_kmajor_desc(smem_addr) + ((uint64_t)(kTcKeys * 128 / 16 - 1) << 16);   // (the K-major one's field is 1)
}
constexpr uint32_t kBMnMajor = 1u << 16;   // instruction descriptor: B is MN-major

// ---- a page of 8-bit rows of K and of V, as the warp that makes operands of it holds it: D / 8 lanes a key ----
template <int D>
struct Page8 {
  static constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes, kSteps = kPageSize / kAtOnce;
};

struct PageScales {
  // the largest codes of K's rows (in lanes 0-15) and of V's, and one more: 0 where no row counts, since those do not
  // that are NaN, zeros or behind the end
  uint32_t most, most_v;
  uint32_t factor;   // this lane's key's (lanes 0-15 K's, 16-31 V's) in units of 2^-7 of that, packed twice; 0 behind the end
  uint32_t zeros;    // the rows that are there and hold nothing: K's, from bit 16 on V's
};

// code: the scale of this lane's key
__device__ __forceinline__ PageScales page_scales(uint32_t code, int rem, uint32_t zeros) {
  const int lane = threadIdx.x & 31;
  PageScales r;
  const bool there = (lane & 15) < rem, zero = zeros >> lane & 1u;
  r.zeros = zeros;
  r.most = there && !zero && code != 255 ? code + 1 : 0;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) r.most = max(r.most, __shfl_xor_sync(0xffffffffu, r.most, o));
  r.most_v = __shfl_sync(0xffffffffu, r.most, 16);
  const int down = (int)code + 1 - (int)r.most;   // 0 or less of the rows that count
  const float scale = !there ? 0.f
                      : code == 255 ? NAN
                      : zero || down < -126 ? 0.f : __uint_as_float((uint32_t)(134 + down) << 23);
  const __half2 scale2 = __floats2half2_rn(scale, scale);
  r.factor = *reinterpret_cast<const uint32_t *>(&scale2);
  return r;
}

// Rows to fp16 operands at the page's place in a tile; rows from `rem` on as zeros (V's, so that 0 * garbage makes no
// NaN; K's scores are masked).  factor: of key i, in lane `first` + i.
template <int D>
__device__ __forceinline__ void convert_page(const uint2 (&in)[Page8<D>::kSteps], uint8_t *dst, uint32_t factor, int first,
                                             int rem) {
  constexpr int kLanes = Page8<D>::kLanes;
  const int lane = threadIdx.x & 31, part = lane % kLanes;
#pragma unroll
  for (int i = 0; i < Page8<D>::kSteps; ++i) {
    const int key = i * Page8<D>::kAtOnce + lane / kLanes;
    const uint32_t f = __shfl_sync(0xffffffffu, factor, first + key);
    const uint32_t x[2] = {key < rem ? in[i].x : 0u, key < rem ? in[i].y : 0u};
    uint32_t out[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t h = f16x2_of_e4m3x2(x[e / 2] >> (e & 1) * 16);
      const __half2 b = __hmul2(*reinterpret_cast<const __half2 *>(&h), *reinterpret_cast<const __half2 *>(&f));
      out[e] = *reinterpret_cast<const uint32_t *>(&b);
    }
    *reinterpret_cast<uint4 *>(dst + (part >> 3) * (kTcKeys * 128) + key * 128 + (((part & 7) ^ (key & 7)) << 4)) =
        make_uint4(out[0], out[1], out[2], out[3]);
  }
}

// A page that may hold rows of zeros: its scales without them, and K converted once more.  A call that reads everything
// again, since it is seldom made: beside the others' code, its own took a tenth of the kernel's time.
// row: K's first (values null: a page that is not there), V's rows_v further on.
template <int D>
__device__ __noinline__ PageScales page_again(const uint8_t *values, const uint8_t *scales, int64_t row, int rows_v, int rem,
                                              uint8_t *dst) {
  const int lane = threadIdx.x & 31;
  const uint8_t *rows = values ? values + row * D : nullptr;
  const uint32_t code = values ? scales[row + (lane >> 4) * rows_v + (lane & 15)] : 127u;
  bool zero = (lane & 15) < rem;
  if (zero && rows) {
    const uint4 *p = reinterpret_cast<const uint4 *>(rows + ((int64_t)(lane >> 4) * rows_v + (lane & 15)) * D);
    uint32_t any = 0;
    for (int i = 0; i < D / 16; ++i) any |= p[i].x | p[i].y | p[i].z | p[i].w;
    zero = !(any & 0x7f7f7f7f);
  }
  const PageScales r = page_scales(code, rem, __ballot_sync(0xffffffffu, zero));
  uint2 k[Page8<D>::kSteps];
#pragma unroll
  for (int i = 0; i < Page8<D>::kSteps; ++i)
    k[i] = rows ? *reinterpret_cast<const uint2 *>(rows + (i * 32 + lane) * 8) : make_uint2(0, 0);
  convert_page<D>(k, dst, r.factor, 0, kPageSize);
  return r;
}

template <int D, int BITS>
__global__ void __launch_bounds__(kTcThreads<BITS>, 1)
    prefix_tc_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap kv_map,
                     const uint8_t *values, const uint8_t *scales, PagesArgs a, PagesWs ws) {
  using L = TcSmem<D>;
  constexpr int DA = D / 64;
  constexpr int KS = kTcStages;
  extern __shared__ __align__(1024) uint8_t tc_raw[];
  __shared__ __align__(8) uint64_t q_full[2], q_empty[2], k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2],
      p_full[2][2], pv_done[2], o_free[2], turn[2], mma_done[2],
      met[2][4], q_ready[2], scales_full[4];
  // 8-bit: of the last four key tiles' pages, 2^(E - 7), F, the same or -infinity where there are rows of V of
  // zeros, and a bit for each of those
  __shared__ float4 s_scales[4][kTcKeys / kPageSize];
  __shared__ float s_row[2][2][2][kTcRows];   // [tile's parity][slot][half]: a row's maximum, or sum
  __shared__ uint32_t tmem_base;
  __shared__ int s_abort, s_pages;
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(tc_raw) + 1023) & ~uintptr_t(1023));
  const int warp = warp_index(), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    s_abort = 0;
    s_pages = 0;
    for (int s = 0; s < 2; ++s) {
      mbar_init(&k_full[s], BITS == 8 ? kConverters + 1 : 1);
      mbar_init(&k_empty[s], 2);   // read by both slots' products, or twice by one's
      mbar_init(&v_full[s], BITS == 8 ? kConverters : 1);
      mbar_init(&v_empty[s], 2);
      mbar_init(&q_full[s], 1);
      mbar_init(&q_empty[s], 1);     // a unit's S products have read the slot's Q
      mbar_init(&s_full[s], 1);
      mbar_init(&p_full[s][0], 4);   // keys 0-63 of P ready (four softmax warps)
      mbar_init(&p_full[s][1], 4);   // keys 64-127
      mbar_init(&pv_done[s], 1);     // a tile's P V product has landed
      mbar_init(&o_free[s], 4 * kHalves<BITS>);   // a unit's epilogue has read O
      mbar_init(&q_ready[s], 4);     // 8-bit: Q turned into fp16 (four softmax warps)
      for (int q = 0; q < 4; ++q) mbar_init(&met[s][q], 2);   // the two warps of 32 rows have left each other something
      mbar_init(&turn[s], 1);        // the other slot's products are issued
      mbar_init(&mma_done[s], 1);
    }
    for (int s = 0; s < 4; ++s) mbar_init(&scales_full[s], kConverters);
    fence_mbar_init();
    prefetch_tensormap(&q_map);
    if (BITS == 16) prefetch_tensormap(&kv_map);
  }
  if (warp == 1) {
    tmem_alloc(&tmem_base, kTcTmemCols);
    tmem_relinquish();
  }
  const PrefixPlan plan = plan_at(reinterpret_cast<int32_t *>(smem + L::kPlan), a.n_prefixes);
  const int spt = tile_sequences(a.G);   // sequences of a row tile
  // Nothing here waits for the kernel before: this one's inputs and workspace were
  // free when that one let it start (its own wait was over), and it waits at its end
  // for that one, for the combine kernel behind both.
  __syncthreads();   // (s_pages is 0)
  if (warp == 2) {   // (the kernel before reports)
    const int rest = plan_prefixes(a, plan, false, [&](int b, int len) { return tc_work(a, b, len); },
                                   [&](int b, int len) { return pages_work(a, b, len); });
    if (lane == 0) atomicAdd(&s_pages, rest);
  } else if (warp > 2) {   // the sequences' own pages, as the kernel before counts them
    int own = 0;
    for (int b = threadIdx.x - 96; b < a.B; b += kTcThreads<BITS> - 96) {
      const int len = a.seq_lens[b];
      if (len > 0 && (int64_t)len <= (int64_t)a.max_pages * kPageSize) own += ceil_div(len, kPageSize);
    }
    own = __reduce_add_sync(0xffffffffu, own);
    if (lane == 0 && own > 0) atomicAdd(&s_pages, own);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  const int total = a.Hkv * plan.pages[a.n_prefixes];
  const int others = pages_ctas((int)gridDim.x, (int64_t)a.Hkv * s_pages, total, BITS == 8);
  const int ctas = others == (int)gridDim.x ? others : (int)gridDim.x - others;   // (one after the other, or at once)
  const int W = max(2, ceil_div(total, ctas));   // (2: every CTA between a segment's first and last has a tile of it)
  const int start = (int)min((int64_t)blockIdx.x * W, (int64_t)total), end = min(start + W, total);
  if (blockIdx.x == 0) {   // for the combine kernel
    for (int i = threadIdx.x; i <= a.n_prefixes; i += kTcThreads<BITS>) {
      ws.tc.blocks[i] = plan.blocks[i];
      ws.tc.pages[i] = plan.pages[i];
    }
    if (threadIdx.x == 0) *ws.tc_W = W;
  }

  // a warp that gave up tells the others, so that no wait is left to time out on its own
  auto aborted = [&]() { return *reinterpret_cast<volatile int *>(&s_abort) != 0; };
  auto give_up = [&]() {
    set_error(a.status, UMIM_ERR_TIMEOUT);
    *reinterpret_cast<volatile int *>(&s_abort) = 1;
  };
  // the whole warp waits, and goes on only if all of it saw the phase
  auto wwait = [&](uint64_t *m, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_try_wait(smem_u32(m), parity) || (!aborted() && mbar_wait(m, parity))) != 0;
  };

  if (warp == 0 || warp == 3) {
    // ---- copies: Q, and 16-bit pages, K's by one warp and V's by the other, a lane a box: two of a
    // page of 128 columns.  (A box takes about 90 cycles to issue: one warp would be
    // busy for as long as the products of a tile take.) ----
    const int kv = warp == 0 ? 0 : 1;
    uint64_t *const full = kv ? v_full : k_full, *const empty = kv ? v_empty : k_empty;
    uint8_t *const to = smem + (kv ? L::kV : L::kK);
    int nq = 0, pos = 0;   // units, and key tiles
    bool ok = true;
    TcUnit u;
    for (int x = start; ok && unit_at(a, plan, x, end, u);) {
      for (int t = 0; t < 2 && ok && kv == 0; ++t) {
        if (nq > 0) ok = wwait(&q_empty[t], (uint32_t)(nq - 1) & 1u);
        if (ok && lane == 0) {
          mbar_arrive_expect_tx(&q_full[t], DA * spt * a.G * 128);
#pragma unroll
          for (int d = 0; d < DA; ++d)
            tma_load_4d(smem + t * L::kTile + d * (kTcRows * 128), &q_map, &q_full[t], d * 64, 0, u.g,
                        plan.first[u.i] + (u.tile + (u.two ? t : 0)) * spt);
        }
      }
      ++nq;
      const int n_pages = ceil_div(u.len, kPageSize), part = u.len % kPageSize, pg = lane & 7;
      const int32_t *table = a.prefix_table + (int64_t)u.i * a.max_prefix_pages;
      if constexpr (BITS == 8) {
        // the pages that the converters will load, on their way into L2: from HBM a tile
        // takes longer than the products of the one before.  A lane an operand's page.
        if (kv == 0) continue;
        auto prefetch = [&](int j) {
          const int at = j * 8 + pg;
          if (lane >= 16 || j >= u.t1 || at >= n_pages) return;
          const int page = table[at];
          if (page < 0 || page >= a.n_pages) return;
          const int64_t row = ((((int64_t)a.layer * a.n_pages + page) * 2 + (lane >> 3)) * a.Hkv + u.g) * kPageSize;
          asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(values + row * D), "r"(kPageSize * D) : "memory");
          asm volatile("prefetch.global.L2 [%0];" ::"l"(scales + row));
        };
        for (int i = 0; i < kAhead; ++i) prefetch(u.t0 + i);
        for (int j = u.t0; ok && j < u.t1; ++j, ++pos) {
          ok = wwait(&k_empty[pos % kTcStages], (uint32_t)(pos / kTcStages & 1) ^ 1u);
          if (!ok) break;
          prefetch(j + kAhead);
          __syncwarp();
          // (part of the tile's arrivals, though it has written nothing: no phase passes this warp unseen)
          if (elect_one()) mbar_arrive(&k_full[pos % kTcStages]);
        }
        continue;
      }
      auto page_at = [&](int j) {   // read a tile ahead
        const int at = j * 8 + pg;
        return j < u.t1 && at < n_pages && in_bounds(at, a.max_prefix_pages, a.status, kSitePrefixTable) ? ld_early(table + at) : 0;
      };
      int page = page_at(u.t0);
      for (int j = u.t0; ok && j < u.t1; ++j, ++pos) {
        const int at = j * 8 + pg, s = pos % kTcStages;
        int c = a.n_layers * a.n_pages;   // a coordinate past the tensor's last page: the copy reads zeros
        if (at < n_pages) {
          if (page >= 0 && page < a.n_pages) c = a.layer * a.n_pages + page;
          else set_error(a.status, UMIM_ERR_INVALID_ARG);
        }
        page = page_at(j + 1);
        ok = wwait(&empty[s], (uint32_t)(pos / kTcStages & 1) ^ 1u);
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&full[s], L::kTile);
        __syncwarp();
        if (lane < 8 * DA)
          tma_load_5d(to + s * L::kTile + (lane >> 3) * (kTcKeys * 128) + pg * (kPageSize * 128), &kv_map, &full[s],
                      (lane >> 3) * 64, at == n_pages - 1 && part ? part - kPageSize : 0, u.g, kv, c, policy_evict_last());
      }
    }
    if (!ok) {
      give_up();
      // copies still in flight when a consumer gave up: wait for them (bounded; a phase that has
      // completed, or was never armed, costs no more than a millisecond)
      for (int i = max(0, pos - kTcStages); i <= pos && BITS == 16; ++i)
        mbar_wait_for(&full[i % kTcStages], (uint32_t)(i / kTcStages & 1), 1000000);
      for (int t = 0; t < 2 && kv == 0; ++t)
        if (nq > 0) mbar_wait_for(&q_full[t], (uint32_t)(nq - 1) & 1u, 1000000);
    }
  } else if (warp <= 2) {
    // ---- the products of slot t, turn by turn: O += P V of its tile before as the halves of P
    // become ready, then S = Q K^T of its next tile once that has landed (P lies over S) ----
    const int t = warp - 1;
    if (elect_one()) {
      constexpr bool kHalf = BITS == 8;   // fp16 operands, and one product for P V
      constexpr uint32_t idesc_s = idesc_f32acc(kTcRows, kTcKeys, kHalf);
      constexpr uint32_t idesc_o = idesc_f32acc(kTcRows, D, kHalf) | kBMnMajor;
      uint64_t *const q_there = BITS == 8 ? q_ready : q_full;
      const uint32_t t_s = tmem + t * kTcKeys, t_o = tmem + 256 + t * 128;
      const uint64_t q_desc = sw128_kmajor_desc(smem_u32(smem) + t * L::kTile);
      int turns = 0, ns = 0, nu = 0;   // turns taken, S issued, units with a tile of this slot
      int pend = -1;                   // ring position of the tile whose P V is due
      bool pend_first = false, pend_two = false;
      bool landing = false;            // a P V product was issued and not waited for
      auto commits = [&](uint64_t *bar, bool two) {   // the slot's part of a stage's two readers, or both
        tc_commit(bar);
        if (!two) tc_commit(bar);
      };
      // rp: ring position of the tile whose S is next, -1 for none; nq: the unit's Q
      auto take_turn = [&](int rp, bool first, bool last, bool two, int nq) {
        const bool due = pend >= 0;
        const uint32_t pt = (uint32_t)(ns - 1) & 1u;
        if (due) {
          if (aborted() || !mbar_wait(&v_full[pend % KS], (uint32_t)(pend / KS & 1)) || !mbar_wait(&p_full[t][0], pt) ||
              (pend_first && nu > 1 && !mbar_wait(&o_free[t], (uint32_t)nu & 1u)))
            return false;
        }
        if ((t == 1 || turns > 0) && (aborted() || !mbar_wait(&turn[t], (uint32_t)(turns + t + 1) & 1u))) return false;
        ++turns;
        if (due) {
          const uint64_t v_desc = sw128_mnmajor_desc(smem_u32(smem + L::kV + pend % KS * L::kTile));
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h == 1 && !mbar_wait(&p_full[t][1], pt)) return false;
            tc_fence_after();
#pragma unroll
            for (int part = 0; part < (BITS == 8 ? 1 : 2); ++part)
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)   // 16 keys: a page
                tc_mma_ts(t_o, t_s + (h * 4 + kk) * (BITS == 8 ? 8 : 16) + part * 8,
                          v_desc + (h * 4 + kk) * (kPageSize * 128 / 16), idesc_o,
                          !pend_first || h || part || kk ? 1u : 0u);
          }
          tc_commit(&pv_done[t]);
          commits(&v_empty[pend % KS], pend_two);
          pend = -1;
          landing = true;
        }
        if (rp < 0) {
          mbar_arrive(&turn[t ^ 1]);
          return true;
        }
        if (aborted() || !mbar_wait(&k_full[rp % KS], (uint32_t)(rp / KS & 1)) ||
            (first && !mbar_wait(&q_there[t], (uint32_t)nq & 1u)) || (landing && !mbar_wait(&pv_done[t], pt)))
          return false;
        landing = false;
        const uint64_t k_desc = sw128_kmajor_desc(smem_u32(smem + L::kK + rp % KS * L::kTile));
        tc_fence_after();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          tc_mma_bf16(t_s, q_desc + (kk >> 2) * (kTcRows * 8) + (kk & 3) * 2,
                      k_desc + (kk >> 2) * (kTcKeys * 8) + (kk & 3) * 2, idesc_s, kk != 0 ? 1u : 0u);
        tc_commit(&s_full[t]);
        mbar_arrive(&turn[t ^ 1]);
        commits(&k_empty[rp % KS], two);
        if (last) tc_commit(&q_empty[t]);   // the unit's S products have read Q
        pend = rp;
        pend_first = first;
        pend_two = two;
        nu += first;
        ++ns;
        return true;
      };
      bool ok = true;
      int pos = 0, nq = 0, x = start;
      TcUnit u;
      bool more = unit_at(a, plan, x, end, u);
      for (int i = 0; ok;) {   // i: the unit's turns so far
        const int n = more ? u.t1 - u.t0 : 0, step = u.two ? 1 : 2, at = u.two ? i : 2 * i + t;
        const bool mine = more && at < n;
        ok = take_turn(mine ? pos + at : -1, i == 0, at + step >= n, u.two, nq);
        if (!more) break;   // (that was the last P V)
        if (ok && i == 0 && !mine) {   // no tile of this slot's: its Q is in nobody's way
          ok = mbar_wait(&q_there[t], (uint32_t)nq & 1u);
          if (ok) mbar_arrive(&q_empty[t]);
        }
        if (++i * step >= n) {
          pos += n;
          ++nq;
          i = 0;
          more = unit_at(a, plan, x, end, u);
        }
      }
      if (!ok) give_up();
      // every product this thread issued has finished before tensor memory is released
      tc_commit(&mma_done[t]);
      mbar_wait_for(&mma_done[t], 0, kWaitLimitNs);
    }
    __syncwarp();
  } else if (warp >= kSoftmax && warp < kConvert<BITS>) {
    // ---- softmax and partial results of slot t: a thread a query row, and all or half of the tile's keys ----
    constexpr int H = kHalves<BITS>, kKeys = kTcKeys / H, kCols = D / H;
    const int t = (warp - kSoftmax) >> (H == 2 ? 3 : 2), half = H == 2 ? (warp - kSoftmax) >> 2 & 1 : 0;
    const int quad = warp & 3;                 // tensor-memory lanes this warp may access
    const int r = quad * 32 + lane;            // row within the tile
    const uint32_t t_s = tmem + ((uint32_t)(quad * 32) << 16) + t * kTcKeys + half * kKeys;
    const uint32_t t_o = tmem + ((uint32_t)(quad * 32) << 16) + 256 + t * 128;
    bool ok = true;
    int ns = 0, meets = 0, nq = 0, pos = 0;   // tiles of the slot, exchanges, units, ring position of the unit's first tile
    // what the other warp of these rows left: a value a row
    auto exchange = [&](float mine, float &other, float alone) {
      other = alone;
      if (H == 1) return true;
      float (&slot)[2][kTcRows] = s_row[meets & 1][t];
      slot[half][r] = mine;
      __syncwarp();
      if (elect_one()) mbar_arrive(&met[t][quad]);
      const bool came = wwait(&met[t][quad], (uint32_t)meets & 1u);
      other = slot[half ^ 1][r];
      ++meets;
      return came;
    };
    TcUnit u;
    for (int x = start; ok && unit_at(a, plan, x, end, u);) {
      const int row_tile = u.tile + (u.two ? t : 0), seq = plan.first[u.i] + row_tile * spt + r / a.G;
      const bool live = r < spt * a.G && seq < plan.first[u.i + 1];
      const bool any = __any_sync(0xffffffffu, live);   // (warps without rows only keep the others going)
      float m_run = -INFINITY, l_run = 0.f;             // running max (log2 units, moved in steps > 8) and row sum
      float top = -INFINITY;                            // 8-bit: the largest score, which the row sum is relative to
      int mine = 0;                                     // tiles
      float sl2 = a.scale_log2;
      if constexpr (BITS == 8) {
        // the row of Q to fp16, its largest magnitude in [2^14, 2^15); rows of zeros (or below 2^-86)
        // and ones that hold no number by a fixed power
        ok = wwait(&q_full[t], (uint32_t)nq & 1u);
        if (!ok) break;
        uint8_t *row = smem + t * L::kTile + r * 128;
        uint32_t m = 0;
#pragma unroll 1
        for (int c = 0; c < D / 8; ++c) {
          const uint4 v = *reinterpret_cast<const uint4 *>(row + (c >> 3) * (kTcRows * 128) + (((c & 7) ^ (r & 7)) << 4));
          m = __vmaxu2(m, __vmaxu2(__vmaxu2(v.x & 0x7fff7fff, v.y & 0x7fff7fff), __vmaxu2(v.z & 0x7fff7fff, v.w & 0x7fff7fff)));
        }
        m = max(m & 0xffff, m >> 16) >> 7;
        const uint32_t e = m == 255 ? 127u : max(m, 41u);
        const float inv = __uint_as_float((268u - e) << 23);   // 2^(14 - (e - 127))
        sl2 *= __uint_as_float((e - 14) << 23);
#pragma unroll 1
        for (int c = 0; c < D / 8; ++c) {
          uint4 *at = reinterpret_cast<uint4 *>(row + (c >> 3) * (kTcRows * 128) + (((c & 7) ^ (r & 7)) << 4));
          auto half2_of = [&](uint32_t v) {
            const __half2 h = __floats2half2_rn(__uint_as_float(v << 16) * inv, __uint_as_float(v & 0xffff0000u) * inv);
            return *reinterpret_cast<const uint32_t *>(&h);
          };
          const uint4 v = *at;
          *at = make_uint4(half2_of(v.x), half2_of(v.y), half2_of(v.z), half2_of(v.w));
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (elect_one()) mbar_arrive(&q_ready[t]);
        ++nq;
      }
      for (int j = u.t0 + (u.two ? 0 : t); j < u.t1; j += u.two ? 1 : 2, ++mine, ++ns) {
        ok = wwait(&s_full[t], (uint32_t)ns & 1u);
        if (!ok) break;
        tc_fence_after();
        if (!any) {
          tc_fence_before();
          __syncwarp();
          if (elect_one()) {
            mbar_arrive(&p_full[t][half]);
            if (H == 1) mbar_arrive(&p_full[t][1]);
          }
          continue;
        }
        const int rem = u.len - j * kTcKeys - half * kKeys;   // keys from this warp's first on
        auto mask = [&](float (&s)[32], int x) {
          if (rem >= x + 32) return;
          // 16-bit pages: the last page's entries are its last rows
          const int left = max(rem, 0), full = left / kPageSize * kPageSize, part = left % kPageSize;
          const uint32_t bits = BITS == 8 ? columns_in(x, 0, left)
                                          : columns_in(x, 0, full) | columns_in(x, full + kPageSize - part, full + kPageSize);
#pragma unroll
          for (int c = 0; c < 32; ++c) s[c] = bits >> c & 1u ? s[c] : -INFINITY;
        };
        auto largest = [&](const float (&s)[32]) {
          float m4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
          for (int c = 4; c < 32; c += 2) m4[(c >> 1) & 3] = max3f(m4[(c >> 1) & 3], s[c], s[c + 1]);
          return fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
        };
        // 8-bit: of each page, the powers of two of K's and V's rows
        const float4 *scale = s_scales[(pos + j - u.t0) & 3];
        if constexpr (BITS == 8) {
          ok = wwait(&scales_full[(pos + j - u.t0) & 3], (uint32_t)((pos + j - u.t0) >> 2) & 1u);
          if (!ok) break;
        }
        auto factor = [&](int page) { return fmaxf(sl2 * scale[page].x, 1e-37f); };   // (never 0: -inf stays -inf)
        float s[32], mx = -INFINITY, most = -INFINITY, low = INFINITY, other;
#pragma unroll 1
        for (int c = kKeys / 32 - 1; c >= 0; --c) {   // (the first 32 last: they are still there below)
          tmem_ld_32x32b_x32(t_s + c * 32, s);
          mask(s, c * 32);
          if constexpr (BITS == 8) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              float m2[2] = {s[16 * g], s[16 * g + 1]};
#pragma unroll
              for (int x = 2; x < 16; x += 4) {
                m2[0] = max3f(m2[0], s[16 * g + x], s[16 * g + x + 1]);
                if (x + 2 < 16) m2[1] = max3f(m2[1], s[16 * g + x + 2], s[16 * g + x + 3]);
              }
              const float y = fmaxf(m2[0], m2[1]) * factor(2 * c + g);
              most = fmaxf(most, y);
              low = fminf(low, scale[2 * c + g].z);
              mx = fmaxf(mx, y + scale[2 * c + g].y);
            }
          } else {
            mx = fmaxf(mx, largest(s));
          }
        }
        ok = exchange(mx, other, mx);
        if (!ok) break;
        mx = BITS == 8 ? mx : fmaxf(mx, other) * sl2;
        float from = 0.f;   // 8-bit: a page's w times 2^(from - F) are its part of the row sum
        bool apart = false;
        if constexpr (BITS == 8) {
          const float was = top;
          top = fmaxf(top, most);
          const float top0 = top == -INFINITY ? 0.f : top;   // (no finite score so far: a sum of NaN stays NaN)
          l_run *= ex2_approx(was - top0);
          const float n = mx > m_run + 8.f ? mx : m_run;   // (as below)
          from = n == -INFINITY ? INFINITY : n - top0 - 7.f;
          apart = __any_sync(0xffffffffu, live && !(from - low < 26.f));   // (one answer for the warp)
          if (__builtin_expect(apart, 0)) {   // the row sum by itself, and the largest weight without the rows of zeros
            const float2 m2 = make_float2(-top0, -top0);
            mx = -INFINITY;
#pragma unroll 1
            for (int c = kKeys / 32 - 1; c >= 0; --c) {
              tmem_ld_32x32b_x32(t_s + c * 32, s);
              mask(s, c * 32);
#pragma unroll
              for (int g = 0; g < 2; ++g) {
                const float k = factor(2 * c + g);
                const uint32_t none = __float_as_uint(scale[2 * c + g].w);
                float2 sum = make_float2(0.f, 0.f);
                float y = -INFINITY;
#pragma unroll
                for (int x = 0; x < 16; x += 2) {
                  const float2 z = make_float2(s[g * 16 + x], s[g * 16 + x + 1]);
                  const float2 e = __ffma2_rn(z, make_float2(k, k), m2);
                  sum = __fadd2_rn(sum, make_float2(ex2_approx(e.x), ex2_approx(e.y)));
                  y = max3f(y, none >> x & 1u ? -INFINITY : z.x, none >> x & 2u ? -INFINITY : z.y);
                }
                l_run += sum.x + sum.y;
                mx = fmaxf(mx, y * k + scale[2 * c + g].y);
              }
            }
          }
        }
        // move the running max only when it grows by more than 2^8
        const bool grow = mx > m_run + 8.f;
        float alpha = 1.f;
        if (grow) {
          alpha = (m_run == -INFINITY) ? 0.f : ex2_approx(m_run - mx);
          m_run = mx;
          if (BITS == 16) l_run *= alpha;
        }
        // O is rescaled before the tile's first product, of half 0 (the tile before's has landed: S followed it)
        if (half == 0 && mine > 0 && __any_sync(0xffffffffu, grow)) {
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            float o[16];
            tmem_ld_32x32b_x16(t_o + c * 16, o);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= alpha;
            tmem_put_32x32b_x16(t_o + c * 16, o);
          }
          tmem_wait_st();
        }
        const float nm = (m_run == -INFINITY) ? 0.f : -m_run;
        const float2 minus = make_float2(-1.f, -1.f);
        float2 sl2x2 = make_float2(sl2, sl2), nm2 = make_float2(nm, nm), la = make_float2(0.f, 0.f), lb = la;
#pragma unroll (H == 2 ? 2 : 1)   // (four chunks unrolled: their code is fetched over and over, and registers spill)
        for (int h = 0; h < kKeys / 32; ++h) {
          if (h > 0) {
            tmem_ld_32x32b_x32(t_s + h * 32, s);
            mask(s, h * 32);
          }
          if constexpr (BITS == 8) {
            float p[16];   // the weights of 32 keys in fp16 pairs
#pragma unroll
            for (int g = 0; g < 2; ++g) {   // a page
              const float f = scale[2 * h + g].y, k = factor(2 * h + g), off = f + nm + 7.f;
              sl2x2 = make_float2(k, k), nm2 = make_float2(off, off);
              la = lb = make_float2(0.f, 0.f);
#pragma unroll
              for (int c = 0; c < 16; c += 2) {
                const float2 x = __ffma2_rn(make_float2(s[g * 16 + c], s[g * 16 + c + 1]), sl2x2, nm2);
                const float2 y = make_float2(ex2_approx(x.x), ex2_approx(x.y));   // masked (-inf): 0
                if (c & 2) lb = __fadd2_rn(lb, y);
                else la = __fadd2_rn(la, y);
                p[g * 8 + c / 2] = __uint_as_float(half2_within(y.x, y.y));   // (a row of zeros: times 0)
              }
              const float2 lab = __fadd2_rn(la, lb);
              if (!apart) l_run = fmaf(lab.x + lab.y, ex2_approx(from - f), l_run);
            }
            // over S columns that have been read: 16 for each 32
            tmem_put_32x32b_x16(t_s + h * 16, p);
          } else {
#pragma unroll
            for (int g = 0; g < 2; ++g) {   // 16 keys: P (<= 2^8) in bf16 pairs, and what that leaves
              float p[16];
#pragma unroll
              for (int c = 0; c < 16; c += 2) {
                const float2 x = __ffma2_rn(make_float2(s[g * 16 + c], s[g * 16 + c + 1]), sl2x2, nm2);
                const float2 y = make_float2(ex2_approx(x.x), ex2_approx(x.y));   // masked (-inf): 0
                if (c & 2) lb = __fadd2_rn(lb, y);
                else la = __fadd2_rn(la, y);
                const __nv_bfloat162 b = __floats2bfloat162_rn(y.x, y.y);
                const uint32_t hi = *reinterpret_cast<const uint32_t *>(&b);
                const float2 d = __ffma2_rn(make_float2(__uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u)), minus, y);
                const __nv_bfloat162 rest = __floats2bfloat162_rn(d.x, d.y);
                p[c / 2] = __uint_as_float(hi);
                p[8 + c / 2] = __uint_as_float(*reinterpret_cast<const uint32_t *>(&rest));
              }
              // over the S columns they come from, which this thread has read
              tmem_put_32x32b_x16(t_s + h * 32 + g * 16, p);
            }
          }
          if (h & 1) {   // 64 keys
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (elect_one()) mbar_arrive(&p_full[t][H == 2 ? half : h / 2]);
          }
        }
        if constexpr (BITS == 16) {
          const float2 lab = __fadd2_rn(la, lb);
          l_run += lab.x + lab.y;
        }
      }
      pos += u.t1 - u.t0;
      if (!ok) break;
      // the unit's partial result, half the columns a warp
      const int64_t piece = 2 * ((int64_t)u.seg + blockIdx.x) + t;
      const bool store = live && in_bounds(piece, 2 * ((int64_t)a.Hkv * plan.blocks[a.n_prefixes] + gridDim.x), a.status,
                                           kSitePrefixPiece);
      float other;
      ok = exchange(l_run, other, 0.f);
      if (!ok) break;
      if (store && half == 0) ws.tc_ml[piece * kTcRows + r] = make_float2(BITS == 8 ? top : m_run, l_run + other);
      float *dst = ws.tc_acc + tc_acc_at<D>(piece, r, half * kCols);
      if (mine > 0) {
        ok = wwait(&pv_done[t], (uint32_t)(ns - 1) & 1u);
        if (!ok) break;
        tc_fence_after();
        if (any) {
          // 8-bit: from O's units to the row sum's (n - m is at most a cache row's exponent)
          const float up = m_run == -INFINITY ? 1.f : exp2f(m_run - top);
#pragma unroll 1
          for (int c = 0; c < kCols / 32; ++c) {
            float o[32];
            tmem_ld_32x32b_x32(t_o + half * kCols + c * 32, o);
            if constexpr (BITS == 8)
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = o[i] * 0x1p-14f * up;
            if (store)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                st_global_v8(dst + (c * 4 + i) * (kTcRows * 8), o[8 * i], o[8 * i + 1], o[8 * i + 2], o[8 * i + 3],
                             o[8 * i + 4], o[8 * i + 5], o[8 * i + 6], o[8 * i + 7]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (elect_one()) mbar_arrive(&o_free[t]);
      } else if (store) {
        for (int i = 0; i < kCols / 8; ++i) st_global_v8(dst + i * (kTcRows * 8), 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f);
      }
    }
    if (!ok) give_up();
  } else if (warp >= kConvert<BITS>) {
    // ---- 8-bit values to fp16 operands: a warp a page of the tile, D / 8 lanes a key.  A tile's
    // values come straight from the pages into registers, a tile ahead: through shared
    // memory they left room for one stage of K, whose products then waited for its
    // conversion, and that for the products before ----
    if constexpr (BITS == 8) {
      constexpr int kLanes = Page8<D>::kLanes, kAtOnce = Page8<D>::kAtOnce, kSteps = Page8<D>::kSteps;
      static_assert(kConverters * kPageSize == kTcKeys, "a warp a page");
      const int w = warp - kConvert<BITS>, part = lane % kLanes;
      const int own = lane / kLanes * D + part * 8;   // this lane's place in a step's keys
      bool ok = true;
      int pos = 0;
      TcUnit u;
      for (int x = start; ok && unit_at(a, plan, x, end, u);) {
        const int n_pages = ceil_div(u.len, kPageSize);
        const int32_t *table = a.prefix_table + (int64_t)u.i * a.max_prefix_pages;
        // this warp's page of a tile, read two tiles ahead; -1 for none, which reads as zeros
        auto page_of = [&](int j) {
          const int at = j * 8 + w;
          if (j >= u.t1 || at >= n_pages || !in_bounds(at, a.max_prefix_pages, a.status, kSitePrefixTable)) return -1;
          return ld_early(table + at);
        };
        auto checked = [&](int page, int j) {
          if (page >= 0 && page < a.n_pages) return page;
          if (j < u.t1 && j * 8 + w < n_pages) set_error(a.status, UMIM_ERR_INVALID_ARG);
          return -1;
        };
        auto row_at = [&](int page, int kv) {   // the page's first row of K or V
          return ((((int64_t)a.layer * a.n_pages + page) * 2 + kv) * a.Hkv + u.g) * kPageSize;
        };
        auto load = [&](uint2 (&v)[kSteps], int page, int kv) {
          const uint8_t *p = values + row_at(page, kv) * D + own;
#pragma unroll
          for (int i = 0; i < kSteps; ++i) v[i] = page >= 0 ? ld_early_v2(p + i * kAtOnce * D) : make_uint2(0, 0);
        };
        auto code_of = [&](int page) {   // a key's: lanes 0-15 K's, 16-31 V's
          return page >= 0 ? ld_early_u8(scales + row_at(page, lane >> 4) + (lane & 15)) : 127u;
        };
        // 0 where a row might be zeros: its first eight bytes say of most that they are not (lanes of part 0)
        auto least_of = [&](const uint2 (&in)[kSteps]) {
          uint32_t least = 0xffffffffu;
#pragma unroll
          for (int i = 0; i < kSteps; ++i) least = min(least, (in[i].x | in[i].y) & 0x7f7f7f7f);
          return least;
        };
        // The order below: a wait for one load is a wait for all loads before it, so what the short ones
        // bring is used before the next long ones are issued.
        uint2 k[kSteps], v[kSteps], v_next[kSteps];
        int page = checked(page_of(u.t0), u.t0);
        uint32_t code = code_of(page);
        load(k, page, 0);
        load(v, page, 1);
        PageScales of = page_scales(code, u.len - (u.t0 * 8 + w) * kPageSize, 0);
        int next = checked(page_of(u.t0 + 1), u.t0 + 1);
        for (int j = u.t0; ok && j < u.t1; ++j, ++pos) {
          const int rem = u.len - (j * 8 + w) * kPageSize;   // keys from the page's first on
          const int s = pos % kTcStages;
          code = code_of(next);
          page = page_of(j + 2);
          ok = wwait(&k_empty[s], (uint32_t)(pos / kTcStages & 1) ^ 1u);
          if (!ok) break;
          uint8_t *const k_at = smem + L::kK + s * L::kTile + w * (kPageSize * 128);
          convert_page<D>(k, k_at, of.factor, 0, kPageSize);
          // (V is a tile ahead like K, so that both are looked at before the softmax warps need their scales)
          const bool doubt = __any_sync(0xffffffffu, part == 0 && min(least_of(k), least_of(v)) == 0);
          if (__builtin_expect(doubt && rem > 0, 0)) {
            const int here = checked(page_of(j), j);
            of = page_again<D>(here >= 0 ? values : nullptr, scales, here >= 0 ? row_at(here, 0) : 0, a.Hkv * kPageSize, rem, k_at);
          }
          if (lane == 0) {   // (four tiles' scales: S of the tile two before is done, so the softmax of the one four before is)
            // (a page without values of V: F below any other's; one behind the end: above, so that it is not the tile's least)
            const float f = rem <= 0 ? 1e30f : of.most_v ? (float)((int)of.most_v - 128) : -1e30f;
            const uint32_t none = of.zeros >> 16;
            s_scales[pos & 3][w] =
                make_float4(e8m0_value(max(of.most, 1u) - 1) * 0x1p-7f, f, none ? -INFINITY : f, __uint_as_float(none));
            mbar_arrive(&scales_full[pos & 3]);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (elect_one()) mbar_arrive(&k_full[s]);
          const uint32_t factor_v = of.factor;
          of = page_scales(code, rem - kTcKeys, 0);   // the next tile's
          page = checked(page, j + 2);
          load(k, next, 0);
          load(v_next, next, 1);
          ok = wwait(&v_empty[s], (uint32_t)(pos / kTcStages & 1) ^ 1u);
          if (!ok) break;
          convert_page<D>(v, smem + L::kV + s * L::kTile + w * (kPageSize * 128), factor_v, 16, rem);
          fence_proxy_async_smem();
          __syncwarp();
          if (elect_one()) mbar_arrive(&v_full[s]);
#pragma unroll
          for (int i = 0; i < kSteps; ++i) v[i] = v_next[i];
          next = page;
        }
      }
      if (!ok) give_up();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTcTmemCols);
  }
  griddep_wait();
}

template <int D, int BITS>
bool launch(const CacheView &kv, const PagesArgs &a, const PagesWs &ws, cudaStream_t stream, int num_sms) {
  using L = TcSmem<D>;
  static_assert(L::kMost + 6144 <= 232448, "shared memory of a CTA");
  EncodeTiledFn enc = get_encode_tiled();
  if (!enc) return false;
  CUtensorMap q_map, kv_map;
  const cuuint32_t one[5] = {1, 1, 1, 1, 1};
  const cuuint64_t H = kv.n_kv_heads, N = (cuuint64_t)kv.n_layers * (cuuint64_t)kv.n_pages, G = a.G;
  const cuuint64_t q_dims[4] = {(cuuint64_t)D, G, H, (cuuint64_t)a.B};
  const cuuint64_t q_strides[3] = {D * 2, G * D * 2, H * G * D * 2};
  const cuuint32_t q_box[4] = {64, (cuuint32_t)G, 1, (cuuint32_t)tile_sequences(a.G)};
  if (enc(&q_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<__nv_bfloat16 *>(a.q), q_dims, q_strides, q_box, one,
          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return false;
  kv_map = q_map;
  if (BITS == 16) {
    const cuuint64_t row = D * 2, dims[5] = {(cuuint64_t)D, 16, H, 2, N};
    const cuuint64_t strides[4] = {row, 16 * row, H * 16 * row, 2 * H * 16 * row};
    const cuuint32_t box[5] = {64, 16, 1, 1, 1};
    if (enc(&kv_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, kv.values, dims, strides, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return false;
  }
  auto kern = prefix_tc_kernel<D, BITS>;
  if (!allow_smem(kern, L::kMost)) return false;
  const size_t smem = L::kPlan + 1024 + 12 * ((size_t)a.n_prefixes + 1);
  return launch_pdl(kern, dim3((unsigned)std::max(1, num_sms)), dim3(kTcThreads<BITS>), smem, stream, q_map, kv_map,
                    static_cast<const uint8_t *>(kv.values), static_cast<const uint8_t *>(kv.scales), a, ws) == cudaSuccess;
}

}  // namespace

bool prefix_tc_launch(const CacheView &kv, int D, const PagesArgs &a, const PagesWs &ws, cudaStream_t stream, int num_sms) {
  if (kv.scales == nullptr)
    return D == 128 ? launch<128, 16>(kv, a, ws, stream, num_sms) : launch<64, 16>(kv, a, ws, stream, num_sms);
  return D == 128 ? launch<128, 8>(kv, a, ws, stream, num_sms) : launch<64, 8>(kv, a, ws, stream, num_sms);
}

}  // namespace umim
