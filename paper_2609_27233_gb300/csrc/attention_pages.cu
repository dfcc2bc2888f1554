// Decode attention over the 8-bit cache, and of groups of sequences that share
// a prefix (16- or 8-bit cache).
//
//   out[b][h] = sum_j softmax_j(scale <q[b][h], K_j>) V_j,
//   j over the entries of b's prefix and then b's own.
//
// The split is attention.cu's: (segment, page) pairs of the whole batch,
// flattened, an equal contiguous range for every warp of a persistent grid, one
// partial result (m, l, acc) a piece of a range that lies in one segment (without
// prefixes, the last ones of a CTA's warps are joined where they are of one segment),
// merged by a small kernel.  A segment is a list of pages with up to 16 query rows that
// attend to all of it: the query heads of one KV head over a sequence's own
// entries, or 16 of the rows (sequence, query head) of a group over the group's
// prefix, so that a page of a prefix is read once for 16 rows.
//
// 8-bit pages.  K = 2^e k, V = 2^f v with e4m3 rows k, v:
//   s_j = scale 2^e_j <q, k_j>,   out = sum_j (p_j 2^f_j) v_j / sum_j p_j,   p_j = exp(s_j - m).
// k and v turn into fp16 exactly, two values an instruction, and the products run as
// mma.sync m16n8k16 on fp16 with fp32 sums.  q is split into a power of two a row
// and fp16 numbers below 2^15 (exact for all but elements below 2^-29 of the row's
// largest, which lose at most 2^-40 of it).  The weights p_j 2^f_j are held relative to
// their own largest: with t_j = s_j + f_j (log2) and n = max t_j, w_j = 2^(t_j - n + 15)
// is at most 2^15 and is taken as two fp16 numbers, high part and remainder
// (22 significant bits down to 2^-18 of the largest weight, 2^-40 of it below).
// n leaves out the rows of V that hold nothing but zeros, whatever scale they are stored with:
// beside values of 2^-30 a single one, stored with 1, would be the unit of all weights.
// Up to eight query heads the two parts are rows 0-7 and 8-15 of one product.
//
// A lane's operands come as 16-byte pieces of rows: the head dimension that
// a product sums over may run in any order, and so may the columns of the output
// (q is read and the output written in that order).  For K a lane reads 16
// values of one key; for V 16 values of four keys, whose bytes are paired key by
// key before they are converted.  A page of 16 entries is 4 KB (D = 128): one TMA
// copy (K and V, rows swizzled so that eight lanes' pieces meet no bank twice) and
// one of its 32 scales.
//
// What bounds the 8-bit decode is what a page goes through in its warp, products, softmax and products one
// after the other, with three warps a scheduler to cover that: DRAM and issue slots are half used.
// 76800 entries of 64 sequences, 32/8 heads, D = 128 (158 MB) take 34.1 us on the device, 27 of them the
// stream of pages (5.8 TB/s) and the rest what a call of one short sequence takes too: lengths, table and
// first page one after the other, and the combine kernel; with 16 query heads a KV head 51.0.  A page costs a warp some 430
// instructions, 120 of them products, conversions and loads.
#include <cuda_fp16.h>

#include "attention_pages.cuh"
#include "kv8.cuh"
#include "mma.cuh"
#include "tmem.cuh"

namespace umim {
namespace {

// what a warp holds of a page: its layout in shared memory
template <int D, int BITS>
struct PageTile {
  static constexpr int kTile = 16 * D * BITS / 8;                // bytes of K, and of V
  static constexpr int kRow = D * BITS / 8 < 128 ? D * BITS / 8 : 128;   // bytes of a row in one box
  static constexpr int kBoxes = D * BITS / 8 / kRow;             // boxes of [K, V][16 rows][kRow]
  static constexpr int kStage = 2 * kTile;
  static constexpr int kStages = kStage >= 8192 ? 2 : 4;
  static constexpr int kScales = BITS == 8 ? 128 : 0;            // bytes of a stage's scales (32 used; TMA wants 128-byte steps)
  static constexpr int kWarp = kStages * kStage;
  static constexpr int kRings = kAttnWarps * kStages * (kStage + kScales);
  // byte offset of 16-byte piece c of row r (of K; V kRow * 16 further) as TMA's
  // swizzle for rows of 128 or 64 bytes puts it
  static __device__ __forceinline__ uint32_t at(int r, int c) {
    if constexpr (kRow == 128)
      return (c >> 3) * (2 * 16 * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
    else
      return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
  }
};

__device__ __forceinline__ uint4 lds_v4(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds_v2(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds_u32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=h"(v) : "r"(a));
  return v;
}

template <int BITS>
__device__ __forceinline__ void mma_page(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (BITS == 8) mma_f16(c, a, b0, b1);
  else mma_bf16(c, a, b0, b1);
}

// One segment as the warp that works on it sees it.
struct Segment {
  int i, g, blk;        // sequence or prefix, KV head, block of rows
  bool prefix;
  int n, len;           // pages, entries
  const int32_t *table;
};

// R8 (8-bit cache, no prefixes): at most eight query rows, the weights' two parts in one product
template <int D, int BITS, bool SHARED, bool R8>
__global__ void __launch_bounds__(kAttnWarps * 32, 1)
    attn_pages_kernel(const __grid_constant__ CUtensorMap kv_map, const __grid_constant__ CUtensorMap scale_map,
                      PagesArgs a, PagesWs ws) {
  using P = PageTile<D, BITS>;
  static_assert(!R8 || BITS == 8, "");
  constexpr int NT = D / 8;                // n-tiles of the output
  constexpr int KC = D / 16;               // k-chunks of Q K^T
  constexpr int NR = R8 ? 1 : 2;           // query rows of a lane
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ uint64_t bars[kAttnWarps][P::kStages];

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int gw = blockIdx.x * kAttnWarps + warp;
  __shared__ int s_tc;
  __shared__ int s_last[kAttnWarps];   // the segment of a warp's last piece, -1 for none
  uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t *wbuf = base + warp * P::kWarp;
  uint8_t *wscales = base + kAttnWarps * P::kWarp + warp * P::kStages * P::kScales;

  if (lane == 0) {
    for (int s = 0; s < P::kStages; ++s) mbar_init(&bars[warp][s], 1);
    fence_mbar_init();
    if (warp == 0) {
      prefetch_tensormap(&kv_map);
      if (BITS == 8) prefetch_tensormap(&scale_map);
    }
  }
  __syncwarp();
  griddep_wait();
  // The tensor cores' kernel, if that follows, is placed as this one's CTAs leave; it reads nothing of this one's.
  // (The combine kernel placed that early cost a call of 34 us four.)
  if (SHARED && a.most_rows != INT32_MAX) griddep_launch();

  const int G = a.G, Hkv = a.Hkv;
  const int32_t *pref = ws.at.pref;
  PrefixPlan pre = ws.pre;
  int own;   // pages of the sequences' own entries, of one KV head
  int32_t *plan = reinterpret_cast<int32_t *>(base + P::kRings);
  if (SHARED) {
    pre = plan_at(plan, a.n_prefixes);
    plan += 3 * (a.n_prefixes + 1);
    if (warp == 0) {
      const int tc = plan_prefixes(a, pre, blockIdx.x == 0, [&](int b, int len) { return pages_work(a, b, len); },
                                   [&](int b, int len) { return tc_work(a, b, len); });
      if (lane == 0) s_tc = tc;
    }
  }
  if (SHARED || a.smem_plan) {
    own = plan_prefix<kAttnWarps * 32>(a.seq_lens, a.B, a.max_pages, plan, blockIdx.x == 0, a.status);
    pref = plan;
    if (blockIdx.x == 0) {   // for the combine kernel
      for (int b = threadIdx.x; b <= a.B; b += kAttnWarps * 32) ws.at.pref[b] = plan[b];
      if (SHARED)
        for (int i = threadIdx.x; i <= a.n_prefixes; i += kAttnWarps * 32) {
          ws.pre.pages[i] = pre.pages[i];
          ws.pre.blocks[i] = pre.blocks[i];
          ws.pre.first[i] = pre.first[i];
        }
    }
  } else {
    own = pref[a.B];
  }
  const int total = Hkv * (own + (SHARED ? pre.pages[a.n_prefixes] : 0));
  // (s_tc: the barriers of plan_prefix have passed)
  const int ctas = SHARED ? pages_ctas((int)gridDim.x, total, (int64_t)Hkv * s_tc, BITS == 8) : (int)gridDim.x;
  if (SHARED && (int)blockIdx.x >= ctas) return;
  const int total_warps = ctas * kAttnWarps;
  const int W = max(1, ceil_div(total, total_warps));
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    ws.at.plan->W = W;
    ws.at.plan->total = total;
  }
  const int start = (int)min((int64_t)gw * W, (int64_t)total);
  const int end = min(total, start + W);
  bool whole = start < end;   // this warp has a last piece to hand in
  if (SHARED && !whole) return;   // (without prefixes there are barriers to come)

  const uint64_t pol = policy_evict_first();

  auto set_own = [&](Segment &s) {
    s.n = pref[s.i + 1] - pref[s.i];
    s.len = a.seq_lens[s.i];
    s.table = a.block_table + (int64_t)s.i * a.max_pages;
  };
  auto blocks_of = [&](int i) { return pre.blocks[i + 1] - pre.blocks[i]; };
  auto set_prefix = [&](Segment &s) {
    s.len = a.prefix_lens[s.i];
    s.n = ceil_div(s.len, kPageSize);
    s.table = a.prefix_table + (int64_t)s.i * a.max_prefix_pages;
  };
  // the segment of a flattened position, and the page in it
  auto locate = [&](int pos, Segment &s, int &pi) {
    s.blk = 0;
    s.prefix = SHARED && pos >= Hkv * own;
    if (!s.prefix) {   // (sequences without pages share their successor's first)
      s.i = last_at_most(pref, a.B, Hkv, pos);
      set_own(s);
      const int r = pos - Hkv * pref[s.i];
      s.g = r / s.n;
      pi = r - s.g * s.n;
    } else {
      pos -= Hkv * own;
      s.i = last_at_most(pre.pages, a.n_prefixes, Hkv, pos);
      set_prefix(s);
      const int r = pos - Hkv * pre.pages[s.i], x = r / s.n, nb = blocks_of(s.i);
      s.g = x / nb;
      s.blk = x - s.g * nb;
      pi = r - x * s.n;
    }
  };
  // the segment behind s, which there is
  auto advance = [&](Segment &s) {
    if (SHARED && s.prefix) {
      if (++s.blk < blocks_of(s.i)) return;
      s.blk = 0;
      if (++s.g < Hkv) return;
      s.g = 0;
      do ++s.i;
      while (pre.pages[s.i + 1] == pre.pages[s.i]);
      set_prefix(s);
    } else {
      if (++s.g < Hkv) return;
      s.g = 0;
      do ++s.i;
      while (s.i < a.B && pref[s.i + 1] == pref[s.i]);
      if (SHARED && s.i == a.B) {
        s.prefix = true;
        s.i = 0;
        while (pre.pages[s.i + 1] == pre.pages[s.i]) ++s.i;
        set_prefix(s);
      } else {
        set_own(s);
      }
    }
  };
  // its number: in the flattened order, so that number + warp is a piece of its own
  auto number = [&](const Segment &s) {
    if (SHARED && s.prefix) return Hkv * (a.B + pre.blocks[s.i]) + s.g * blocks_of(s.i) + s.blk;
    return s.i * Hkv + s.g;
  };
  // query row r of 16 as a row of q, -1 for none
  auto query_row = [&](const Segment &s, int r) {
    if (SHARED && s.prefix) {
      const int x = s.blk * 16 + r, b = pre.first[s.i] + x / G;
      return b < pre.first[s.i + 1] ? (int64_t)b * a.Hq + s.g * G + x % G : int64_t(-1);
    }
    return r < G ? (int64_t)s.i * a.Hq + s.g * G + r : int64_t(-1);
  };

  // ---- compute cursor and loader cursor (every lane keeps both; one issues the copies) ----
  Segment cs, ls;
  int cpi, lpi;
  int ld_pos = start;
  if (SHARED || whole) locate(start, cs, cpi);
  ls = cs;
  lpi = cpi;
  auto page_of = [&]() {
    const int cols = SHARED && ls.prefix ? a.max_prefix_pages : a.max_pages;
    return in_bounds(lpi, cols, a.status, kSitePagesTable) ? ls.table[lpi] : -1;
  };
  // looked up a copy ahead: the copy does not wait for the table
  int next_page = SHARED || whole ? page_of() : -1;
  auto issue = [&](int stage) {
    int c = a.layer * a.n_pages + next_page;
    if (next_page < 0 || next_page >= a.n_pages) {
      // a coordinate past the tensor's last page: the copy reads zeros
      set_error(a.status, UMIM_ERR_INVALID_ARG);
      c = a.n_layers * a.n_pages;
    }
    if (elect_one()) {
      uint64_t *bar = &bars[warp][stage];
      uint8_t *dst = wbuf + stage * P::kStage;
      mbar_arrive_expect_tx(bar, P::kStage + (BITS == 8 ? 32 : 0));
#pragma unroll
      for (int x = 0; x < P::kBoxes; ++x)
        tma_load_5d(dst + x * 32 * P::kRow, &kv_map, bar, x * (P::kRow * 8 / BITS), 0, ls.g, 0, c, pol);
      if constexpr (BITS == 8) tma_load_4d(wscales + stage * P::kScales, &scale_map, bar, 0, ls.g, 0, c);
    }
    if (++ld_pos < end) {
      if (++lpi == ls.n) {
        lpi = 0;
        advance(ls);
      }
      next_page = page_of();
    }
  };
  for (int s = 0; s < P::kStages && ld_pos < end; ++s) issue(s);

  // ---- compute state ----
  const int qr = lane >> 2, qc = lane & 3;      // mma fragment row / column group
  int64_t rows[NR];                             // rows of q
  uint32_t qa[KC][2 * NR];
  float q_scale[NR];                            // scale_log2, times the power of two taken out of the row
  auto load_q = [&]() {
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      rows[j] = query_row(cs, qr + 8 * j);
      const __nv_bfloat16 *src = a.q + rows[j] * D;
      q_scale[j] = a.scale_log2;
      if constexpr (BITS == 16) {
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const uint32_t *p = reinterpret_cast<const uint32_t *>(src + c * 16 + 2 * qc);
          qa[c][j] = rows[j] >= 0 ? p[0] : 0u;
          qa[c][j + NR] = rows[j] >= 0 ? p[4] : 0u;
        }
      } else {
        // chunk c of the products: 4 elements of this lane's 16-byte pieces of K
        uint2 x[KC];
        uint32_t m = 0;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const int piece = D == 128 ? qc * 2 + c / 4 : qc;
          x[c] = make_uint2(0, 0);
          if (rows[j] >= 0) x[c] = *reinterpret_cast<const uint2 *>(src + piece * 16 + c % 4 * 4);
          m = __vmaxu2(m, __vmaxu2(x[c].x & 0x7fff7fff, x[c].y & 0x7fff7fff));
        }
        m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 2));
        m = max(m & 0xffff, m >> 16) >> 7;   // the exponent field of the row's largest
        // the largest to [2^14, 2^15); rows of zeros (or below 2^-86) and ones that hold no number by a fixed power
        const uint32_t e = m == 255 ? 127u : max(m, 41u);
        const float inv = __uint_as_float((268u - e) << 23);   // 2^(14 - (e - 127))
        q_scale[j] *= __uint_as_float((e - 14) << 23);
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          auto half2_of = [&](uint32_t v) {
            const __half2 h = __floats2half2_rn(__uint_as_float(v << 16) * inv, __uint_as_float(v & 0xffff0000u) * inv);
            return *reinterpret_cast<const uint32_t *>(&h);
          };
          qa[c][j] = half2_of(x[c].x);
          qa[c][j + NR] = half2_of(x[c].y);
        }
      }
    }
  };
  if (SHARED || whole) load_q();
  float acc[NT][4];
  // a row's largest score and weight (log2), and sum of exp2(score - m)
  float m[NR], n[NR], l[NR];
  auto reset = [&]() {
#pragma unroll
    for (int j = 0; j < NR; ++j) m[j] = n[j] = -INFINITY, l[j] = 0.f;
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
  };
  reset();

  // the segment's rows to [16] (m, l) and [16] rows of D columns, `stride` apart
  auto hand_in = [&](float2 *ml, float *columns, int stride) {
    // complete the row sums across the 4 threads of each row
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      l[j] += __shfl_xor_sync(0xffffffffu, l[j], 1);
      l[j] += __shfl_xor_sync(0xffffffffu, l[j], 2);
    }
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      if (rows[j] < 0) continue;
      if (qc == 0) ml[qr + 8 * j] = make_float2(m[j], l[j]);
      float *dst = columns + (qr + 8 * j) * stride;
      if constexpr (BITS == 16) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
          *reinterpret_cast<float2 *>(dst + t * 8 + 2 * qc) = make_float2(acc[t][2 * j], acc[t][2 * j + 1]);
      } else {
        // from units of 2^(n - 15) to those of the row sum (n - m is a cache row's exponent at most)
        const float up = n[j] == -INFINITY ? 1.f : exp2f(n[j] - m[j]);   // (no value so far: acc is 0, or NaN)
        auto out = [&](int t, int c) {
          const float x = R8 ? acc[t][c] + acc[t][2 + c] : acc[t][2 * j + c];
          return x * 0x1p-15f * up;
        };
#pragma unroll
        for (int c = 0; c < 2; ++c)   // column t of piece 2 qc + c
#pragma unroll
          for (int t = 0; t < NT; t += 4)
            *reinterpret_cast<float4 *>(dst + (2 * qc + c) * NT + t) =
                make_float4(out(t, c), out(t + 1, c), out(t + 2, c), out(t + 3, c));
      }
    }
  };
  // a piece's place in the workspace, -1 for none (debug build)
  auto place = [&](int64_t piece) {
    const int64_t n = (int64_t)Hkv * (a.B + (SHARED ? pre.blocks[a.n_prefixes] : 0)) + total_warps;
    return in_bounds(piece, n, a.status, kSitePagesPiece) ? piece : int64_t(-1);
  };
  auto flush = [&]() {
    const int64_t at = place((int64_t)number(cs) + gw);
    if (at >= 0) hand_in(ws.at.part_ml + at * 16, ws.at.part_acc + at * 16 * D, D);
  };

  int it = 0;
  for (int pos = start; pos < end; ++pos, ++it) {
    if (cpi == cs.n) {   // next segment
      flush();
      cpi = 0;
      advance(cs);
      load_q();
      reset();
    }
    const int stage = it % P::kStages;
    const uint32_t parity = (it / P::kStages) & 1;
    if (!mbar_wait(&bars[warp][stage], parity)) {
      set_error(a.status, UMIM_ERR_TIMEOUT);
      // let the copies still in flight land (each wait bounded) before leaving
      for (int k = 1; k < P::kStages && pos + k < ld_pos; ++k)
        mbar_wait(&bars[warp][(it + k) % P::kStages], ((it + k) / P::kStages) & 1);
      if (SHARED) return;
      whole = false;
      break;
    }
    const uint32_t ks = smem_u32(wbuf + stage * P::kStage), vs = ks + 16 * P::kRow;
    const uint32_t sc = smem_u32(wscales + stage * P::kScales);
    const int nvalid = min(16, cs.len - cpi * 16);
    ++cpi;

    // S = Q K^T, 16 keys as two n-tiles of 8; even and odd chunks apart, to halve the dependent chain
    float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    float s2[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    auto q_of = [&](int c, uint32_t (&f)[4]) {
      f[0] = qa[c][0], f[2] = qa[c][NR];
      f[1] = R8 ? 0u : qa[c][NR - 1], f[3] = R8 ? 0u : qa[c][2 * NR - 1];
    };
    if constexpr (BITS == 16) {
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        uint32_t b0, b1, b2, b3, f[4];
        q_of(c, f);
        ldsm_x4(ks + P::at((lane & 7) + ((lane >> 4) << 3), 2 * c + ((lane >> 3) & 1)), b0, b1, b2, b3);
        mma_bf16(c & 1 ? s2[0] : s[0], f, b0, b1);
        mma_bf16(c & 1 ? s2[1] : s[1], f, b2, b3);
      }
    } else {
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int t = 0; t < D / 64; ++t) {
          const uint4 x = lds_v4(ks + P::at(nt * 8 + qr, D == 128 ? qc * 2 + t : qc));
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t f[4];
            q_of(t * 4 + w, f);
            mma_f16(w & 1 ? s2[nt] : s[nt], f, f16x2_of_e4m3x2(xs[w]), f16x2_of_e4m3x2(xs[w] >> 16));
          }
        }
    }
    // to log2 units; keys past the end masked.  This lane's keys are nt * 8 + 2 qc + {0, 1}.
    float w[2][4];   // weights' exponents (8-bit), then the weights
    float own = 0.f;   // 8-bit: a lane turns one of the 32 scales into 2^e (lanes 0-15, K's) or e (V's)
    if constexpr (BITS == 8) {
      const uint32_t code = lds_u8(sc + lane);
      own = lane < 16 ? e8m0_value(code) : code == 255 ? NAN : (float)((int)code - 127);
    }
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      float ke[2] = {1.f, 1.f}, ve[2] = {0.f, 0.f};
      if constexpr (BITS == 8) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          ke[e] = __shfl_sync(0xffffffffu, own, nt * 8 + 2 * qc + e);
          ve[e] = __shfl_sync(0xffffffffu, own, 16 + nt * 8 + 2 * qc + e);
        }
      }
#pragma unroll
      for (int e = 0; e < 2 * NR; ++e) {
        s[nt][e] = (s[nt][e] + s2[nt][e]) * q_scale[e >> 1] * ke[e & 1];
        w[nt][e] = s[nt][e] + ve[e & 1];
      }
    }
    if (nvalid < 16) {
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 2 * NR; ++e)
          if (nt * 8 + 2 * qc + (e & 1) >= nvalid) s[nt][e] = w[nt][e] = -INFINITY;
    }
    auto row_max = [&](const float (&x)[2][4], int j) {
      float y = fmaxf(fmaxf(x[0][2 * j], x[0][2 * j + 1]), fmaxf(x[1][2 * j], x[1][2 * j + 1]));
      y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 1));
      return fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 2));
    };
    float top[NR];   // the page's largest weights
    if constexpr (BITS == 8) {
      // Rows of zeros are looked for by two lanes a row: 4 bytes each, and all of the row where that leaves a doubt.
      // (64 sequences of 1200 entries, three batches in turn: 37.8 -> 38.6 us.  Only where a largest weight would
      // move, but whole rows: 39.4.)
      auto rows_of = [&](uint32_t x) {   // bit 2 r: row r holds something
        const uint32_t held = __ballot_sync(0xffffffffu, (x & 0x7f7f7f7f) != 0);
        return (held | held >> 1) & 0x55555555;
      };
      uint32_t held = rows_of(lds_u32(vs + P::at(lane >> 1, lane & 1)));
      if (held != 0x55555555) {
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const uint4 x = lds_v4(vs + P::at(lane >> 1, (lane & 1) * (D / 32) + i));
          any |= x.x | x.y | x.z | x.w;
        }
        held = rows_of(any);
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
          for (int e = 0; e < 2 * NR; ++e)   // (NaN, of a scale, stays)
            if (!(held >> 2 * (nt * 8 + 2 * qc + (e & 1)) & 1)) w[nt][e] -= INFINITY;
      }
#pragma unroll
      for (int j = 0; j < NR; ++j) top[j] = row_max(w, j);
    }
    bool moved = false;
    float c[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      const float m_was = m[j], n_was = n[j];
      m[j] = fmaxf(m[j], row_max(s, j));
      n[j] = BITS == 8 ? fmaxf(n[j], top[j]) : m[j];
      // no finite score so far: weights from 0, so that a score of -inf weighs 0 and NaN stays NaN
      const float m0 = m[j] == -INFINITY ? 0.f : m[j], n0 = n[j] == -INFINITY ? 0.f : n[j];
      c[j] = ex2_approx(n_was - n0);
      moved = moved || c[j] != 1.f;
      float sum = 0.f;
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 2 * j; e < 2 * j + 2; ++e) {
          const float p = ex2_approx(s[nt][e] - m0);
          sum += p;
          w[nt][e] = BITS == 8 ? ex2_approx(w[nt][e] - n0 + 15.f) : p;
        }
      l[j] = l[j] * ex2_approx(m_was - m0) + sum;
    }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        acc[t][0] *= c[0];
        acc[t][1] *= c[0];
        acc[t][2] *= c[NR - 1];
        acc[t][3] *= c[NR - 1];
      }
    }
    // the weights as the A operand: a high part and what it leaves
    uint32_t ph[4], pl[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {   // rows qr, qr + 8 of keys 0-7, then of keys 8-15
      if (R8 && (r & 1)) continue;
      const float x = w[r >> 1][2 * (r & 1)], y = w[r >> 1][2 * (r & 1) + 1];
      if constexpr (BITS == 8) {
        const __half2 h = __floats2half2_rn(x, y);
        const __half2 rest = __floats2half2_rn(x - __low2float(h), y - __high2float(h));
        ph[r] = *reinterpret_cast<const uint32_t *>(&h);
        pl[r] = *reinterpret_cast<const uint32_t *>(&rest);
      } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        ph[r] = *reinterpret_cast<const uint32_t *>(&h);
        pl[r] = pack_bf16(x - __low2float(h), y - __high2float(h));
      }
    }
    if constexpr (R8) ph[1] = pl[0], ph[3] = pl[2];
    // O += P V
    if constexpr (BITS == 16) {
      if (nvalid < 16) {
        // zero V rows past the end so that 0 * garbage cannot make a NaN
        for (int idx = lane; idx < (16 - nvalid) * (D / 8); idx += 32) {
          const uint32_t at = vs + P::at(nvalid + idx / (D / 8), idx % (D / 8));
          asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
        }
        // order these generic-proxy writes before the next TMA write of the stage
        fence_proxy_async_smem();
        __syncwarp();
      }
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        uint32_t b0, b1, b2, b3;
        ldsm_x4_t(vs + P::at((lane & 7) + (((lane >> 3) & 1) << 3), 2 * j + (lane >> 4)), b0, b1, b2, b3);
        mma_bf16(acc[2 * j], ph, b0, b1);
        mma_bf16(acc[2 * j + 1], ph, b2, b3);
        mma_bf16(acc[2 * j], pl, b0, b1);
        mma_bf16(acc[2 * j + 1], pl, b2, b3);
      }
    } else {
      // column t of n-tile t is value t of this lane's piece qr (D / 8 values) of a row
      uint32_t v[4][NT / 4];   // keys 2 qc, 2 qc + 1, 2 qc + 8, 2 qc + 9
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int key = 2 * qc + (k & 1) + (k >> 1) * 8;
        if constexpr (D == 128) {
          const uint4 x = lds_v4(vs + P::at(key, qr));
          v[k][0] = x.x, v[k][1] = x.y, v[k][2] = x.z, v[k][3] = x.w;
        } else {
          const uint2 x = lds_v2(vs + P::at(key, qr >> 1) + (qr & 1) * 8);
          v[k][0] = x.x, v[k][1] = x.y;
        }
        if (nvalid < 16 && key >= nvalid) {   // 0 * garbage must not make a NaN
#pragma unroll
          for (int i = 0; i < NT / 4; ++i) v[k][i] = 0;
        }
      }
#pragma unroll
      for (int i = 0; i < NT / 4; ++i) {
        const uint32_t a01 = __byte_perm(v[0][i], v[1][i], 0x5140), a23 = __byte_perm(v[0][i], v[1][i], 0x7362);
        const uint32_t b01 = __byte_perm(v[2][i], v[3][i], 0x5140), b23 = __byte_perm(v[2][i], v[3][i], 0x7362);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t lo = (x < 2 ? a01 : a23) >> (x & 1) * 16, hi = (x < 2 ? b01 : b23) >> (x & 1) * 16;
          const uint32_t f0 = f16x2_of_e4m3x2(lo), f1 = f16x2_of_e4m3x2(hi);
          mma_f16(acc[i * 4 + x], ph, f0, f1);
          if constexpr (!R8) mma_f16(acc[i * 4 + x], pl, f0, f1);
        }
      }
    }
    __syncwarp();
    // refill this stage
    if (ld_pos < end) issue(stage);
  }

  // (With prefixes the same took 3 to 8 % longer: 16 rows a piece to join, in place of 4 or 7.)
  if constexpr (SHARED) {
    flush();
    return;
  }
  // The warps' last pieces: those of one segment meet in shared memory, where the rings were, and become one
  // piece of the first of its warps: with four sequences of 32768 entries a row had 114 pieces, one a
  // warp, and a call took 33.0 us in place of 29.4.
  constexpr int kStride = D + 4;   // of a row there: eight rows of a store meet no bank twice
  static_assert(16 * kStride * 4 + 128 <= P::kWarp, "a piece where a warp's ring was");
  if (lane == 0) s_last[warp] = whole ? number(cs) : -1;
  __syncthreads();
  const int last = lane < kAttnWarps ? s_last[lane] : -1;
  const int before = __shfl_up_sync(0xffffffffu, last, 1), behind = __shfl_down_sync(0xffffffffu, last, 1);
  const bool first_of = last >= 0 && (lane == 0 || before != last);
  const bool alone = first_of && (lane == kAttnWarps - 1 || behind != last);
  const uint32_t firsts = __ballot_sync(0xffffffffu, first_of), alones = __ballot_sync(0xffffffffu, alone);
  if (whole) {
    if (alones >> warp & 1) flush();
    else hand_in(reinterpret_cast<float2 *>(wbuf + 16 * kStride * 4), reinterpret_cast<float *>(wbuf), kStride);
  }
  __syncthreads();
  for (uint32_t runs = firsts & ~alones; runs; runs &= runs - 1) {
    constexpr int E = D / 32;
    const int w0 = __ffs(runs) - 1, seg = __shfl_sync(0xffffffffu, last, w0);
    const int n = __popc(__ballot_sync(0xffffffffu, last == seg && lane >= w0));
    for (int row = warp; row < G; row += kAttnWarps) {
      float2 ml = make_float2(-INFINITY, 0.f);
      if (lane < n) ml = reinterpret_cast<const float2 *>(base + (w0 + lane) * P::kWarp + 16 * kStride * 4)[row];
      float M = ml.x;
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
      M = __shfl_sync(0xffffffffu, M, 0);
      const float c = exp2f(ml.x - (M == -INFINITY ? 0.f : M));   // (no finite score: weighted, not skipped)
      float L = ml.y * c, o[E];
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) L += __shfl_xor_sync(0xffffffffu, L, d);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 4
      for (int w = 0; w < n; ++w) {
        const float cw = __shfl_sync(0xffffffffu, c, w);
        const float *src = reinterpret_cast<const float *>(base + (w0 + w) * P::kWarp) + row * kStride + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(src[e], cw, o[e]);
      }
      const int64_t at = place((int64_t)seg + blockIdx.x * kAttnWarps + w0);
      if (at < 0) continue;
      if (lane == 0) ws.at.part_ml[at * 16 + row] = make_float2(M, L);
      float *dst = ws.at.part_acc + (at * 16 + row) * D + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) dst[e] = o[e];
    }
  }
}

// ---------------------------------------------------------------------------
// combine: WPR warps per (b, query head) row, over the pieces of its own entries'
// segment and then of its prefix's block
// ---------------------------------------------------------------------------
template <int D, bool SHARED, int WPR>
__global__ void __launch_bounds__(kCombineThreads)
    pages_combine_kernel(PagesWs ws, bool tc, int B, int n_prefixes, int Hq, int Hkv, int G, __nv_bfloat16 *out) {
  constexpr int E = D / 32;
  constexpr int kWarps = kCombineThreads / 32, RPB = kWarps / WPR;   // rows per CTA
  __shared__ float s_m[kWarps], s_l[kWarps];
  __shared__ float s_acc[WPR > 1 ? kWarps : 1][D];
  griddep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row_g = blockIdx.x * RPB + warp / WPR, sub = warp % WPR;
  const bool live = row_g < B * Hq;
  float M = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  bool any = false;
  if (live) {
    const int b = row_g / Hq, h = row_g % Hq, g = h / G, W = ws.at.plan->W, total = ws.at.plan->total;
    // Pieces of the segment that takes n positions from `at` on: seg + w for the warps w that meet them.
    // Without prefixes they are joined: the first of those warps has one, the first of every further CTA,
    // and the last warp where the segment ends inside its range (handed in by itself).
    auto merge = [&](int seg, int at, int n, int row) {
      if (n <= 0) return;
      any = true;
      const int w0 = at / W, w1 = (at + n - 1) / W, c0 = w0 / kAttnWarps, c1 = w1 / kAttnWarps;
      const bool inside = w1 > w0 && w1 % kAttnWarps != 0 && at + n < min((w1 + 1) * (int64_t)W, (int64_t)total);
      auto row_of = [&](int k) {
        const int w = SHARED || k == 0 ? w0 + k : k <= c1 - c0 ? (c0 + k) * kAttnWarps : w1;
        return (int64_t)(seg + w) * 16 + row;
      };
      merge_pieces<E>(
          SHARED ? w1 - w0 + 1 : 1 + c1 - c0 + (inside ? 1 : 0), sub, WPR, M, l, o,
          [&](int k) { return ws.at.part_ml + row_of(k); },
          [&](int k) { return ws.at.part_acc + row_of(k) * D + lane * E; });
    };
    const int first = ws.at.pref[b], n = ws.at.pref[b + 1] - first;
    merge(b * Hkv + g, Hkv * first + g * n, n, h % G);
    const int i = SHARED ? last_at_most(ws.pre.first, n_prefixes, 1, b) : 0;
    if (SHARED && b >= ws.pre.first[i] && b < ws.pre.first[i + 1]) {
      const int nb = ws.pre.blocks[i + 1] - ws.pre.blocks[i], bi = b - ws.pre.first[i];
      const int ns = tc ? ws.tc.blocks[i + 1] - ws.tc.blocks[i] : 0;
      if (nb > 0) {
        const int x = bi * G + h % G;
        const int np = (ws.pre.pages[i + 1] - ws.pre.pages[i]) / nb;
        merge(Hkv * (B + ws.pre.blocks[i]) + g * nb + x / 16,
              Hkv * (ws.at.pref[B] + ws.pre.pages[i]) + (g * nb + x / 16) * np, np, x % 16);
      } else if (ns > 0) {
        // two pieces a CTA: of the pair's row tiles, or of one tile's even and odd key tiles
        const int spt = tile_sequences(G), tiles = ceil_div(ws.pre.first[i + 1] - ws.pre.first[i], spt);
        const int work = ws.tc.pages[i + 1] - ws.tc.pages[i], keys = work / tiles;
        const int s = bi / spt / 2, row = bi % spt * G + h % G, width = 2 * s + 1 < tiles ? 2 : 1;
        const int at = Hkv * ws.tc.pages[i] + g * work + s * 2 * keys, W = *ws.tc_W;
        const int c0 = at / W, c1 = (at + (keys - 1) * width) / W;
        const int64_t piece = 2 * (int64_t)(Hkv * ws.tc.blocks[i] + g * ns + s + c0);
        any = true;
        const int64_t from = piece + (width == 2 ? bi / spt % 2 : 0);
        merge_pieces<E>((c1 - c0 + 1) * (3 - width), sub, WPR, M, l, o,
                        [&](int x) { return ws.tc_ml + (from + x * width) * kTcRows + row; },
                        [&](int x) { return ws.tc_acc + tc_acc_at<D>(from + x * width, row, lane * E); });
      }
    }
  }
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
  const float inv = any ? 1.f / l : 0.f;   // (no entries: zeros)
  __nv_bfloat16 *dst = out + (int64_t)row_g * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = __float2bfloat16_rn(o[e] * inv);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
template <int D, int BITS>
bool encode_maps(const CacheView &kv, CUtensorMap *values, CUtensorMap *scales) {
  using P = PageTile<D, BITS>;
  EncodeTiledFn enc = get_encode_tiled();
  if (!enc) return false;
  const cuuint64_t H = kv.n_kv_heads, N = (cuuint64_t)kv.n_layers * (cuuint64_t)kv.n_pages, row = D * BITS / 8;
  const cuuint64_t dims[5] = {(cuuint64_t)D, 16, H, 2, N};
  const cuuint64_t strides[4] = {row, 16 * row, H * 16 * row, 2 * H * 16 * row};
  const cuuint32_t box[5] = {(cuuint32_t)(P::kRow * 8 / BITS), 16, 1, 2, 1};
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  if (enc(values, BITS == 8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, kv.values, dims,
          strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
          P::kRow == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return false;
  *scales = *values;
  if (BITS == 16) return true;
  const cuuint64_t sdims[4] = {16, H, 2, N}, sstrides[3] = {16, 16 * H, 32 * H};
  const cuuint32_t sbox[4] = {16, 1, 2, 1};
  return enc(scales, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, kv.scales, sdims, sstrides, sbox, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int BITS, bool SHARED>
umim_status run_pages(const CacheView &kv, PagesArgs a, void *out, void *workspace, cudaStream_t stream, int num_sms) {
  using P = PageTile<D, BITS>;
  CUtensorMap map, scale_map;
  if (!encode_maps<D, BITS>(kv, &map, &scale_map)) return UMIM_ERR_CUDA;
  a.n_layers = kv.n_layers;
  a.n_pages = kv.n_pages;
  a.Hkv = kv.n_kv_heads;
  a.G = a.Hq / a.Hkv;
  const int total_warps = std::max(1, num_sms) * kAttnWarps;
  PagesWs ws;
  pages_carve(workspace, &ws, a.B, SHARED ? a.n_prefixes : 0, a.G, a.Hkv, D, num_sms);
  const bool tc = SHARED && tc_pays(a.B, a.n_prefixes, a.G, a.Hkv, D, BITS == 8, a.max_prefix_pages);
  a.most_rows = tc ? kTcMinRows : INT32_MAX;
  a.smem_plan = a.B <= kSmemPlanBatch ? 1 : 0;
  if (!a.smem_plan) {   // (never with prefixes: their batch is limited)
    trace_mark(stream, "attention.plan");
    if (launch_pdl(attn_plan_kernel, dim3(1), dim3(kPlanThreadsA), 0, stream, a.seq_lens, a.B, a.max_pages, ws.at,
                   a.status) != cudaSuccess)
      return UMIM_ERR_CUDA;
  }
  constexpr size_t kBase = P::kRings + 1024;
  const size_t plan = a.smem_plan ? sizeof(int32_t) * ((size_t)a.B + 1 + (SHARED ? 3 * ((size_t)a.n_prefixes + 1) : 0)) : 0;
  constexpr size_t kMost = kBase + sizeof(int32_t) * (kSmemPlanBatch + 1 + (SHARED ? 3 * (kSharedMaxPrefixes + 1) : 0));
  static_assert(kMost + 1024 <= 232448 && kSharedMaxBatch <= kSmemPlanBatch, "shared memory of a CTA");
  auto kern = attn_pages_kernel<D, BITS, SHARED, false>;
  if constexpr (BITS == 8 && !SHARED)
    if (a.G <= 8) kern = attn_pages_kernel<D, BITS, SHARED, true>;
  if (!allow_smem(kern, kMost)) return UMIM_ERR_CUDA;
  trace_mark(stream, SHARED ? "attention.shared" : "attention.decode_kv8");
  if (launch_pdl(kern, dim3((unsigned)(total_warps / kAttnWarps)), dim3(kAttnWarps * 32), kBase + plan, stream, map,
                 scale_map, a, ws) != cudaSuccess)
    return UMIM_ERR_CUDA;
  if (tc) {
    trace_mark(stream, "attention.prefix");
    if (!prefix_tc_launch(kv, D, a, ws, stream, num_sms)) return UMIM_ERR_CUDA;
  }
  trace_mark(stream, "attention.combine");
  __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(out);
  // About as many pieces as a row has: one or two a CTA that has some of its entries.  With prefixes half of them,
  // one a warp for two segments: 64 sequences behind 16384 entries take 46.1 us (47.8 with twice
  // the warps, 51.7 with four times), behind eight of 500 17.4 (20.0).
  const int n = SHARED ? a.n_prefixes : 0, segments = std::max(1, (n + a.B) * a.Hkv);
  const int wpr = combine_warps(SHARED ? 1 + total_warps / segments : 2 + 2 * (total_warps / kAttnWarps) / segments);
  const int rows = kCombineThreads / 32 / wpr;
  auto comb = wpr == 8 ? pages_combine_kernel<D, SHARED, 8>
              : wpr == 4 ? pages_combine_kernel<D, SHARED, 4>
              : wpr == 2 ? pages_combine_kernel<D, SHARED, 2> : pages_combine_kernel<D, SHARED, 1>;
  if (launch_pdl(comb, dim3((unsigned)((a.B * a.Hq + rows - 1) / rows)), dim3(kCombineThreads), 0, stream, ws, tc, a.B, n,
                 a.Hq, a.Hkv, a.G, o) != cudaSuccess)
    return UMIM_ERR_CUDA;
  trace_mark(stream, nullptr);
  return cudaGetLastError() == cudaSuccess ? UMIM_OK : UMIM_ERR_CUDA;
}

}  // namespace

size_t decode_attention_kv8_workspace_bytes(int B, int Hkv, int D, int num_sms) {
  return pages_carve(nullptr, nullptr, B, 0, 1, Hkv, D, num_sms);
}

size_t decode_attention_shared_workspace_bytes(int B, int n, int Hq, int Hkv, int D, int num_sms) {
  return pages_carve(nullptr, nullptr, B, std::max(1, n), Hq / Hkv, Hkv, D, num_sms);
}

umim_status decode_attention_kv8(const void *q, int Hq, const umim_paged_kv8 *kv, int layer, const int32_t *block_table,
                                 int max_pages, const int32_t *seq_lens, int B, float scale, void *out, void *workspace,
                                 int32_t *status, cudaStream_t stream, int num_sms) {
  PagesArgs a{};
  a.q = static_cast<const __nv_bfloat16 *>(q);
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.B = B;
  a.Hq = Hq;
  a.max_pages = max_pages;
  a.layer = layer;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.status = status;
  const CacheView c{kv->values, kv->scales, kv->n_layers, kv->n_pages, kv->n_kv_heads};
  return kv->head_dim == 128 ? run_pages<128, 8, false>(c, a, out, workspace, stream, num_sms)
                             : run_pages<64, 8, false>(c, a, out, workspace, stream, num_sms);
}

bool decode_attention_shared_supported(int B, int n) { return B <= kSharedMaxBatch && n <= kSharedMaxPrefixes; }

// scales null: a bf16 cache
umim_status decode_attention_shared(const void *q, int Hq, void *values, void *scales, int n_layers, int n_pages,
                                    int Hkv, int D, int layer, const int32_t *prefix_table, int max_prefix_pages,
                                    const int32_t *prefix_lens, const int32_t *prefix_offsets, int n_prefixes,
                                    const int32_t *block_table, int max_pages, const int32_t *seq_lens, int B,
                                    float scale, void *out, void *workspace, int32_t *status, cudaStream_t stream,
                                    int num_sms) {
  PagesArgs a{};
  a.q = static_cast<const __nv_bfloat16 *>(q);
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.prefix_table = prefix_table;
  a.prefix_lens = prefix_lens;
  a.prefix_offsets = prefix_offsets;
  a.n_prefixes = n_prefixes;
  a.max_prefix_pages = max_prefix_pages;
  a.B = B;
  a.Hq = Hq;
  a.max_pages = max_pages;
  a.layer = layer;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.status = status;
  const CacheView c{values, scales, n_layers, n_pages, Hkv};
  if (scales == nullptr)
    return D == 128 ? run_pages<128, 16, true>(c, a, out, workspace, stream, num_sms)
                    : run_pages<64, 16, true>(c, a, out, workspace, stream, num_sms);
  return D == 128 ? run_pages<128, 8, true>(c, a, out, workspace, stream, num_sms)
                  : run_pages<64, 8, true>(c, a, out, workspace, stream, num_sms);
}

}  // namespace umim
