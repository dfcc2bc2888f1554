// Rows of logits as the loss and log-probability kernels read them: 16-byte
// vectors of bf16, fp16 or fp32 elements, computed on in fp32.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace umim {

constexpr int kMaxLogitVocab = 262144;   // vocabulary size of the calls below, at most
constexpr int kMaxLogitRows = 1 << 30;   // rows and pairs, at most: a row's number and a stride more fit 32 bits
constexpr int kMaxTop = 128;             // alternatives per row, at most
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// The hardware's base-2 exponential (relative error about 2^-22; subnormal results flush to zero).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// An asynchronous copy of whole vectors into shared memory; its bytes count on bar.
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}

// Brings whole vectors, one at least, into L2 (16-byte aligned).
__device__ __forceinline__ void bulk_prefetch(const void *src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}

// An asynchronous store of 16 bytes into a CTA of the cluster; they count on its mbarrier.
__device__ __forceinline__ void st_async16(uint32_t to, float4 v, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to),
               "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(bar)
               : "memory");
}

// the maximum over the warp; NaN only where every lane holds one
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}

// sum over the warp by xor butterflies: every lane gets the same bits
__device__ __forceinline__ float2 warp_sum2(float2 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    v = __fadd2_rn(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
  return v;
}

__device__ __forceinline__ float2 half2_to_float2(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

// The three element types: VEC elements to a 16-byte vector, unpacked to and
// packed from fp32 (packing rounds to nearest even).  max_words takes the
// maximum of the elements of two 32-bit words place by place, word_max that of
// one word's; both pass a number over a NaN.  finite_words brings a 16-bit word's -inf up
// to a finite value so far below that it may stand for it (see its type), and
// keeps NaN.  order_key maps an element's bits
// to a number that grows with its value, both zeros to one.
__device__ __forceinline__ uint32_t order_key16(uint16_t b) {
  const uint32_t u = b == 0x8000u ? 0u : b;
  return u & 0x8000u ? 0xffffu - u : u + 0x8000u;
}
__device__ __forceinline__ uint16_t from_key16(uint32_t k) {
  return (uint16_t)(k & 0x8000u ? k - 0x8000u : 0xffffu - k);
}

struct ElemBf16 {
  using T = uint16_t;
  static constexpr int VEC = 8;
  static constexpr uint32_t kNegInf2 = 0xff80ff80u;
  static constexpr T kNegInf = 0xff80;
  static __device__ __forceinline__ uint32_t max_words(uint32_t x, uint32_t y) {
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(y));
    return d;
  }
  static __device__ __forceinline__ T word_max_bits(uint32_t w) { return (T)max_words(w, w >> 16); }
  // all ones in the place of each element of x that is >= y's, else zeros
  static __device__ __forceinline__ uint32_t reach_words(uint32_t x, uint32_t y) {
    return __hge2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
  }
  // -1e30: beside a maximum of any size that fp32 exponents of differences are taken of
  static constexpr bool kHasFinite = true;
  static __device__ __forceinline__ uint32_t finite_words(uint32_t x) {
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(0xf149f149u));
    return d;
  }
  static __device__ __forceinline__ uint32_t order_key(T b) { return order_key16(b); }
  static __device__ __forceinline__ T from_key(uint32_t k) { return from_key16(k); }
  static __device__ __forceinline__ float2 pair(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&p);
  }
  static __device__ __forceinline__ float to_float(T x) { return __uint_as_float((uint32_t)x << 16); }
  static __device__ __forceinline__ T from_float(float x) {
    __nv_bfloat16 h = __float2bfloat16_rn(x);
    return *reinterpret_cast<T *>(&h);
  }
};

struct ElemFp16 {
  using T = uint16_t;
  static constexpr int VEC = 8;
  static constexpr uint32_t kNegInf2 = 0xfc00fc00u;
  static constexpr T kNegInf = 0xfc00;
  static __device__ __forceinline__ uint32_t max_words(uint32_t x, uint32_t y) {
    uint32_t d;
    asm("max.f16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(y));
    return d;
  }
  static __device__ __forceinline__ T word_max_bits(uint32_t w) { return (T)max_words(w, w >> 16); }
  static __device__ __forceinline__ uint32_t reach_words(uint32_t x, uint32_t y) {
    return __hge2_mask(*reinterpret_cast<const __half2 *>(&x), *reinterpret_cast<const __half2 *>(&y));
  }
  // no finite half is far enough below the others
  static constexpr bool kHasFinite = false;
  static __device__ __forceinline__ uint32_t order_key(T b) { return order_key16(b); }
  static __device__ __forceinline__ T from_key(uint32_t k) { return from_key16(k); }
  static __device__ __forceinline__ float2 pair(uint32_t w) { return half2_to_float2(w); }
  static __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&p);
  }
  static __device__ __forceinline__ float to_float(T x) { return __half2float(*reinterpret_cast<const __half *>(&x)); }
  static __device__ __forceinline__ T from_float(float x) {
    __half h = __float2half_rn(x);
    return *reinterpret_cast<T *>(&h);
  }
};

struct ElemFp32 {
  using T = float;
  static constexpr int VEC = 4;
  static constexpr uint32_t kNegInf2 = 0xff800000u;
  static constexpr T kNegInf = -INFINITY;
  static __device__ __forceinline__ uint32_t max_words(uint32_t x, uint32_t y) {
    return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y)));
  }
  static __device__ __forceinline__ T word_max_bits(uint32_t w) { return __uint_as_float(w); }
  static constexpr bool kHasFinite = false;   // a maximum per element, as it costs where it is used
  static __device__ __forceinline__ uint32_t order_key(T b) {
    const uint32_t u = b == 0.f ? 0u : __float_as_uint(b);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
  }
  static __device__ __forceinline__ T from_key(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
  }
  static __device__ __forceinline__ float to_float(T x) { return x; }
  static __device__ __forceinline__ T from_float(float x) { return x; }
};

// The vector at element e of a row of V; none at or past V is read, they come out as -inf.
template <class E>
__device__ __forceinline__ uint4 load_raw(const typename E::T *row, int e, int V) {
  if (e + E::VEC <= V) return *reinterpret_cast<const uint4 *>(row + e);
  uint32_t w[4] = {E::kNegInf2, E::kNegInf2, E::kNegInf2, E::kNegInf2};
#pragma unroll
  for (int j = 0; j < E::VEC; ++j)
    if (e + j < V) {
      if constexpr (E::VEC == 8) {
        const uint32_t keep = (j & 1) ? 0x0000ffffu : 0xffff0000u;
        w[j / 2] = (w[j / 2] & keep) | ((uint32_t)row[e + j] << (16 * (j & 1)));
      } else {
        w[j] = __float_as_uint(row[e + j]);
      }
    }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ uint32_t word(const uint4 &u, int i) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  return w[i];
}

// words i and i + 1 of fp32 elements, or both elements of a 16-bit word, as two floats
template <class E>
__device__ __forceinline__ float2 pair_of(const uint4 &u, int i) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  if constexpr (E::VEC == 8)
    return E::pair(w[i]);
  else
    return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
}

// the elements of a 16-byte vector as floats, and back
template <class E>
__device__ __forceinline__ void unpack(const uint4 &u, float (&f)[E::VEC]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  if constexpr (E::VEC == 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = E::pair(w[i]);
      f[2 * i] = p.x;
      f[2 * i + 1] = p.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
  }
}

template <class E>
__device__ __forceinline__ uint4 pack(const float (&f)[E::VEC]) {
  if constexpr (E::VEC == 8)
    return make_uint4(E::pack2(f[0], f[1]), E::pack2(f[2], f[3]), E::pack2(f[4], f[5]), E::pack2(f[6], f[7]));
  else
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// Store the elements of a vector at element e of a row that are below V.
template <class E>
__device__ __forceinline__ void store_vec(typename E::T *row, int e, int V, const float (&f)[E::VEC]) {
  if (e + E::VEC <= V) {
    *reinterpret_cast<uint4 *>(row + e) = pack<E>(f);
  } else {
#pragma unroll
    for (int j = 0; j < E::VEC; ++j)
      if (e + j < V) row[e + j] = E::from_float(f[j]);
  }
}

inline size_t dtype_bytes(int dtype) { return dtype == UMIM_DTYPE_FP32 ? 4 : 2; }

}  // namespace umim
