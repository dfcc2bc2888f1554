// Rows of logits as the loss and log-probability kernels read them: 16-byte
// vectors of bf16, fp16 or fp32 elements, computed on in fp32.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace umim {

constexpr int kMaxLogitVocab = 262144;   // vocabulary size of the calls below, at most
constexpr int kMaxTop = 128;             // alternatives per row, at most
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float2 half2_to_float2(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

// The three element types: VEC elements to a 16-byte vector, unpacked to and
// packed from fp32 (packing rounds to nearest even).
struct ElemBf16 {
  using T = uint16_t;
  static constexpr int VEC = 8;
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
  static __device__ __forceinline__ float to_float(T x) { return x; }
  static __device__ __forceinline__ T from_float(float x) { return x; }
};

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

// The elements of the vector at element e of a row; none at or past V is read, they come out as `fill`.
template <class E>
__device__ __forceinline__ void load_vec(const typename E::T *row, int e, int V, float fill, float (&f)[E::VEC]) {
  if (e + E::VEC <= V) {
    unpack<E>(*reinterpret_cast<const uint4 *>(row + e), f);
  } else {
#pragma unroll
    for (int j = 0; j < E::VEC; ++j) f[j] = e + j < V ? E::to_float(row[e + j]) : fill;
  }
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
