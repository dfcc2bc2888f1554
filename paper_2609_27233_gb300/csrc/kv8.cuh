// The 8-bit cache: e4m3 values, and for each row of head_dim values a power of
// two 2^e as an e8m0 code e + 127.
#pragma once

#include "common.cuh"

namespace umim {

// Rows are rounded to the nearest e4m3 number (ties to even) of x / 2^e, e the
// smallest whole number with max |x| <= 448 * 2^e, 448 the largest e4m3 number.
// e stays within [-100, 120]: bf16's largest magnitude needs 120, and below -100
// nothing is left of a row that any other row would not drown.
constexpr int kKv8MinExp = -100, kKv8MaxExp = 120;
// The bf16 bits of 240 * 2^120, the largest magnitude that is stored: the next e4m3 number up,
// 256, times 2^120 is 2^128, which is finite neither in bf16 nor in fp32.
constexpr uint32_t kKv8Top = 0x7f70;

// e + 127 of a row whose largest magnitude has the bf16 bits `most` (finite):
// 448 = 1.75 * 2^8, so a significand above 1.75 (fraction bits above 96) needs one more.
__device__ __forceinline__ uint32_t kv8_scale_code(uint32_t most) {
  const int code = (int)((most + 31) >> 7) - 8;
  return most == 0 ? 127u : (uint32_t)min(max(code, kKv8MinExp + 127), kKv8MaxExp + 127);
}

// 2^(code - 127), NaN for code 255
__device__ __forceinline__ float e8m0_value(uint32_t code) {
  const uint32_t edge = ((code + 1) & 0xff) <= 1 ? 0x400000u : 0u;   // 2^-127 is no normal number, 255 is NaN
  return __uint_as_float(code << 23 | edge);
}

// two fp32 numbers to two e4m3 codes (the first in the low byte); NaN for NaN
__device__ __forceinline__ uint32_t e4m3x2_of(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// two e4m3 codes (the low 16 bits of x) as packed fp16: exact
__device__ __forceinline__ uint32_t f16x2_of_e4m3x2(uint32_t x) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)x));
  return r;
}

}  // namespace umim
