// Eight-bit values with a scale for each block of 128: conversions, and the scale of a block.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "ks.h"

namespace ks {

constexpr int kScaleBlock = KS_SCALE_BLOCK;

__host__ __device__ constexpr int64_t scale_blocks(int64_t n) { return (n + kScaleBlock - 1) / kScaleBlock; }

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float(float v) { return v; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

// What an element adds to its block's maximum: values that are not finite do not count.
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a < __int_as_float(0x7F800000) ? a : 0.0f;
}

// Scale of a block whose largest finite magnitude is `amax`, as it is stored, and the factor its values are multiplied
// by. e8m0: 2^e with the smallest e that brings the block to 448 = 1.75 * 2^8 or below. Multiplying by a power of two is
// exact, so that the only rounding of the quantiser is that to e4m3. f32: amax / 448, of a maximum that is at least
// 2^-100 (what lies below becomes zero): then neither the scale nor its reciprocal over- or underflows.
template <bool kE8m0>
__device__ __forceinline__ float block_scale(float amax, uint32_t& stored) {
  if (kE8m0) {
    const uint32_t bits = __float_as_uint(amax);
    // exponent of amax (subnormals: below every scale that is kept) minus 8, one more above 1.75
    int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = amax > 0.0f ? (e < -127 ? -127 : e) : -127;
    stored = static_cast<uint32_t>(e + 127);
    return __uint_as_float(static_cast<uint32_t>(127 - e) << 23);  // 127 - e is 7 .. 254
  }
  const float a = fmaxf(amax, 7.8886090522101181e-31f);  // 2^-100
  stored = __float_as_uint(__fdiv_rn(a, 448.0f));
  return __fdiv_rn(448.0f, a);
}

// Value of a stored scale.
__device__ __forceinline__ float e8m0_value(uint32_t b) {  // (0 is 2^-127, below the normal numbers; 255 is not a number)
  return b == 0u ? __uint_as_float(0x400000u) : b == 255u ? __uint_as_float(0x7FFFFFFFu) : __uint_as_float(b << 23);
}

// Two scaled values as e4m3, `lo` in the low byte; what is not finite becomes the code that is no number. The first form is for
// values that are not infinite (the conversion makes 448 of those).
__device__ __forceinline__ uint32_t e4m3_pair_finite(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
  uint32_t v = e4m3_pair_finite(lo, hi);
  const float inf = __int_as_float(0x7F800000);
  if (fabsf(lo) == inf) v |= 0x7Fu;
  if (fabsf(hi) == inf) v |= 0x7F00u;
  return v;
}
__device__ __forceinline__ uint32_t e4m3_quad(float a, float b, float c, float d) {
  return e4m3_pair(a, b) | (e4m3_pair(c, d) << 16);
}

}  // namespace ks
