// Quantiser: rows or weights to e4m3 with a scale for each block of 1 x 128 or 128 x 128 (ks_quantize_e4m3).
//
// Bound by memory: an element is read once and its byte written once. Every block's values stay in registers between its
// maximum and their rounding.
#include <algorithm>

#include "ks_e4m3.cuh"
#include "ks_internal.h"
#include "ks_tcgen.cuh"

namespace ks {
namespace {

struct QuantArgs {
  const void* x;
  int64_t rows, cols, ldx;
  uint8_t* q;
  int64_t ldq;
  void* scale;
};

template <bool kE8m0>
__device__ __forceinline__ void store_scale(void* scale, int64_t at, uint32_t stored) {
  if (kE8m0) static_cast<uint8_t*>(scale)[at] = static_cast<uint8_t>(stored);
  else static_cast<uint32_t*>(scale)[at] = stored;
}

// N values of a row from column c on; zeros behind its end. kVec: the address is a multiple of 16 bytes.
template <typename T, int N, bool kVec>
__device__ __forceinline__ void load_values(const T* row, int64_t c, int64_t cols, float (&v)[N]) {
  if (kVec && c + N <= cols) {
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(row + c));
    T t[N];
    static_assert(sizeof(t) == 16, "one load");
    memcpy(t, &w, 16);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = to_float(t[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = c + i < cols ? to_float(row[c + i]) : 0.0f;
  }
}

// N bytes of a row from column c on, nothing behind its end. The row's address and c are multiples of N.
template <int N>
__device__ __forceinline__ void store_values(uint8_t* row, int64_t c, int64_t cols, const float (&v)[N], float inv) {
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) w[i] = e4m3_quad(v[4 * i] * inv, v[4 * i + 1] * inv, v[4 * i + 2] * inv, v[4 * i + 3] * inv);
  if (c + N <= cols) {
    if (N == 8) *reinterpret_cast<uint2*>(row + c) = make_uint2(w[0], w[N / 4 - 1]);
    else *reinterpret_cast<uint32_t*>(row + c) = w[0];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < cols) row[c + i] = static_cast<uint8_t>(w[i / 4] >> (8 * (i % 4)));
  }
}

constexpr int kQuantThreads = 256;

// A block of 1 x 128 belongs to the 16 or 32 lanes that its 16-byte pieces fill.
template <typename T, bool kE8m0, bool kVec>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kernel(const __grid_constant__ QuantArgs a) {
  next_may_start();
  wait_for_last();
  constexpr int kN = 16 / sizeof(T), kLanes = kScaleBlock / kN, kGroups = kQuantThreads / kLanes;
  const int64_t per_row = scale_blocks(a.cols), items = a.rows * per_row;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / kLanes;
  const bool live = item < items;
  const int64_t row = live ? item / per_row : 0, blk = live ? item - row * per_row : 0;
  const int64_t c = blk * kScaleBlock + (threadIdx.x % kLanes) * kN;
  float v[kN];
  load_values<T, kN, kVec>(static_cast<const T*>(a.x) + row * a.ldx, c, a.cols, v);
  float amax = 0.0f;
#pragma unroll
  for (int i = 0; i < kN; ++i) amax = fmaxf(amax, finite_abs(v[i]));
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
  if (!live) return;
  uint32_t stored;
  const float inv = block_scale<kE8m0>(amax, stored);
  if (threadIdx.x % kLanes == 0) store_scale<kE8m0>(a.scale, item, stored);
  store_values<kN>(a.q + row * a.ldq, c, a.cols, v, inv);
}

// A block of 128 x 128 belongs to a CTA, 64 values a thread.
template <typename T, bool kE8m0, bool kVec>
__global__ void __launch_bounds__(kQuantThreads) quantize_tiles_kernel(const __grid_constant__ QuantArgs a) {
  next_may_start();
  wait_for_last();
  constexpr int kN = 16 / sizeof(T), kLanes = kScaleBlock / kN, kRows = kQuantThreads / kLanes;
  constexpr int kSteps = kScaleBlock / kRows;
  __shared__ float s_max[kQuantThreads / 32];
  const int64_t per_row = scale_blocks(a.cols);
  const int64_t tr = blockIdx.x / per_row, tc = blockIdx.x - tr * per_row;
  const int64_t c = tc * kScaleBlock + (threadIdx.x % kLanes) * kN, r0 = tr * kScaleBlock + threadIdx.x / kLanes;
  float v[kSteps][kN];
  float amax = 0.0f;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int64_t r = r0 + s * kRows;
    load_values<T, kN, kVec>(static_cast<const T*>(a.x) + (r < a.rows ? r : 0) * a.ldx, c, r < a.rows ? a.cols : 0, v[s]);
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
#pragma unroll
    for (int i = 0; i < kN; ++i) amax = fmaxf(amax, finite_abs(v[s][i]));
#pragma unroll
  for (int d = 1; d < 32; d *= 2) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
  if (threadIdx.x % 32 == 0) s_max[threadIdx.x / 32] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQuantThreads / 32; ++w) amax = fmaxf(amax, s_max[w]);
  uint32_t stored;
  const float inv = block_scale<kE8m0>(amax, stored);
  if (threadIdx.x == 0) store_scale<kE8m0>(a.scale, blockIdx.x, stored);
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int64_t r = r0 + s * kRows;
    if (r < a.rows) store_values<kN>(a.q + r * a.ldq, c, a.cols, v[s], inv);
  }
}

template <typename T, bool kE8m0, bool kVec>
cudaError_t launch_quantize_as(const QuantArgs& a, int block_rows, cudaStream_t stream) {
  constexpr int kGroups = kQuantThreads * (16 / static_cast<int>(sizeof(T))) / kScaleBlock;
  const int64_t blocks = block_rows == 1 ? (a.rows * scale_blocks(a.cols) + kGroups - 1) / kGroups
                                         : scale_blocks(a.rows) * scale_blocks(a.cols);
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_following(block_rows == 1 ? &quantize_rows_kernel<T, kE8m0, kVec> : &quantize_tiles_kernel<T, kE8m0, kVec>,
                          dim3(static_cast<unsigned>(blocks)), kQuantThreads, 0, 0, stream, a);
}

template <typename T>
cudaError_t launch_quantize_type(const QuantArgs& a, int block_rows, int scale_type, cudaStream_t stream) {
  const bool vec = (reinterpret_cast<uintptr_t>(a.x) & 15u) == 0 && (a.rows == 1 || a.ldx * sizeof(T) % 16 == 0);
  if (scale_type == KS_SCALE_E8M0)
    return vec ? launch_quantize_as<T, true, true>(a, block_rows, stream) : launch_quantize_as<T, true, false>(a, block_rows, stream);
  return vec ? launch_quantize_as<T, false, true>(a, block_rows, stream) : launch_quantize_as<T, false, false>(a, block_rows, stream);
}

}  // namespace

cudaError_t launch_quantize_e4m3(const void* x, int x_type, int64_t rows, int64_t cols, int64_t ldx, int block_rows,
                                 int scale_type, uint8_t* q, int64_t ldq, void* scale, cudaStream_t stream, int64_t* launches) {
  const QuantArgs a{x, rows, cols, ldx, q, ldq, scale};
  ++*launches;
  switch (x_type) {
    case KS_F32: return launch_quantize_type<float>(a, block_rows, scale_type, stream);
    case KS_BF16: return launch_quantize_type<__nv_bfloat16>(a, block_rows, scale_type, stream);
    default: return launch_quantize_type<__half>(a, block_rows, scale_type, stream);
  }
}

}  // namespace ks
