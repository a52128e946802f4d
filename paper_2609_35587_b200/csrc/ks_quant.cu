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
    const uint4 w = *reinterpret_cast<const uint4*>(row + c);
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
// `odd`: some of the block's may be infinite.
template <int N>
__device__ __forceinline__ void store_values(uint8_t* row, int64_t c, int64_t cols, const float (&v)[N], float inv, bool odd) {
  uint32_t w[N / 4];
  if (odd) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) w[i] = e4m3_quad(v[4 * i] * inv, v[4 * i + 1] * inv, v[4 * i + 2] * inv, v[4 * i + 3] * inv);
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      w[i] = e4m3_pair_finite(v[4 * i] * inv, v[4 * i + 1] * inv) | (e4m3_pair_finite(v[4 * i + 2] * inv, v[4 * i + 3] * inv) << 16);
  }
  if (c + N <= cols) {
    if (N == 8) *reinterpret_cast<uint2*>(row + c) = make_uint2(w[0], w[N / 4 - 1]);
    else *reinterpret_cast<uint32_t*>(row + c) = w[0];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < cols) row[c + i] = static_cast<uint8_t>(w[i / 4] >> (8 * (i % 4)));
  }
}

constexpr int kQuantThreads = 256, kTileThreads = 512;

// A block of 1 x 128 belongs to eight lanes with 16 neighbouring values each. A CTA takes `across` neighbouring blocks (a power of
// two) of some rows, so that nothing is divided. What bounds it is not only memory: a thread with one 16-byte piece had 170
// instructions for its eight bf16 values, of which most place the piece and its scale (60,000 x 1,024: 43 us).
constexpr int kEach = 16, kLanes = kScaleBlock / kEach, kGroups = kQuantThreads / kLanes;

template <typename T, bool kE8m0, bool kVec>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kernel(const __grid_constant__ QuantArgs a, int across_bits) {
  next_may_start();
  wait_for_last();
  constexpr int kN = 16 / sizeof(T), kPieces = kEach / kN;
  const int group = threadIdx.x / kLanes, across = 1 << across_bits;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kGroups >> across_bits) + (group >> across_bits);
  const int64_t per_row = scale_blocks(a.cols);
  const T* x = static_cast<const T*>(a.x) + (row < a.rows ? row : 0) * a.ldx;
  uint8_t* q = a.q + row * a.ldq;
  for (int64_t first = static_cast<int64_t>(blockIdx.y) << across_bits; first < per_row; first += static_cast<int64_t>(gridDim.y) << across_bits) {
    const int64_t blk = first + (group & (across - 1)), c = blk * kScaleBlock + (threadIdx.x % kLanes) * kEach;
    const bool live = row < a.rows && blk < per_row;
    float v[kPieces][kN];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) load_values<T, kN, kVec>(x, c + p * kN, live ? a.cols : 0, v[p]);
    float amax = 0.0f;
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
      for (int i = 0; i < kN; ++i) amax = fmaxf(amax, fabsf(v[p][i]));  // (of what is not a number nothing)
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
    const bool odd = amax == __int_as_float(0x7F800000);
    if (__any_sync(0xFFFFFFFFu, odd)) {
      amax = 0.0f;
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int i = 0; i < kN; ++i) amax = fmaxf(amax, finite_abs(v[p][i]));
#pragma unroll
      for (int d = 1; d < kLanes; d *= 2) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
    }
    if (!live) continue;
    uint32_t stored;
    const float inv = block_scale<kE8m0>(amax, stored);
    if (threadIdx.x % kLanes == 0) store_scale<kE8m0>(a.scale, row * per_row + blk, stored);
    if (c + kEach <= a.cols && !odd) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* f = &v[0][0] + 4 * i;
        w[i] = e4m3_pair_finite(f[0] * inv, f[1] * inv) | (e4m3_pair_finite(f[2] * inv, f[3] * inv) << 16);
      }
      *reinterpret_cast<uint4*>(q + c) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int p = 0; p < kPieces; ++p) store_values<kN>(q, c + p * kN, a.cols, v[p], inv, odd);
    }
  }
}

// A block of 128 x 128 belongs to a CTA, 32 values a thread.
template <typename T, bool kE8m0, bool kVec>
__global__ void __launch_bounds__(kTileThreads) quantize_tiles_kernel(const __grid_constant__ QuantArgs a) {
  next_may_start();
  wait_for_last();
  constexpr int kN = 16 / sizeof(T), kAcross = kScaleBlock / kN, kRows = kTileThreads / kAcross;
  constexpr int kSteps = kScaleBlock / kRows;
  __shared__ float s_max[kTileThreads / 32];
  const int64_t per_row = scale_blocks(a.cols);
  const int64_t tr = blockIdx.x / per_row, tc = blockIdx.x - tr * per_row;
  const int64_t c = tc * kScaleBlock + (threadIdx.x % kAcross) * kN, r0 = tr * kScaleBlock + threadIdx.x / kAcross;
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
    for (int i = 0; i < kN; ++i) amax = fmaxf(amax, fabsf(v[s][i]));  // (of what is not a number nothing)
  const bool odd = __syncthreads_or(amax == __int_as_float(0x7F800000));
  if (odd) {
    amax = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int i = 0; i < kN; ++i) amax = fmaxf(amax, finite_abs(v[s][i]));
  }
#pragma unroll
  for (int d = 1; d < 32; d *= 2) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
  if (threadIdx.x % 32 == 0) s_max[threadIdx.x / 32] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kTileThreads / 32; ++w) amax = fmaxf(amax, s_max[w]);
  uint32_t stored;
  const float inv = block_scale<kE8m0>(amax, stored);
  if (threadIdx.x == 0) store_scale<kE8m0>(a.scale, blockIdx.x, stored);
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int64_t r = r0 + s * kRows;
    if (r < a.rows) store_values<kN>(a.q + r * a.ldq, c, a.cols, v[s], inv, odd);
  }
}

template <typename T, bool kE8m0, bool kVec>
cudaError_t launch_quantize_as(const QuantArgs& a, int block_rows, cudaStream_t stream) {
  if (block_rows == 1) {
    const int64_t per_row = scale_blocks(a.cols);
    int across_bits = 0;
    while ((2 << across_bits) <= kGroups && (1 << across_bits) < per_row) ++across_bits;
    const int64_t rows = kGroups >> across_bits;
    const int64_t stretches = std::min<int64_t>(65535, (per_row + (1 << across_bits) - 1) >> across_bits);
    return launch_following(&quantize_rows_kernel<T, kE8m0, kVec>, dim3(static_cast<unsigned>((a.rows + rows - 1) / rows), static_cast<unsigned>(stretches)),
                            kQuantThreads, 0, 0, stream, a, across_bits);
  }
  const int64_t blocks = scale_blocks(a.rows) * scale_blocks(a.cols);
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_following(&quantize_tiles_kernel<T, kE8m0, kVec>, dim3(static_cast<unsigned>(blocks)), kTileThreads, 0, 0, stream, a);
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
