// Product of two operands held in e4m3 with a scale for each block of 128 (ks_matmul_e4m3).
//
// d[m][n] = sum over blocks b of sa[m][b] * sb[n / 128][b] * (sum over k in b of a[m][k] * b[n][k]): the sum within a block
// is plain, so that the scales come in once per block and not once per element.
#include <cuda_fp8.h>

#include <algorithm>

#include "ks_e4m3.cuh"
#include "ks_internal.h"

namespace ks {
namespace {

constexpr int kRows = 32, kCols = kScaleBlock, kStep = 32, kThreads = 256;

__device__ __forceinline__ float e4m3_value(uint8_t v) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(v, __NV_E4M3)));
}

__device__ __forceinline__ float scale_value(const void* s, int64_t at, int type) {
  return type == KS_SCALE_E8M0 ? e8m0_value(static_cast<const uint8_t*>(s)[at]) : static_cast<const float*>(s)[at];
}

// A CTA makes 32 rows x 128 columns: a warp four rows, a lane every 32nd column of them, so that a row's 128 columns, the
// block of a quantised result, lie in one warp.
__global__ void __launch_bounds__(kThreads) matmul_kernel(const __grid_constant__ MatmulE4m3 p) {
  __shared__ float s_a[kRows][kStep + 1], s_b[kCols][kStep + 1];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * kRows, n0 = static_cast<int64_t>(blockIdx.x) * kCols;
  const int64_t kb = scale_blocks(p.k);
  float sum[4][4] = {};
  for (int64_t b = 0; b < kb; ++b) {
    float part[4][4] = {};
    for (int64_t k0 = b * kScaleBlock; k0 < p.k && k0 < (b + 1) * kScaleBlock; k0 += kStep) {
      __syncthreads();
      for (int i = threadIdx.x; i < kRows * kStep; i += kThreads) {
        const int64_t m = m0 + i / kStep, k = k0 + i % kStep;
        s_a[i / kStep][i % kStep] = m < p.m && k < p.k ? e4m3_value(p.a[m * p.lda + k]) : 0.0f;
      }
      for (int i = threadIdx.x; i < kCols * kStep; i += kThreads) {
        const int64_t n = n0 + i / kStep, k = k0 + i % kStep;
        s_b[i / kStep][i % kStep] = n < p.n && k < p.k ? e4m3_value(p.b[n * p.ldb + k]) : 0.0f;
      }
      __syncthreads();
      for (int k = 0; k < kStep; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) part[i][j] = fmaf(s_a[warp * 4 + i][k], s_b[lane + 32 * j][k], part[i][j]);
    }
    const float sb = scale_value(p.b_scale, static_cast<int64_t>(blockIdx.x) * kb + b, p.scale_type);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t m = m0 + warp * 4 + i;
      const float s = m < p.m ? scale_value(p.a_scale, m * kb + b, p.scale_type) * sb : 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[i][j] = fmaf(part[i][j], s, sum[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t m = m0 + warp * 4 + i;
    if (m >= p.m) continue;
    float amax = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t n = n0 + lane + 32 * j;
      if (n < p.n && p.bias) sum[i][j] += p.bias[n];
      if (p.relu) sum[i][j] = sum[i][j] > 0.0f ? sum[i][j] : 0.0f;
      if (n < p.n) amax = fmaxf(amax, finite_abs(sum[i][j]));
    }
    float inv = 1.0f;
    if (p.d_type == KS_E4M3) {
#pragma unroll
      for (int d = 1; d < 32; d *= 2) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
      uint32_t stored;
      inv = p.scale_type == KS_SCALE_E8M0 ? block_scale<true>(amax, stored) : block_scale<false>(amax, stored);
      const int64_t at = m * scale_blocks(p.n) + blockIdx.x;
      if (lane == 0) {
        if (p.scale_type == KS_SCALE_E8M0) static_cast<uint8_t*>(p.d_scale)[at] = static_cast<uint8_t>(stored);
        else static_cast<uint32_t*>(p.d_scale)[at] = stored;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t n = n0 + lane + 32 * j, at = m * p.ldd + n;
      if (n >= p.n) continue;
      const float v = sum[i][j];
      switch (p.d_type) {
        case KS_F32: static_cast<float*>(p.d)[at] = v; break;
        case KS_BF16: static_cast<__nv_bfloat16*>(p.d)[at] = __float2bfloat16_rn(v); break;
        case KS_F16: static_cast<__half*>(p.d)[at] = __float2half_rn(v); break;
        default: static_cast<uint8_t*>(p.d)[at] = static_cast<uint8_t>(e4m3_pair(v * inv, 0.0f));
      }
    }
  }
}

}  // namespace

cudaError_t launch_matmul_e4m3(const MatmulE4m3& p, int* status, cudaStream_t stream, int64_t* launches, const FastWait* wait) {
  const int64_t bx = scale_blocks(p.n), by = (p.m + kRows - 1) / kRows;
  if (by > 65535) return cudaErrorInvalidConfiguration;
  matmul_kernel<<<dim3(static_cast<unsigned>(bx), static_cast<unsigned>(by)), kThreads, 0, stream>>>(p);
  ++*launches;
  return cudaGetLastError();
}

}  // namespace ks
