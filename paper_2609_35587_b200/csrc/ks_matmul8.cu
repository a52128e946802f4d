// Product of two operands held in e4m3 with a scale for each block of 128 (ks_matmul_e4m3).
//
// d[m][n] = sum over blocks b of sa[m][b] * sb[n / 128][b] * (sum over k in b of a[m][k] * b[n][k]): the sum within a block
// is plain, so that the scales come in once per block. A tensor core makes a block's sums (128 of K, four MMAs of 32) into one
// of two accumulators, the epilogue's threads read them and add them, scaled, to fp32 sums in their registers, while the other
// accumulator is filled. So the sums of blocks are added with rounding, not with the tensor core's truncation, and scales of
// any value cost the same (matmul_pair_kernel; matmul_few_kernel for few results). Scales that are powers of two the tensor
// core multiplies in, and a long sum is read once (matmul_scaled_kernel).
#include <cuda.h>

#include <algorithm>
#include <cstring>

#include "ks_e4m3.cuh"
#include "ks_internal.h"
#include "ks_tcgen.cuh"

namespace ks {
namespace {

using Wide = unsigned long long;

constexpr int kSms = 148;  // of the one device this library is built for

__device__ __forceinline__ float scale_value(const void* s, int64_t at, int type) {
  return type == KS_SCALE_E8M0 ? e8m0_value(static_cast<const uint8_t*>(s)[at]) : static_cast<const float*>(s)[at];
}

// sum += value * s for two neighbours
__device__ __forceinline__ void add_scaled(Wide& sum, uint32_t lo, uint32_t hi, Wide s) {
  asm("{\n .reg .b64 t;\n mov.b64 t, {%1, %2};\n fma.rn.f32x2 %0, t, %3, %0;\n}\n" : "+l"(sum) : "r"(lo), "r"(hi), "l"(s));
}
__device__ __forceinline__ float low(Wide v) { return __uint_as_float(static_cast<uint32_t>(v)); }
__device__ __forceinline__ float high(Wide v) { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }

// D fp32, A and B e4m3, K-major
__host__ __device__ constexpr uint32_t instr_desc(int m, int n) {
  return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}

template <int kPair>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (kPair)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void commit_one(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// box of [rows][128 of K]; completes on a barrier of either CTA of the pair, or of this CTA
__device__ __forceinline__ void load_pair(uint32_t dst, const CUtensorMap* map, int k, int row, uint32_t cluster_bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
      "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(k), "r"(row), "r"(cluster_bar)
      : "memory");
}
__device__ __forceinline__ void load_one(uint32_t dst, const CUtensorMap* map, int k, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(k), "r"(row), "r"(bar)
      : "memory");
}

struct MatmulArgs {
  const void *a_scale, *b_scale;
  int scale_type;
  int m, n, kblocks;
  const float* bias;
  int relu;
  void* d;
  int64_t ldd;
  int row_bytes;  // rows of d begin on boundaries of 32 bytes, 16, or (0) less
  void* d_scale;
  int wait_limit, starve;
  int* status;
};

// Value of an element of the result before it is rounded.
__device__ __forceinline__ float finish(const MatmulArgs& p, float v, int n) {
  if (p.bias) v += p.bias[n];
  if (p.relu) v = v > 0.0f ? v : 0.0f;
  return v;
}

template <int kType>
__device__ __forceinline__ void store_one(const MatmulArgs& p, int64_t at, float v) {
  if (kType == KS_F32) static_cast<float*>(p.d)[at] = v;
  else if (kType == KS_BF16) static_cast<__nv_bfloat16*>(p.d)[at] = __float2bfloat16_rn(v);
  else if (kType == KS_F16) static_cast<__half*>(p.d)[at] = __float2half_rn(v);
  else static_cast<uint8_t*>(p.d)[at] = static_cast<uint8_t>(e4m3_pair(v, 0.0f));
}

template <int kType>
__device__ __forceinline__ uint32_t pack(const float* v) {  // four bytes of the result
  if (kType == KS_F32) return __float_as_uint(v[0]);
  if (kType == KS_BF16) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t*>(&t);
  }
  if (kType == KS_F16) {
    const __half2 t = __floats2half2_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t*>(&t);
  }
  return e4m3_quad(v[0], v[1], v[2], v[3]);
}
template <int kType> constexpr int kBytes = kType == KS_F32 ? 4 : kType == KS_E4M3 ? 1 : 2;

__device__ __forceinline__ float stored_scale(const MatmulArgs& p, float amax, int64_t at, bool write) {
  uint32_t stored;
  if (p.scale_type == KS_SCALE_E8M0) {
    const float inv = block_scale<true>(amax, stored);
    if (write) static_cast<uint8_t*>(p.d_scale)[at] = static_cast<uint8_t>(stored);
    return inv;
  }
  const float inv = block_scale<false>(amax, stored);
  if (write) static_cast<uint32_t*>(p.d_scale)[at] = stored;
  return inv;
}

// ------------------------------------------------------------------------------------------
// many rows: pairs of CTAs, 256 x 256 of the result at a time
// ------------------------------------------------------------------------------------------

// Two warps that have nothing else to do bring the scales, eight blocks of K at a time: the epilogue's threads would each read
// a row's, 32 sectors an instruction, which cost a fifth of the kernel's time. The epilogue has sixteen warps of 64 columns:
// what a warp does for a block of K is a chain of waits and loads, and four warps a scheduler hide each other's.
constexpr int kThreads = 640;  // warp 0 loads, warp 1 issues MMAs, warps 2 and 3 bring scales, warps 4..19 are the epilogue
constexpr int kRegs = 96, kRegsFew = 32, kRegsEpilogue = 112;  // a thread's registers at launch, and after the split
static_assert(128 * kRegsFew + 512 * kRegsEpilogue <= kThreads * kRegs, "the split hands out what the block was launched with");
constexpr int kTile = 256, kHalf = kTile / 2;
constexpr int kStages = 6;
constexpr int kOperandBytes = kHalf * kScaleBlock;  // a CTA's 128 rows of A, or its half of B's
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kChunk = 8;  // blocks of K whose scales are brought together
constexpr int kCols = 64;  // of an epilogue warp
constexpr int kStorePitch = 9;
// The next stage of the warp that issues MMAs: its barriers, and the low half of its operands' descriptor.
__device__ __forceinline__ uint32_t operand_low(uint32_t saddr) { return static_cast<uint32_t>(operand_desc(saddr)); }
__device__ __forceinline__ uint64_t operand_at(uint32_t low) { return (operand_desc(0) & 0xFFFFFFFF00000000ull) | low; }
struct Ring {
  uint32_t full, empty, low, parity;
  int stage;
  __device__ __forceinline__ void next() {
    const bool wraps = ++stage == kStages;
    stage = wraps ? 0 : stage;
    parity ^= wraps ? 1u : 0u;
    full += wraps ? 8u - 8u * kStages : 8u;
    empty += wraps ? 8u - 8u * kStages : 8u;
    low += wraps ? (kStageBytes >> 4) - (kStageBytes >> 4) * kStages : (kStageBytes >> 4);
  }
};

struct Tile {
  int m, n;
};
struct PairShared {  // behind the stages
  float a_scale[2][kChunk][kHalf];
  float b_scale[2][2][kChunk];
  float bias[2][kTile];
  Tile tile[2];
  alignas(16) float store[16][32 * kStorePitch];  // of a warp, for results whose rows do not begin on 16-byte boundaries
  float amax[2][16][32];  // of a warp's rows, for the one that has the block's other half
};
constexpr int kSmem = 1024 + kStages * kStageBytes + static_cast<int>(sizeof(PairShared));
constexpr int kGroup = 8;  // row tiles that share a stretch of column tiles, for L2

__device__ __forceinline__ Tile tile_at(uint32_t t, uint32_t tiles_m, uint32_t tiles_n) {
  const uint32_t per = kGroup * tiles_n, group = t / per, in = t - group * per, first = group * kGroup;
  const uint32_t rows = tiles_m - first < kGroup ? tiles_m - first : kGroup, col = in / rows;
  return Tile{static_cast<int>((first + in - col * rows) * kTile), static_cast<int>(col * kTile)};
}

// Bias and ReLU on a thread's 64 neighbouring elements of a row.
__device__ __forceinline__ void finish_block(const MatmulArgs& p, float (&sum)[kCols], const float* bias) {
  if (p.bias) {
    const float4* b = reinterpret_cast<const float4*>(bias);
#pragma unroll
    for (int q = 0; q < kCols / 4; ++q) {
      const float4 x = b[q];
      sum[4 * q] += x.x;
      sum[4 * q + 1] += x.y;
      sum[4 * q + 2] += x.z;
      sum[4 * q + 3] += x.w;
    }
  }
  if (p.relu) {
#pragma unroll
    for (int q = 0; q < kCols; ++q) sum[q] = fmaxf(sum[q], 0.0f);  // (of what is not a number 0)
  }
}

// Largest magnitude of them; `odd`: some may be infinite (those do not count).
__device__ __forceinline__ float block_max(const float (&sum)[kCols], bool& odd) {
  float amax = 0.0f;
#pragma unroll
  for (int q = 0; q < kCols; ++q) amax = fmaxf(amax, fabsf(sum[q]));
  odd = amax == __int_as_float(0x7F800000);
  if (odd) {
    amax = 0.0f;
#pragma unroll
    for (int q = 0; q < kCols; ++q) amax = fmaxf(amax, finite_abs(sum[q]));
  }
  return amax;
}

// Writes them, rounded to the result's type (e4m3: already scaled).
template <int kType, bool kLines>
__device__ __forceinline__ void store_block(const MatmulArgs& p, int row, int n0, const float (&sum)[kCols], bool odd, float* s_store) {
  const int lane = threadIdx.x & 31;
  if constexpr (kLines && kType != KS_F32) {
    // whole lines through shared memory, 1 KB at a time: a thread that writes its own row touches 32 lines a store (60,000 x 1,024 x
    // 1,024, bf16: 73 us so, 66 by lines). Where the instructions of the sums bound the kernel it does not pay (e4m3: 86 and 92).
    if (p.row_bytes > 0 && n0 + kCols <= p.n) {
      constexpr int kRow = kCols * kBytes<kType>, kPieces = kRow / 16, kRows = 1024 / kRow, kPer = 4 / kBytes<kType>;
      auto at = [](int r, int c) { return r * kRow + (c ^ (kPieces == 8 ? r & 7 : r >> 1 & 3)) * 16; };  // (no conflicts)
      char* stage = reinterpret_cast<char*>(s_store);
      char* out = static_cast<char*>(p.d) + (static_cast<int64_t>(row - lane) * p.ldd + n0) * kBytes<kType>;
      uint32_t w[kRow / 4];
#pragma unroll
      for (int i = 0; i < kRow / 4; ++i) {
        const float* v = sum + i * kPer;
        if (kType == KS_E4M3 && !odd) w[i] = e4m3_pair_finite(v[0], v[1]) | (e4m3_pair_finite(v[2], v[3]) << 16);
        else w[i] = pack<kType>(v);
      }
#pragma unroll
      for (int g = 0; g < 32; g += kRows) {
        __syncwarp();
        if (lane / kRows == g / kRows)
#pragma unroll
          for (int c = 0; c < kPieces; ++c)
            *reinterpret_cast<uint4*>(stage + at(lane % kRows, c)) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 64; i += 32) {
          const int r = (i + lane) / kPieces, c = lane % kPieces;
          if (row - lane + g + r < p.m)
            *reinterpret_cast<uint4*>(out + (g + r) * p.ldd * kBytes<kType> + c * 16) = *reinterpret_cast<const uint4*>(stage + at(r, c));
        }
      }
      return;
    }
  }
  constexpr int kPer = 4 / kBytes<kType>;  // elements of four bytes
  // (rows on boundaries of 16 bytes, 20,357 x 4,340 x 1,230: fp32 322 us by threads that write their own row, 235 through shared
  // memory; bf16 197 and 201. Of 32 bytes, n = 4,352: 183 and 174, 151 and 201.)
  if ((kType == KS_F32 ? p.row_bytes == 32 : p.row_bytes > 0) && n0 + kCols <= p.n) {
    char* out = static_cast<char*>(p.d) + (static_cast<int64_t>(row) * p.ldd + n0) * kBytes<kType>;
#pragma unroll
    for (int g = 0; g < kCols / (8 * kPer); ++g) {  // 32 bytes at a time: a sector of the thread's row
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float* v = sum + (g * 8 + i) * kPer;
        if (kType == KS_E4M3 && !odd) w[i] = e4m3_pair_finite(v[0], v[1]) | (e4m3_pair_finite(v[2], v[3]) << 16);
        else w[i] = pack<kType>(v);
      }
      if (row >= p.m) continue;
      if (p.row_bytes == 16) {
        reinterpret_cast<uint4*>(out)[2 * g] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(out)[2 * g + 1] = make_uint4(w[4], w[5], w[6], w[7]);
      } else {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + 32 * g), "r"(w[0]), "r"(w[1]),
                     "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
      }
    }
    return;
  }
  // through shared memory, so that neighbouring threads write neighbouring elements of a row: 8 columns at a time
#pragma unroll
  for (int c0 = 0; c0 < kCols; c0 += 8) {
    if (n0 + c0 >= p.n) break;
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q) s_store[lane * kStorePitch + q] = sum[c0 + q];
    __syncwarp();
    const int n = n0 + c0 + lane % 8, row0 = row - lane;
    if (n < p.n)
      for (int r = lane / 8; r < 32 && row0 + r < p.m; r += 4)
        store_one<kType>(p, static_cast<int64_t>(row0 + r) * p.ldd + n, s_store[r * kStorePitch + lane % 8]);
  }
}

template <int kType>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
matmul_pair_kernel(const __grid_constant__ MatmulArgs p, const __grid_constant__ CUtensorMap map_a,
                   const __grid_constant__ CUtensorMap map_b) {
  extern __shared__ unsigned char smem_raw[];
  // full[kStages] (the leader's are used), empty[kStages], accumulator full[2] and read out[2] (the leader's), scales full[2]
  // and used[2], halves of a block's maxima [8]
  __shared__ __align__(16) Wide s_bar[2 * kStages + 16];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = blockIdx.x & 1;  // CTA of the pair; 0 issues the MMAs
  const uint32_t pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  unsigned char* smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  PairShared& sh = *reinterpret_cast<PairShared*>(smem + kStages * kStageBytes);
  const uint32_t sbase = smem_addr(smem), bar0 = smem_addr(&s_bar[0]);
  auto bar_full = [&](int s) { return bar0 + 8u * s; };
  auto bar_empty = [&](int s) { return bar0 + 8u * (kStages + s); };
  auto bar_acc = [&](uint32_t i) { return bar0 + 8u * (2 * kStages + i); };
  auto bar_read = [&](uint32_t i) { return bar0 + 8u * (2 * kStages + 2 + i); };
  auto bar_scale = [&](uint32_t i) { return bar0 + 8u * (2 * kStages + 4 + i); };
  auto bar_used = [&](uint32_t i) { return bar0 + 8u * (2 * kStages + 6 + i); };
  auto bar_max = [&](int i) { return bar0 + 8u * (2 * kStages + 8 + i); };

  if (tid == 0) {
    s_fail = 0;
    for (int s = 0; s < kStages; ++s) {
      bar_init(bar_full(s), 1);
      bar_init(bar_empty(s), 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(bar_acc(i), 1);
      bar_init(bar_read(i), 32);  // sixteen epilogue warps of each CTA
      bar_init(bar_scale(i), 2);
      bar_init(bar_used(i), 16);
    }
    for (int i = 0; i < 8; ++i) bar_init(bar_max(i), 2);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers exist before either is used
  fence_after();
  next_may_start();
  wait_for_last();
  const uint32_t tmem = s_tmem;
  const int tiles_m = (p.m + kTile - 1) / kTile, tiles_n = (p.n + kTile - 1) / kTile;
  const uint32_t tiles = static_cast<uint32_t>(tiles_m) * tiles_n;  // (checked by the host)
  const int chunks = p.kblocks > 0 ? (p.kblocks + kChunk - 1) / kChunk : 1;
  volatile int* v_fail = &s_fail;

  // Bounded wait; after the first that runs out every role of the CTA leaves its loop, and the pair's other CTA runs into
  // its own limit.
  auto wait_ok = [&](uint32_t bar, uint32_t parity) {
    if (bar_try_tmem(bar, parity)) return true;
    for (int i = 0; i < p.wait_limit; ++i) {
      if (bar_try_tmem(bar, parity)) return true;
      if ((i & 63) == 63 && *v_fail) return false;
    }
    *v_fail = 1;
    if (p.status) atomicExch(p.status, KS_ERR_TIMEOUT);
    return false;
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
    // The warps that load and issue stay together and one lane of them does the work, so that what it works with is uniform:
    // a lane of its own took 250 clocks for a wait that was over and as many for four MMAs.
    if (warp == 0) {
      const bool lead = elect_one();
      uint32_t s = 0, parity = 1;
      bool ok = true;
      for (uint32_t t = pair; t < tiles && ok; t += n_pairs) {
        const Tile at = tile_at(t, tiles_m, tiles_n);
        const int row_a = at.m + static_cast<int>(rank) * kHalf, row_b = at.n + static_cast<int>(rank) * kHalf;
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (!(ok = wait_ok(bar_empty(s), parity))) break;
          const uint32_t full = to_cluster(bar_full(s), 0), dst = sbase + s * kStageBytes;
          if (lead) {
            if (rank == 0) bar_expect(bar_full(s), 2u * kStageBytes);
            if (!p.starve) {  // test hook: without the copies the waits on this barrier run out
              load_pair(dst, &map_a, kb * kScaleBlock, row_a, full);
              load_pair(dst + kOperandBytes, &map_b, kb * kScaleBlock, row_b, full);
            }
          }
          if (++s == kStages) {
            s = 0;
            parity ^= 1u;
          }
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      if (rank == 0) {
        const bool lead = elect_one();
        // (what a block of K takes this warp is a chain: the next stage, accumulator and barriers are kept, not computed)
        Ring ring{bar_full(0), bar_empty(0), operand_low(sbase), 0, 0};
        uint32_t acc = 0, parity_acc = 1;
        bool ok = true;
        constexpr uint32_t idesc = instr_desc(kTile, kTile);
        for (uint32_t t = pair; t < tiles && ok; t += n_pairs) {
          for (int kb = 0; kb < p.kblocks; ++kb) {
            if (!(ok = wait_ok(bar_read(0) + 8u * acc, parity_acc) && wait_ok(ring.full, ring.parity))) break;
            fence_after();
            if (lead) {
#pragma unroll
              for (int k = 0; k < 4; ++k)  // 32 bytes on in K: two units of the address field
                mma<1>(tmem + acc * kTile, operand_at(ring.low + 2u * k), operand_at(ring.low + (kOperandBytes >> 4) + 2u * k), idesc, k > 0);
              commit_pair(ring.empty);
              commit_pair(bar_acc(0) + 8u * acc);
            }
            ring.next();
            parity_acc ^= acc;  // (after the second of the two)
            acc ^= 1u;
          }
        }
      }
      __syncwarp();
    } else {
      // scales of this CTA's rows and of both blocks of columns; with a tile's first also its bias
      const int r0 = (warp - 2) * 64 + lane;
      uint32_t it = 0;
      bool ok = true;
      uint32_t tile_par = 0;
      for (uint32_t t = pair; t < tiles && ok; t += n_pairs, tile_par ^= 1u) {
        const Tile at = tile_at(t, tiles_m, tiles_n);
        for (int c = 0; c < chunks; ++c, ++it) {
          const uint32_t buf = it & 1u;
          if (!(ok = __all_sync(0xFFFFFFFFu, wait_ok(bar_used(buf), ((it >> 1) & 1u) ^ 1u)))) break;
          const int kb0 = c * kChunk, n_kb = p.kblocks - kb0 < kChunk ? p.kblocks - kb0 : kChunk;
          if (c == 0 && warp == 2 && lane == 0) sh.tile[tile_par] = at;
          if (c == 0 && p.bias)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int n = (warp - 2) * kHalf + 32 * i + lane;
              sh.bias[tile_par][n] = at.n + n < p.n ? p.bias[at.n + n] : 0.0f;
            }
          const int j = warp - 2, nb = at.n / kScaleBlock + j;
          float w = 0.0f;
          if (lane < n_kb && nb * kScaleBlock < p.n) w = scale_value(p.b_scale, static_cast<int64_t>(nb) * p.kblocks + kb0 + lane, p.scale_type);
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            const int row = at.m + static_cast<int>(rank) * kHalf + r0 + 32 * h;
            const int64_t from = static_cast<int64_t>(row < p.m ? row : 0) * p.kblocks + kb0;
            float v[kChunk];
#pragma unroll
            for (int k = 0; k < kChunk; ++k) v[k] = k < n_kb ? scale_value(p.a_scale, from + k, p.scale_type) : 0.0f;
#pragma unroll
            for (int k = 0; k < kChunk; ++k) sh.a_scale[buf][k][r0 + 32 * h] = v[k];
          }
          if (lane < kChunk) sh.b_scale[buf][j][lane] = w;
          __syncwarp();
          if (lane == 0) bar_arrive(bar_scale(buf));
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpilogue));
    // warp w owns lanes 32 (w % 4) .. and 64 of a tile's columns, half of block j
    const int quarter = warp & 3, part = (warp - 4) >> 2, j = part >> 1;
    const int trow = quarter * 32 + lane;
    // the accumulator that comes next: its columns and barriers, of which those of the other differ in one bit
    uint32_t acc_col = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + part * kCols;
    uint32_t acc_bar = bar_acc(0), read_bar = to_cluster(bar_read(0), 0), acc_parity = 0;
    const uint32_t first = lane == 0;
    auto warp_wait = [&](uint32_t bar, uint32_t parity) {
      return bar_try_warp(bar, parity) || __all_sync(0xFFFFFFFFu, wait_ok(bar, parity));
    };
    uint32_t it = 0, tile_par = 0;
    bool ok = true;
    for (uint32_t t = pair; t < tiles && ok; t += n_pairs, tile_par ^= 1u) {
      float sum[kCols];
#pragma unroll
      for (int q = 0; q < kCols; ++q) sum[q] = 0.0f;
      for (int c = 0; c < chunks && ok; ++c, ++it) {
        const uint32_t buf = it & 1u;
        if (!(ok = warp_wait(bar_scale(buf), (it >> 1) & 1u))) break;
        const int n_kb = p.kblocks - c * kChunk;
        const float *sa = &sh.a_scale[buf][0][trow], *sb = &sh.b_scale[buf][j][0];
#pragma unroll
        for (int k = 0; k < kChunk; ++k) {
          if (k >= n_kb) break;
          const float s = sa[k * kHalf] * sb[k];
          if (!(ok = warp_wait(acc_bar, acc_parity))) break;
          fence_after();
          uint32_t r[32];
          tmem_read32(acc_col, r);
#pragma unroll
          for (int q = 0; q < 32; ++q) sum[q] = fmaf(__uint_as_float(r[q]), s, sum[q]);
          tmem_read32(acc_col + 32, r);
          fence_before();
          bar_arrive_tmem_if(read_bar, first);
#pragma unroll
          for (int q = 0; q < 32; ++q) sum[32 + q] = fmaf(__uint_as_float(r[q]), s, sum[32 + q]);
          acc_parity ^= (acc_bar >> 3) & 1u;  // (after the second of the two)
          acc_bar ^= 8u;
          read_bar ^= 8u;
          acc_col ^= kTile;
        }
        if (ok && c + 1 < chunks) {
          __syncwarp();
          if (lane == 0) bar_arrive(bar_used(buf));
        }
      }
      if (!ok) break;
      const Tile at = sh.tile[tile_par];
      const int row = at.m + static_cast<int>(rank) * kHalf + trow, n0 = at.n + part * kCols;
      const bool inside = n0 < p.n;  // (of the warp's columns any)
      finish_block(p, sum, sh.bias[tile_par] + part * kCols);
      bool odd = false;
      float amax = 0.0f;
      if (kType == KS_E4M3) {  // the block's other 64 columns are another warp's
        amax = block_max(sum, odd);
        sh.amax[tile_par][warp - 4][lane] = amax;
        __syncwarp();
        const int which = j * 4 + quarter;
        if (lane == 0) bar_arrive(bar_max(which));
        if (!(ok = __all_sync(0xFFFFFFFFu, wait_ok(bar_max(which), tile_par)))) break;
        amax = fmaxf(amax, sh.amax[tile_par][(warp - 4) ^ 4][lane]);
      }
      // (with the last chunk's scales the bias is read too; behind the stores the arrival would wait for them)
      __syncwarp();
      if (lane == 0) bar_arrive(bar_used((it - 1) & 1u));
      if (kType == KS_E4M3) {
        const float inv = stored_scale(p, amax, static_cast<int64_t>(row) * scale_blocks(p.n) + n0 / kScaleBlock,
                                       row < p.m && inside && !(part & 1));
#pragma unroll
        for (int q = 0; q < kCols; ++q) sum[q] *= inv;
      }
      if (inside) store_block<kType, false>(p, row, n0, sum, odd, sh.store[warp - 4]);
    }
  }
  // after a failure: time for the copies and MMAs in flight to end
  if (*v_fail)
    for (int i = 0; i < 64; ++i) __nanosleep(2000);
  __syncthreads();
  cluster_sync();
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// ------------------------------------------------------------------------------------------
// many rows, scales that are powers of two: the tensor core multiplies them in
// ------------------------------------------------------------------------------------------

// The same tiles, with MMAs that take a power of two for each row of A, row of B and 32 of K (of a block of 128 the same four
// times) from tensor memory. So one accumulator takes a whole part of K and is read once: of the 26,000 instructions that a
// tile of K = 1,024 takes an SM in matmul_pair_kernel, 17,000 read the accumulators of its blocks. The tensor core adds by
// truncation, always towards zero and by up to 2^-23 of the sum an addition, so a part is 4,096 of K at most (128 additions), and the
// parts are added in registers, with rounding. Measured against 64 bits, 4,352 x 512 results of operands without a sign, root mean
// square and largest of the sums: K = 1,024 2e-7 and 6e-7, 4,096 1.5e-6 and 2.4e-6, 8,192 the same (the mean is as large: all are too
// small); matmul_pair_kernel, which rounds between blocks, 5e-8, 9e-8 and 1.3e-7, 6e-7 at most. Operands of both signs, of the magnitudes'
// sum: 2.9e-9, 5.4e-9 and 3.9e-9, the other kernel 2.9e-9 to 2.6e-9. Parts of 1,024 would cost 8,192^3 six more readings of 700
// clocks a tile, beside 33,000.
// The scales' places leave room for one accumulator: the MMAs stand still while it is read into registers, 700 clocks of the
// 4,100 of K = 1,024, but not while a tile is finished and written. That takes about 6,000 clocks (60,000 x 1,024 results: 41 us
// for K = 128 quantised, 45 as bf16, 74 as fp32), so up to K = 1,024 it bounds the kernel as much as the MMAs do.
constexpr int kPart = 32;         // blocks of K that an accumulator takes
constexpr int kWords = 4;         // blocks of K whose scales are in a word
constexpr int kScaleBuffers = 4;
constexpr int kScaleBytes = 3 * 512;  // of a CTA's 128 rows and of both blocks of 128 columns
constexpr int kScaleColumn = 256;     // of tensor memory, 32 columns a buffer
struct ScaledShared {  // behind the stages
  alignas(128) uint8_t scale[kScaleBuffers][kScaleBytes];
  alignas(16) float bias[2][kTile];
  Tile tile[2];
  alignas(16) float store[16][32 * kStorePitch];
  float amax[2][16][32];
};
constexpr int kSmemScaled = 1024 + kStages * kStageBytes + static_cast<int>(sizeof(ScaledShared));

// D fp32, A and B e4m3, K-major, scales e8m0; of their words byte `k`
__device__ __forceinline__ uint32_t scaled_desc(int m, int n, uint32_t k) {
  return instr_desc(m, n) & ~(1u << 4) | (k << 4) | (1u << 23) | (k << 29);
}
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
      " tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
      : "memory");
}
// 32 rows of 16 bytes to four columns of tensor memory in both CTAs, the same for each quarter of the lanes
__device__ __forceinline__ void copy_scales(uint32_t column, uint32_t saddr) {
  const uint64_t desc = static_cast<uint64_t>((saddr >> 4) & 0x3FFFu) | (1ull << 16) | (8ull << 32) | (1ull << 46);  // groups of eight rows 128 bytes apart
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(column), "l"(desc) : "memory");
}

template <int kType>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
matmul_scaled_kernel(const __grid_constant__ MatmulArgs p, const __grid_constant__ CUtensorMap map_a,
                     const __grid_constant__ CUtensorMap map_b) {
  extern __shared__ unsigned char smem_raw[];
  // full[kStages] (the leader's are used), empty[kStages], scales full[kScaleBuffers] (the leader's) and used[kScaleBuffers],
  // accumulator full and read out (the leader's), bias there[2] and read[2], halves of a block's maxima [8]
  constexpr int kBars = 2 * kStages + 2 * kScaleBuffers + 2 + 4 + 8;
  __shared__ __align__(16) Wide s_bar[kBars];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = blockIdx.x & 1;  // CTA of the pair; 0 issues the MMAs
  const uint32_t pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  unsigned char* smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  ScaledShared& sh = *reinterpret_cast<ScaledShared*>(smem + kStages * kStageBytes);
  const uint32_t sbase = smem_addr(smem), bar0 = smem_addr(&s_bar[0]);
  auto bar_full = [&](int s) { return bar0 + 8u * s; };
  auto bar_empty = [&](int s) { return bar0 + 8u * (kStages + s); };
  constexpr int kAt = 2 * kStages;
  auto bar_scale = [&](uint32_t i) { return bar0 + 8u * (kAt + i); };
  auto bar_used = [&](uint32_t i) { return bar0 + 8u * (kAt + kScaleBuffers + i); };
  const uint32_t bar_acc = bar0 + 8u * (kAt + 2 * kScaleBuffers), bar_read = bar_acc + 8u;
  auto bar_bias = [&](uint32_t i) { return bar_read + 8u * (1 + i); };
  auto bar_bias_read = [&](uint32_t i) { return bar_read + 8u * (3 + i); };
  auto bar_max = [&](int i) { return bar_read + 8u * (5 + i); };

  if (tid == 0) {
    s_fail = 0;
    for (int s = 0; s < kStages; ++s) {
      bar_init(bar_full(s), 1);
      bar_init(bar_empty(s), 1);
    }
    for (int i = 0; i < kScaleBuffers; ++i) {
      bar_init(bar_scale(i), 4);  // two warps of each CTA
      bar_init(bar_used(i), 1);
    }
    bar_init(bar_acc, 1);
    bar_init(bar_read, 32);  // sixteen epilogue warps of each CTA
    for (int i = 0; i < 2; ++i) {
      bar_init(bar_bias(i), 2);
      bar_init(bar_bias_read(i), 16);
    }
    for (int i = 0; i < 8; ++i) bar_init(bar_max(i), 2);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers exist before either is used
  fence_after();
  next_may_start();
  wait_for_last();
  const uint32_t tmem = s_tmem;
  const int tiles_m = (p.m + kTile - 1) / kTile, tiles_n = (p.n + kTile - 1) / kTile;
  const uint32_t tiles = static_cast<uint32_t>(tiles_m) * tiles_n;
  volatile int* v_fail = &s_fail;
  auto wait_ok = [&](uint32_t bar, uint32_t parity) {  // (as in matmul_pair_kernel)
    if (bar_try_tmem(bar, parity)) return true;
    for (int i = 0; i < p.wait_limit; ++i) {
      if (bar_try_tmem(bar, parity)) return true;
      if ((i & 63) == 63 && *v_fail) return false;
    }
    *v_fail = 1;
    if (p.status) atomicExch(p.status, KS_ERR_TIMEOUT);
    return false;
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
    if (warp == 0) {
      const bool lead = elect_one();
      uint32_t s = 0, parity = 1;
      bool ok = true;
      for (uint32_t t = pair; t < tiles && ok; t += n_pairs) {
        const Tile at = tile_at(t, tiles_m, tiles_n);
        const int row_a = at.m + static_cast<int>(rank) * kHalf, row_b = at.n + static_cast<int>(rank) * kHalf;
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (!(ok = wait_ok(bar_empty(s), parity))) break;
          const uint32_t full = to_cluster(bar_full(s), 0), dst = sbase + s * kStageBytes;
          if (lead) {
            if (rank == 0) bar_expect(bar_full(s), 2u * kStageBytes);
            if (!p.starve) {  // test hook: without the copies the waits on this barrier run out
              load_pair(dst, &map_a, kb * kScaleBlock, row_a, full);
              load_pair(dst + kOperandBytes, &map_b, kb * kScaleBlock, row_b, full);
            }
          }
          if (++s == kStages) {
            s = 0;
            parity ^= 1u;
          }
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      if (rank == 0) {
        const bool lead = elect_one();
        Ring ring{bar_full(0), bar_empty(0), operand_low(sbase), 0, 0};
        uint32_t parity_acc = 1, buf = 0, parity_scale = 0;
        bool ok = true;
        const uint32_t scale0 = smem_addr(&sh.scale[0][0]);
        for (uint32_t t = pair; t < tiles && ok; t += n_pairs) {
          for (int kb0 = 0; kb0 < p.kblocks && ok; kb0 += kWords) {
            const uint32_t sa = tmem + kScaleColumn + 32u * buf, sb = sa + 16u;
            // (a buffer that is filled again has been used: the warps that fill it waited for its MMAs. The peer's threads
            // wrote half of it)
            while (ok && !bar_try(bar_scale(buf), parity_scale)) ok = wait_ok(bar_scale(buf), parity_scale);
            const bool part_begins = kb0 % kPart == 0;
            if (!ok || (part_begins && !(ok = wait_ok(bar_read, parity_acc)))) break;
            if (part_begins) parity_acc ^= 1u;
            fence_after();
            if (lead)
#pragma unroll
              for (int i = 0; i < 3; ++i) copy_scales(sa + (i == 0 ? 0 : 12 + 4 * i), scale0 + buf * kScaleBytes + i * 512);
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
              if (kb0 + j >= p.kblocks || !(ok = wait_ok(ring.full, ring.parity))) break;
              fence_after();
              if (lead) {
#pragma unroll
                for (int k = 0; k < 4; ++k)  // 32 bytes on in K: two units of the address field
                  mma_scaled(tmem, operand_at(ring.low + 2u * k), operand_at(ring.low + (kOperandBytes >> 4) + 2u * k),
                             scaled_desc(kTile, kTile, j), sa, sb, j > 0 || k > 0 || !part_begins);
                commit_pair(ring.empty);
              }
              ring.next();
            }
            if (ok && lead) {
              commit_pair(bar_used(buf));
              if (kb0 + kWords >= p.kblocks || (kb0 + kWords) % kPart == 0) commit_pair(bar_acc);
            }
            if (++buf == kScaleBuffers) {
              buf = 0;
              parity_scale ^= 1u;
            }
          }
        }
      }
      __syncwarp();
    } else {
      // scales of this CTA's rows (two rows a thread) and of one of the blocks of columns; a tile's place and bias
      const int j = warp - 2, r0 = j * 64 + lane;
      uint32_t buf = 0, parity_used = 1, tile_par = 0, tile_count = 0;
      bool ok = true;
      const bool words = p.kblocks % kWords == 0 && reinterpret_cast<uintptr_t>(p.a_scale) % 4 == 0 && reinterpret_cast<uintptr_t>(p.b_scale) % 4 == 0;
      auto word_at = [&](const void* scales, int64_t at, int n_kb) {
        const uint8_t* from = static_cast<const uint8_t*>(scales) + at;
        if (words) return *reinterpret_cast<const uint32_t*>(from);
        uint32_t w = 0;
#pragma unroll
        for (int k = 0; k < kWords; ++k)
          if (k < n_kb) w |= static_cast<uint32_t>(from[k]) << (8 * k);
        return w;
      };
      for (uint32_t t = pair; t < tiles && ok; t += n_pairs, tile_par ^= 1u, ++tile_count) {
        const Tile at = tile_at(t, tiles_m, tiles_n);
        float bias[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int n = at.n + j * kHalf + 32 * i + lane;
          bias[i] = p.bias && n < p.n ? p.bias[n] : 0.0f;
        }
        if (!(ok = __all_sync(0xFFFFFFFFu, wait_ok(bar_bias_read(tile_par), ((tile_count >> 1) & 1u) ^ 1u)))) break;
        if (j == 0 && lane == 0) sh.tile[tile_par] = at;
#pragma unroll
        for (int i = 0; i < 4; ++i) sh.bias[tile_par][j * kHalf + 32 * i + lane] = bias[i];
        __syncwarp();
        if (lane == 0) bar_arrive(bar_bias(tile_par));
        const int row = at.m + static_cast<int>(rank) * kHalf + r0, nb = at.n / kScaleBlock + j;
        for (int kb = 0; kb < p.kblocks; kb += kWords) {
          const int n_kb = p.kblocks - kb;  // (loaded in front of the wait)
          const uint32_t w0 = row < p.m ? word_at(p.a_scale, static_cast<int64_t>(row) * p.kblocks + kb, n_kb) : 0u;
          const uint32_t w1 = row + 32 < p.m ? word_at(p.a_scale, static_cast<int64_t>(row + 32) * p.kblocks + kb, n_kb) : 0u;
          const uint32_t wb = nb * kScaleBlock < p.n ? word_at(p.b_scale, static_cast<int64_t>(nb) * p.kblocks + kb, n_kb) : 0u;
          if (!(ok = __all_sync(0xFFFFFFFFu, wait_ok(bar_used(buf), parity_used)))) break;
          uint32_t* out = reinterpret_cast<uint32_t*>(sh.scale[buf]);
          // row r of 128: 16 bytes a lane r % 32, word r / 32 of them
          out[lane * 4 + 2 * j] = w0;
          out[lane * 4 + 2 * j + 1] = w1;
          *reinterpret_cast<uint4*>(out + 128 + 128 * j + 4 * lane) = make_uint4(wb, wb, wb, wb);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive_cluster(to_cluster(bar_scale(buf), 0));
          if (++buf == kScaleBuffers) {
            buf = 0;
            parity_used ^= 1u;
          }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpilogue));
    const int quarter = warp & 3, part = (warp - 4) >> 2, j = part >> 1;  // (as in matmul_pair_kernel)
    const int trow = quarter * 32 + lane;
    const uint32_t acc_col = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + part * kCols;
    const uint32_t read_bar = to_cluster(bar_read, 0), first = lane == 0;
    auto warp_wait = [&](uint32_t bar, uint32_t parity) {
      return bar_try_warp(bar, parity) || __all_sync(0xFFFFFFFFu, wait_ok(bar, parity));
    };
    uint32_t acc_parity = 0, tile_par = 0, tile_count = 0;
    bool ok = true;
    for (uint32_t t = pair; t < tiles && ok; t += n_pairs, tile_par ^= 1u, ++tile_count) {
      float sum[kCols];
#pragma unroll
      for (int q = 0; q < kCols; ++q) sum[q] = 0.0f;
      for (int kb = 0; kb < p.kblocks; kb += kPart) {
        if (!(ok = warp_wait(bar_acc, acc_parity))) break;
        acc_parity ^= 1u;
        fence_after();
        uint32_t r[32];
        tmem_read32(acc_col, r);
#pragma unroll
        for (int q = 0; q < 32; ++q) sum[q] += __uint_as_float(r[q]);
        tmem_read32(acc_col + 32, r);
        fence_before();
        bar_arrive_tmem_if(read_bar, first);
#pragma unroll
        for (int q = 0; q < 32; ++q) sum[32 + q] += __uint_as_float(r[q]);
      }
      if (!ok || !(ok = warp_wait(bar_bias(tile_par), (tile_count >> 1) & 1u))) break;
      const Tile at = sh.tile[tile_par];
      const int row = at.m + static_cast<int>(rank) * kHalf + trow, n0 = at.n + part * kCols;
      const bool inside = n0 < p.n;  // (of the warp's columns any)
      finish_block(p, sum, sh.bias[tile_par] + part * kCols);
      __syncwarp();
      if (lane == 0) bar_arrive(bar_bias_read(tile_par));
      bool odd = false;
      if (kType == KS_E4M3) {  // the block's other 64 columns are another warp's
        float amax = block_max(sum, odd);
        sh.amax[tile_par][warp - 4][lane] = amax;
        __syncwarp();
        const int which = j * 4 + quarter;
        if (lane == 0) bar_arrive(bar_max(which));
        if (!(ok = warp_wait(bar_max(which), tile_par))) break;
        amax = fmaxf(amax, sh.amax[tile_par][(warp - 4) ^ 4][lane]);
        const float inv = stored_scale(p, amax, static_cast<int64_t>(row) * scale_blocks(p.n) + n0 / kScaleBlock,
                                       row < p.m && inside && !(part & 1));
#pragma unroll
        for (int q = 0; q < kCols; ++q) sum[q] *= inv;
      }
      if (inside) store_block<kType, true>(p, row, n0, sum, odd, sh.store[warp - 4]);
    }
  }
  // after a failure: time for the copies and MMAs in flight to end
  if (*v_fail)
    for (int i = 0; i < 64; ++i) __nanosleep(2000);
  __syncthreads();
  cluster_sync();
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// ------------------------------------------------------------------------------------------
// few rows: a CTA takes 128 rows of the weights and a part of K
// ------------------------------------------------------------------------------------------

// The weights are the MMA's 128 rows and the few rows its columns, so that a CTA reads 16 KB of weights for a block of K
// whatever m is. The CTAs of a cluster share out K; their sums meet in shared memory, added in the order of the parts, so
// that the result's bits do not depend on timing.
constexpr int kFewThreads = 256;  // warp 0 loads, warp 1 issues MMAs, warps 2 and 3 bring scales, 4..7 are the epilogue
constexpr int kRedPitch = kScaleBlock + 4;

constexpr int kFewStages = 4;
template <int kN> constexpr int kFewStageBytes = kOperandBytes + kN * kScaleBlock;
template <int kN> constexpr int kFewSmem = 1024 + kFewStages * kFewStageBytes<kN>;
static_assert(kFewSmem<16> - 1024 >= 16 * kRedPitch * 4 && kFewSmem<64> - 1024 >= 64 * kRedPitch * 4, "the sums fit the stages");

template <int kType, int kN>
__global__ void __launch_bounds__(kFewThreads, 2)
matmul_few_kernel(const __grid_constant__ MatmulArgs p, const __grid_constant__ CUtensorMap map_a,
                  const __grid_constant__ CUtensorMap map_b, int parts) {
  extern __shared__ unsigned char smem_raw[];
  constexpr int kS = kFewStages;
  constexpr int kAcc = 4;  // accumulators
  constexpr int kTmem = kAcc * kN;
  constexpr int kChunk = 8;  // blocks of K whose scales are brought together
  __shared__ __align__(8) Wide s_bar[2 * kS + 2 * kAcc + 4];  // full, empty, accumulator full and read out, scales full[2] and used[2]
  __shared__ __align__(16) float s_scale[2][kChunk][kN];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int part = static_cast<int>(blockIdx.x) % parts, n0 = static_cast<int>(blockIdx.x) / parts * kScaleBlock;
  const int m0 = static_cast<int>(blockIdx.y) * kN;
  const int kb0 = static_cast<int>(static_cast<int64_t>(p.kblocks) * part / parts);
  const int kb1 = static_cast<int>(static_cast<int64_t>(p.kblocks) * (part + 1) / parts);
  unsigned char* smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_addr(smem), bar0 = smem_addr(&s_bar[0]);
  auto bar_full = [&](int s) { return bar0 + 8u * s; };
  auto bar_empty = [&](int s) { return bar0 + 8u * (kS + s); };
  auto bar_acc = [&](int i) { return bar0 + 8u * (2 * kS + i); };
  auto bar_read = [&](int i) { return bar0 + 8u * (2 * kS + kAcc + i); };
  auto bar_scale = [&](int i) { return bar0 + 8u * (2 * kS + 2 * kAcc + i); };
  auto bar_used = [&](int i) { return bar0 + 8u * (2 * kS + 2 * kAcc + 2 + i); };

  if (tid == 0) {
    s_fail = 0;
    for (int s = 0; s < kS; ++s) {
      bar_init(bar_full(s), 1);
      bar_init(bar_empty(s), 1);
    }
    for (int i = 0; i < kAcc; ++i) {
      bar_init(bar_acc(i), 1);
      bar_init(bar_read(i), 4);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(bar_scale(i), 2);
      bar_init(bar_used(i), 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "r"(kTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  next_may_start();
  wait_for_last();
  const uint32_t tmem = s_tmem;
  volatile int* v_fail = &s_fail;
  auto wait_ok = [&](uint32_t bar, uint32_t parity) {
    for (int i = 0; i < p.wait_limit; ++i) {
      if (bar_try_tmem(bar, parity)) return true;
      if ((i & 63) == 63 && *v_fail) return false;
    }
    *v_fail = 1;
    if (p.status) atomicExch(p.status, KS_ERR_TIMEOUT);
    return false;
  };

  float* s_sum = reinterpret_cast<float*>(smem);  // [kN][kRedPitch], once the stages are done with
  if (warp == 0) {
    if (lane == 0) {
      for (int kb = kb0, it = 0; kb < kb1; ++kb, ++it) {
        const int s = it % kS;
        if (!wait_ok(bar_empty(s), ((it / kS) & 1u) ^ 1u)) break;
        bar_expect(bar_full(s), kFewStageBytes<kN>);
        if (p.starve) continue;
        load_one(sbase + s * kFewStageBytes<kN>, &map_b, kb * kScaleBlock, n0, bar_full(s));
        load_one(sbase + s * kFewStageBytes<kN> + kOperandBytes, &map_a, kb * kScaleBlock, m0, bar_full(s));
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = instr_desc(kScaleBlock, kN);
      for (int kb = kb0, it = 0; kb < kb1; ++kb, ++it) {
        const int s = it % kS, acc = it % kAcc;
        if (!wait_ok(bar_read(acc), ((it / kAcc) & 1u) ^ 1u) || !wait_ok(bar_full(s), (it / kS) & 1u)) break;
        fence_after();
        const uint64_t dw = operand_desc(sbase + s * kFewStageBytes<kN>);
        const uint64_t dx = operand_desc(sbase + s * kFewStageBytes<kN> + kOperandBytes);
#pragma unroll
        for (int k = 0; k < 4; ++k) mma<0>(tmem + acc * kN, dw + 2u * k, dx + 2u * k, idesc, k > 0);
        commit_one(bar_empty(s));
        commit_one(bar_acc(acc));
      }
    }
    __syncwarp();
  } else if (warp < 4) {
    // The scales' products: threads by row and by stretches of a chunk, once for the four warps that use them (each of which
    // fetching its own took 28 us where this takes 20: 64 rows by 8,192 x 8,192, fp32 scales)
    constexpr int kOf = kN * kChunk / 64;  // blocks of a thread
    const int t = threadIdx.x - 64, r = t % kN, first = t / kN * kOf, m = m0 + r;
    const int64_t sa_at = static_cast<int64_t>(m < p.m ? m : 0) * p.kblocks, sb_at = static_cast<int64_t>(n0 / kScaleBlock) * p.kblocks;
    for (int kb = kb0, it = 0; kb < kb1; kb += kChunk, ++it) {
      float v[kOf];
#pragma unroll
      for (int k = 0; k < kOf; ++k)
        v[k] = m < p.m && kb + first + k < kb1 ? scale_value(p.a_scale, sa_at + kb + first + k, p.scale_type) *
                                                     scale_value(p.b_scale, sb_at + kb + first + k, p.scale_type) : 0.0f;
      if (!__all_sync(0xFFFFFFFFu, wait_ok(bar_used(it & 1), ((it >> 1) & 1u) ^ 1u))) break;
#pragma unroll
      for (int k = 0; k < kOf; ++k) s_scale[it & 1][first + k][r] = v[k];
      __syncwarp();
      if (lane == 0) bar_arrive(bar_scale(it & 1));
    }
  } else {
    const int w = warp - 4;
    const uint32_t tmem_mine = tmem + (static_cast<uint32_t>(w * 32) << 16);
    constexpr int kLoad = kN < 32 ? kN : 32;
    Wide sum[kN / 2];
#pragma unroll
    for (int q = 0; q < kN / 2; ++q) sum[q] = 0;
    for (int kb = kb0, it = 0; kb < kb1; ++kb, ++it) {
      const int acc = it % kAcc, buf = (it / kChunk) & 1;
      if (it % kChunk == 0 && !__all_sync(0xFFFFFFFFu, wait_ok(bar_scale(buf), (it / kChunk / 2) & 1u))) break;
      if (!__all_sync(0xFFFFFFFFu, wait_ok(bar_acc(acc), (it / kAcc) & 1u))) break;
      fence_after();
      const ulonglong2* sc = reinterpret_cast<const ulonglong2*>(s_scale[buf][it % kChunk]);
#pragma unroll
      for (int c = 0; c < kN; c += kLoad) {
        uint32_t r[32];
        if (kN < 32) {
          asm volatile(
              "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
              : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
              : "r"(tmem_mine + acc * kN));
#pragma unroll
          for (int q = 16; q < 32; ++q) r[q] = 0;
        } else {
          tmem_ld32(tmem_mine + acc * kN + c, r);
        }
        tmem_wait(r);
#pragma unroll
        for (int q = 0; q < kLoad / 4; ++q) {
          const ulonglong2 f = sc[c / 4 + q];
          add_scaled(sum[c / 2 + 2 * q], r[4 * q], r[4 * q + 1], f.x);
          add_scaled(sum[c / 2 + 2 * q + 1], r[4 * q + 2], r[4 * q + 3], f.y);
        }
      }
      fence_before();
      __syncwarp();
      if (lane == 0) {
        bar_arrive(bar_read(acc));
        if (it % kChunk == kChunk - 1) bar_arrive(bar_used(buf));
      }
    }
    // (the last accumulator is read: every copy has arrived and every MMA is done)
    asm volatile("barrier.cta.sync 1, 128;" ::: "memory");
    if (!*v_fail) {
#pragma unroll
      for (int q = 0; q < kN / 2; ++q) {
        s_sum[(2 * q) * kRedPitch + w * 32 + lane] = low(sum[q]);
        s_sum[(2 * q + 1) * kRedPitch + w * 32 + lane] = high(sum[q]);
      }
    }
  }
  if (*v_fail)
    for (int i = 0; i < 64; ++i) __nanosleep(2000);
  __syncthreads();
  if (parts > 1) cluster_sync();
  // rows of the result, dealt among the cluster's warps; a warp adds the parts of 128 columns, a lane four neighbours
  const int rows = min(p.m - m0, kN);
  const int n = n0 + 4 * lane;
  if (!*v_fail)
    for (int r = part * (kFewThreads / 32) + warp; r < rows; r += parts * (kFewThreads / 32)) {
      float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      const uint32_t mine = smem_addr(s_sum + r * kRedPitch + 4 * lane);
      for (int q = 0; q < parts; ++q) {
        float4 x;
        const uint32_t from = parts > 1 ? to_cluster(mine, q) : mine;
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(from));
        v[0] += x.x;
        v[1] += x.y;
        v[2] += x.z;
        v[3] += x.w;
      }
      float amax = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = n + e < p.n ? finish(p, v[e], n + e) : 0.0f;
        amax = fmaxf(amax, finite_abs(v[e]));
      }
      const int64_t row = m0 + r;
      if (kType == KS_E4M3) {
#pragma unroll
        for (int d = 1; d < 32; d *= 2) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
        const float inv = stored_scale(p, amax, row * scale_blocks(p.n) + n0 / kScaleBlock, lane == 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= inv;
      }
      if (p.row_bytes && n + 4 <= p.n) {
        char* out = static_cast<char*>(p.d) + (row * p.ldd + n) * kBytes<kType>;
        if (kType == KS_F32) *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[2], v[3]);
        else if (kType == KS_E4M3) *reinterpret_cast<uint32_t*>(out) = pack<kType>(v);
        else *reinterpret_cast<uint2*>(out) = make_uint2(pack<kType>(v), pack<kType>(v + 2));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < p.n) store_one<kType>(p, row * p.ldd + n + e, v[e]);
      }
    }
  if (parts > 1) cluster_sync();  // its sums are read by the others
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmem) : "memory");
}

// ------------------------------------------------------------------------------------------
// host
// ------------------------------------------------------------------------------------------

// [rows][k] bytes, boxes of `box_rows` rows and 128 of K, in the operands' swizzled form; zeros behind both ends
cudaError_t make_map(CUtensorMap* map, const void* base, int64_t rows, int64_t k, int64_t ld, int box_rows) {
  std::memset(map, 0, sizeof(*map));
  if (k == 0) return cudaSuccess;  // (no copy is made)
  const EncodeTiled fn = encode_tiled();
  if (!fn) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(k), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld)};
  const cuuint32_t box[2] = {kScaleBlock, static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t step[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}

template <int kType, bool kScaled>
cudaError_t launch_pair(const MatmulE4m3& q, const MatmulArgs& p, cudaStream_t stream) {
  void (*const kernel)(MatmulArgs, CUtensorMap, CUtensorMap) = kScaled ? &matmul_scaled_kernel<kType> : &matmul_pair_kernel<kType>;
  const void* address = reinterpret_cast<const void*>(kernel);
  // the register split is made for this count
  static const cudaError_t fits = [address] {
    cudaFuncAttributes attr{};
    const cudaError_t e = cudaFuncGetAttributes(&attr, address);
    return e != cudaSuccess ? e : attr.numRegs == kRegs ? cudaSuccess : cudaErrorInvalidKernelImage;
  }();
  if (fits != cudaSuccess) return fits;
  constexpr int kBytes = kScaled ? kSmemScaled : kSmem;
  CUtensorMap ma, mb;
  cudaError_t e = make_map(&ma, q.a, q.m, q.k, q.lda, kHalf);
  if (e == cudaSuccess) e = make_map(&mb, q.b, q.n, q.k, q.ldb, kHalf);
  if (e == cudaSuccess) e = ensure_dynamic_smem(address, kBytes);
  if (e != cudaSuccess) return e;
  const int64_t tiles = ((q.m + kTile - 1) / kTile) * ((q.n + kTile - 1) / kTile);
  if (tiles + kSms > UINT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_following(kernel, dim3(2 * static_cast<unsigned>(std::min<int64_t>(tiles, kSms / 2))), kThreads, kBytes, 0, stream, p, ma, mb);
}

template <int kType, int kN>
cudaError_t launch_few(const MatmulE4m3& q, const MatmulArgs& p, cudaStream_t stream) {
  CUtensorMap ma, mb;
  cudaError_t e = make_map(&ma, q.a, q.m, q.k, q.lda, kN);
  if (e == cudaSuccess) e = make_map(&mb, q.b, q.n, q.k, q.ldb, kScaleBlock);
  const void* kernel = reinterpret_cast<const void*>(&matmul_few_kernel<kType, kN>);
  if (e == cudaSuccess) e = ensure_dynamic_smem(kernel, kFewSmem<kN>);
  if (e != cudaSuccess) return e;
  const int64_t tiles = scale_blocks(q.n), rows = (q.m + kN - 1) / kN;  // (below 2^24; launch_type gives few)
  // parts of K, so that the machine's CTAs have work each
  int parts = 1;
  while (parts < 8 && 2 * parts <= p.kblocks && tiles * rows * parts * 2 <= kSms * 2) parts *= 2;
  return launch_following(&matmul_few_kernel<kType, kN>, dim3(static_cast<unsigned>(tiles * parts), static_cast<unsigned>(rows)), kFewThreads,
                          kFewSmem<kN>, parts, stream, p, ma, mb, parts);
}

template <int kType>
cudaError_t launch_type(const MatmulE4m3& q, const MatmulArgs& p, cudaStream_t stream) {
  // Layers of a ranker's sizes with powers of two: the kernel does not go by m, so that a row's result does not depend on the rows
  // beside it (the other kernel adds in another order, and a last bit in front of the rounding to e4m3 is a step of 6 % in an
  // activation). In a graph, us here and by the other kernel: 1 x 1,024 x 256 5.7 and 3.5, 1 x 1,024 x 1,024 7.7 and 3.9, 64 x 256 x
  // 256 6.1 and 5.7, 512 x 1,024 x 256 7.1 and 6.5, 4,096 x 128 x 256 6.0 and 6.4.
  if (q.scale_type == KS_SCALE_E8M0 && q.n <= KS_MLP_MAX_WIDTH && q.k <= KS_MLP_MAX_WIDTH) return launch_pair<kType, true>(q, p, stream);
  if (q.m <= 16) return launch_few<kType, 16>(q, p, stream);
  if (q.m <= 32) return launch_few<kType, 32>(q, p, stream);
  // Many rows too, where their results are so few that pairs would leave most of the machine idle (K is shared out there): K = 8,192,
  // 128 x 1,024 results with powers of two 25 us by pairs, 12 so, 512 x 1,024 26 and 19, 512 x 2,048 26 and 28. Pairs are slower
  // with fp32 scales: K = 8,192, 512 x 2,048 34 and 28, 512 x 4,096 34 and 48; K = 512, 512 x 2,048 7.7 and 8.4.
  const int64_t few = q.scale_type == KS_SCALE_F32 && p.kblocks >= 16 ? 128 : 64;
  if (q.m <= 64 || (q.m <= 64 * few && (q.m + 63) / 64 * scale_blocks(q.n) <= few)) return launch_few<kType, 64>(q, p, stream);
  return q.scale_type == KS_SCALE_E8M0 ? launch_pair<kType, true>(q, p, stream) : launch_pair<kType, false>(q, p, stream);
}

}  // namespace

cudaError_t launch_matmul_e4m3(const MatmulE4m3& q, int* status, cudaStream_t stream, int64_t* launches, const FastWait* wait) {
  const int bytes = q.d_type == KS_F32 ? 4 : q.d_type == KS_E4M3 ? 1 : 2;
  MatmulArgs p{};
  p.a_scale = q.a_scale;
  p.b_scale = q.b_scale;
  p.scale_type = q.scale_type;
  p.m = static_cast<int>(q.m);
  p.n = static_cast<int>(q.n);
  p.kblocks = static_cast<int>(scale_blocks(q.k));
  p.bias = q.bias;
  p.relu = q.relu;
  p.d = q.d;
  p.ldd = q.ldd;
  const uintptr_t ends = reinterpret_cast<uintptr_t>(q.d) | (q.m == 1 ? 0 : static_cast<uintptr_t>(q.ldd * bytes));
  p.row_bytes = ends % 32 == 0 ? 32 : ends % 16 == 0 ? 16 : 0;
  p.d_scale = q.d_scale;
  p.wait_limit = wait->limit > 0 ? wait->limit : kMlpWaitLimit;
  p.starve = wait->starve;
  p.status = status;
  ++*launches;
  switch (q.d_type) {
    case KS_F32: return launch_type<KS_F32>(q, p, stream);
    case KS_BF16: return launch_type<KS_BF16>(q, p, stream);
    case KS_F16: return launch_type<KS_F16>(q, p, stream);
    default: return launch_type<KS_E4M3>(q, p, stream);
  }
}

}  // namespace ks
