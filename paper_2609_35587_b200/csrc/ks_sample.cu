// Draws from the softmax of scores with temperature, top-k, top-p and min-p (ks_sample).
//
// A score's weight exp((x - best) / t) is held as a whole number of 2^-s of the best one's, with 64-bit sums. Sums of whole
// numbers do not depend on the order they are taken in, so the cuts and the draws do not depend on how a row is shared out;
// and what a rounding of 2^-s moves at a border lies far below what 32 bits of a weight would (a draw among 100,000 equal
// candidates meets a border within 2^-24 once in 100 times).
//
// The candidates that stay are the front of the order (score descending, index ascending), so top-k and top-p are each a
// place in it. A histogram over the distance to the best score narrows it down to one bin, in which some hundred candidates
// lie; they are sorted. Bins that hold more are narrowed down further by the bits of (score, index).
//
// A row of a call with few rows belongs to a cluster of up to 16 CTAs that keep its scores in shared memory, each thread its
// own; the CTAs' results meet there too. Where there are rows for the whole machine a CTA takes a row by itself and reads it
// again in every phase, mostly from L2: four smaller CTAs an SM hide each other's barriers, of which a cluster has more and
// longer ones (1,024 x 60,000 scores: 947 us by clusters of 4).
#include <algorithm>
#include <cmath>

#include "ks_e4m3.cuh"
#include "ks_internal.h"
#include "ks_tcgen.cuh"
#include "ks_topk.cuh"

namespace ks {
namespace {

using Wide = unsigned long long;

// (what is not inlined passes a load's scores through memory)
#define KS_INLINE __attribute__((always_inline))

template <typename T> constexpr bool is_bf16 = false;
template <> constexpr bool is_bf16<__nv_bfloat16> = true;

constexpr int kBins = 1024;
constexpr int kList = 1024;        // candidates of a bin that are sorted
constexpr int kMaxCtas = 16;       // of a cluster
constexpr int kHeldLoads = 8;      // 16-byte loads that a thread keeps at most
constexpr int kEntries = 1024;     // sums over stretches of a row that a CTA keeps
constexpr float kReach = 36.05f;   // (best - x) / t behind which every weight rounds to 0 (51 bits)
constexpr int kDigit = 10;         // bits of (score, index) that a bin is narrowed down by

struct Row {
  float best;
  float reach;        // scores further below the best one have no weight
  float bins;         // bins a unit of score
  double best_wide;
  double steps;       // 64ths of a power of two a unit of score
  double one;         // weight of the best score, 2^s
  double least;       // weights below do not stay (min-p)
};

// Weight of a score within reach in units of 2^-s, before it is rounded: 2^(n / 64) from a table of 64 (times 2^s) and the
// exponent, times the exponential of what is left, at most ln 2 / 128, by its series (P. T. P. Tang's table-driven method, ACM
// TOMS 15, 1989). The first term that is left out is below 2^-54. The best score's weight is exact, also where it is infinite.
__device__ __forceinline__ double scaled_weight(const Row& r, const double* table, float x) {
  constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: adding it rounds to a whole number in the low word
  constexpr double kL = 0.69314718055994530942 / 64.0;
  const double z = (static_cast<double>(x) - r.best_wide) * r.steps, m = z + kRound;
  const int n = __double2loint(m);
  const double f = z - (m - kRound);
  double e = fma(f, kL * kL * kL * kL * kL / 120.0, kL * kL * kL * kL / 24.0);
  e = fma(f, e, kL * kL * kL / 6.0);
  e = fma(f, e, kL * kL / 2.0);
  e = fma(f, e, kL);
  e = fma(f, e, 1.0);
  const double w = table[n & 63] * e;
  const double v = __hiloint2double(__double2hiint(w) + ((n >> 6) << 20), __double2loint(w));
  return x == r.best ? r.one : v;
}
// rounded; w <= 2^51, so that the sum's low bits are the whole number
__device__ __forceinline__ Wide whole(double w) {
  return static_cast<Wide>(__double_as_longlong(w + 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
}

__device__ __forceinline__ int bin_of(const Row& r, float x) {
  return static_cast<int>(fminf((r.best - x) * r.bins, static_cast<float>(kBins - 1)));
}

__device__ __forceinline__ Wide warp_scan(Wide v, int lane) {  // inclusive
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const Wide u = __shfl_up_sync(0xFFFFFFFFu, v, d);
    if (lane >= d) v += u;
  }
  return v;
}
__device__ __forceinline__ Wide warp_sum(Wide v) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// Exclusive sum over the block's threads; the block's in `total`.
template <int kWarps>
__device__ __forceinline__ Wide block_scan(Wide v, Wide (&s_warp)[kWarps], Wide& total) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const Wide in = warp_scan(v, lane);
  __syncthreads();
  if (lane == 31) s_warp[warp] = in;
  __syncthreads();
  const Wide all = warp_scan(lane < kWarps ? s_warp[lane] : 0, lane);
  total = __shfl_sync(0xFFFFFFFFu, all, kWarps - 1);
  const Wide before = __shfl_sync(0xFFFFFFFFu, all, warp > 0 ? warp - 1 : 0);
  return (warp > 0 ? before : 0) + in - v;
}

// The same of two numbers at once.
template <int kWarps>
__device__ __forceinline__ void block_scan2(Wide& v, Wide& w, Wide (&s_warp)[2][kWarps], Wide& total_v, Wide& total_w) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const Wide in_v = warp_scan(v, lane), in_w = warp_scan(w, lane);
  __syncthreads();
  if (lane == 31) {
    s_warp[0][warp] = in_v;
    s_warp[1][warp] = in_w;
  }
  __syncthreads();
  const Wide all_v = warp_scan(lane < kWarps ? s_warp[0][lane] : 0, lane), all_w = warp_scan(lane < kWarps ? s_warp[1][lane] : 0, lane);
  total_v = __shfl_sync(0xFFFFFFFFu, all_v, kWarps - 1);
  total_w = __shfl_sync(0xFFFFFFFFu, all_w, kWarps - 1);
  const Wide before_v = __shfl_sync(0xFFFFFFFFu, all_v, warp > 0 ? warp - 1 : 0);
  const Wide before_w = __shfl_sync(0xFFFFFFFFu, all_w, warp > 0 ? warp - 1 : 0);
  v = (warp > 0 ? before_v : 0) + in_v - v;
  w = (warp > 0 ? before_w : 0) + in_w - w;
}

template <int kWarps>
struct Shared {
  double table[64];
  unsigned count[kBins];
  unsigned low[kBins], high[kBins];  // of a bin's sum
  unsigned m_count[kBins / 2];  // this CTA's share of the bins, over the cluster
  Wide m_sum[kBins / 2];
  Wide list[kList];
  Wide warp[kWarps], warp2[2][kWarps];
  // what the cluster's other CTAs read
  Wide best;
  float least[kWarps], min;
  Wide share_count, share_sum, before_count, before_sum, total, cut, cut_sum;
  int bin;
  unsigned held, listed;
};

template <typename U>
__device__ __forceinline__ U* of_rank(U* p, int rank, int ctas) {  // the same variable of the cluster's CTA `rank`
  if (ctas == 1) return p;
  uint64_t a;
  asm("mapa.u64 %0, %1, %2;" : "=l"(a) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
  return reinterpret_cast<U*>(a);
}

__device__ __forceinline__ void meet(int ctas) {
  if (ctas == 1) __syncthreads();
  else cluster_sync();
}

// The block's list of n <= kList keys, descending.
template <int kThreads>
__device__ __forceinline__ void sort_list(Wide* list, int n) {
  int size = 64;
  while (size < n) size *= 2;
  for (int i = n + threadIdx.x; i < size; i += kThreads) list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      for (int i = threadIdx.x; i < size / 2; i += kThreads) {
        const int a = 2 * i - (i & (j - 1)), b = a + j;
        const Wide x = list[a], y = list[b];
        if ((x < y) == ((a & k) == 0)) {
          list[a] = y;
          list[b] = x;
        }
      }
      if (j > 32 || j == 1) __syncthreads();  // (from 32 down a warp's pairs are its own)
      else __syncwarp();
    }
}

// The scores of one load, with what is no number as -inf and of the two zeros one.
__device__ __forceinline__ float normal(float y) { return fmaxf(y + 0.0f, __int_as_float(0xFF800000)); }
__device__ __forceinline__ void unpack(const uint4& w, float (&y)[4], float) {
  y[0] = normal(__uint_as_float(w.x));
  y[1] = normal(__uint_as_float(w.y));
  y[2] = normal(__uint_as_float(w.z));
  y[3] = normal(__uint_as_float(w.w));
}
__device__ __forceinline__ void unpack(const uint4& w, float (&y)[8], __nv_bfloat16) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = normal(__uint_as_float(u[i] << 16));
    y[2 * i + 1] = normal(__uint_as_float(u[i] & 0xFFFF0000u));
  }
}
__device__ __forceinline__ void unpack(const uint4& w, float (&y)[8], __half) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
    y[2 * i] = normal(f.x);
    y[2 * i + 1] = normal(f.y);
  }
}
// Four bytes of a load: scores where `live` says so, -inf elsewhere.
__device__ __forceinline__ uint32_t word_of(const float* base, bool live) { return live ? __float_as_uint(*base) : 0xFF800000u; }
template <typename T>
__device__ __forceinline__ uint32_t word_of(const T* base, bool live0, bool live1, uint32_t none) {
  const uint32_t lo = live0 ? *reinterpret_cast<const uint16_t*>(base) : none;
  const uint32_t hi = live1 ? *reinterpret_cast<const uint16_t*>(base + 1) : none;
  return lo | (hi << 16);
}

template <typename T, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) sample_kernel(const __grid_constant__ SampleArgs a, int ctas, int held_loads) {
  constexpr int kWarps = kThreads / 32;
  __shared__ Shared<kWarps> s;
  extern __shared__ uint4 s_held[];  // [held_loads][threads]
  constexpr int V = 16 / static_cast<int>(sizeof(T));  // scores a load
  const int rank = ctas == 1 ? 0 : static_cast<int>(blockIdx.x) % ctas;
  const int64_t p = blockIdx.x / ctas;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t begin = a.seg_off ? a.seg_off[p] : p * a.ld;
  const int len = static_cast<int>(a.seg_off ? a.seg_off[p + 1] - begin : a.c);
  const T* row = static_cast<const T*>(a.scores) + begin;
  const ks_sampling set = a.params ? a.params[p] : a.all;
  const float none = __int_as_float(0xFF800000);

  // This CTA's stretch of the row, in places that are counted from the last 16-byte boundary at or before its first score. It
  // is kept in shared memory where it fits, one tile, else read again in every phase, in tiles that are few enough for the
  // sums over their warps' parts to be kept.
  const int shift = static_cast<int>(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
  const T* base = row - shift;
  const int64_t places = static_cast<int64_t>(len) + shift;
  const int64_t chunk = ((places + ctas - 1) / ctas + 32 * V - 1) / (32 * V) * (32 * V);
  const int64_t first = rank * chunk, last = first + chunk < places ? first + chunk : places;
  const int64_t all_loads = first < last ? (last - first + kThreads * V - 1) / (kThreads * V) : 0;
  const bool held = all_loads <= held_loads;
  const int64_t least_loads = (all_loads + kEntries / kWarps - 1) / (kEntries / kWarps);
  const int loads = static_cast<int>(held ? all_loads : least_loads > kHeldLoads ? least_loads : kHeldLoads);
  const int tiles = loads > 0 ? static_cast<int>((all_loads + loads - 1) / loads) : 0;

  auto fetch = [&](int64_t at) KS_INLINE {  // the load of V scores at a place; what lies outside the stretch as -inf
    if (at >= shift && at + V <= last) return __ldg(reinterpret_cast<const uint4*>(base + at));
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t e = at + i * (V / 4);
      const bool live0 = e >= shift && e < last, live1 = e + 1 >= shift && e + 1 < last;
      if constexpr (V == 4) u[i] = word_of(reinterpret_cast<const float*>(base + e), live0);
      else u[i] = word_of(base + e, live0, live1, sizeof(T) == 2 && is_bf16<T> ? 0xFF80u : 0xFC00u);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  };
  // Place of a load: those of a warp are neighbours, and warps follow one another in a tile.
  auto place = [&](int tile, int w, int q) KS_INLINE {
    return first + ((static_cast<int64_t>(tile) * kWarps + w) * loads + q) * (32 * V) + lane * V;
  };
  auto get = [&](int tile, int w, int q) KS_INLINE { return held ? s_held[q * kThreads + w * 32 + lane] : fetch(place(tile, w, q)); };
  auto key_of = [&](int64_t at, float y) KS_INLINE { return make_key(y, static_cast<int>(at - shift)); };
  // f(place, scores) for all loads of this thread
  auto each = [&](auto f) KS_INLINE {
    for (int tile = 0; tile < tiles; ++tile) {
      int64_t at = place(tile, warp, 0);
      uint4 next = get(tile, warp, 0);
#pragma unroll 1
      for (int q = 0; q < loads && at - lane * V < last; ++q, at += 32 * V) {
        float y[V];
        unpack(next, y, T{});
        if (q + 1 < loads) next = get(tile, warp, q + 1);  // on its way while these are worked on
        f(at, y);
      }
    }
  };

  // ---- the best candidate, and the least score that is a number ----
  float top = none, low = __int_as_float(0x7F800000);
  for (int tile = 0; tile < tiles; ++tile)
    for (int q0 = 0; q0 < loads; q0 += 4) {
      uint4 w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q0 + q < loads) w[q] = fetch(place(tile, warp, q0 + q));
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q0 + q >= loads) break;
        if (held) s_held[(q0 + q) * kThreads + threadIdx.x] = w[q];
        float y[V];
        unpack(w[q], y, T{});
#pragma unroll
        for (int v = 0; v < V; ++v) {
          top = fmaxf(top, y[v]);
          low = fminf(low, y[v] > none ? y[v] : low);
        }
      }
    }
  // Temperature 0 is the limit of small ones: the best candidate alone, of several that share its score the first.
  const bool greedy = !(set.temperature > 0.0f);
  Wide best = top > none ? make_key(top, 0) : 0;
  if (greedy && top > none) {
    unsigned at = 0xFFFFFFFFu;
    each([&](int64_t i, const float (&y)[V]) KS_INLINE {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (y[v] == top) at = min(at, static_cast<unsigned>(i + v - shift));
    });
    best = make_key(top, static_cast<int>(at));
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) {
    const Wide u = __shfl_xor_sync(0xFFFFFFFFu, best, d);
    best = u > best ? u : best;
    low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, d));
  }
  if (lane == 0) {
    s.warp[warp] = best;
    s.least[warp] = low;
  }
  __syncthreads();
  if (warp == 0) {
    best = lane < kWarps ? s.warp[lane] : 0;
    low = lane < kWarps ? s.least[lane] : low;
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
      const Wide u = __shfl_xor_sync(0xFFFFFFFFu, best, d);
      best = u > best ? u : best;
      low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, d));
    }
    if (lane == 0) {
      s.best = best;
      s.min = low;
      s.listed = 0;
    }
  }
  for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = s.low[i] = s.high[i] = 0;
  meet(ctas);
  best = 0;
  for (int r = 0; r < ctas; ++r) {
    const Wide u = *of_rank(&s.best, r, ctas);
    best = u > best ? u : best;
    low = fminf(low, *of_rank(&s.min, r, ctas));
  }
  if (best == 0) {  // nothing has weight
    if (rank == 0)
      for (int i = threadIdx.x; i < a.draws; i += kThreads) {
        a.idx[p * a.draws + i] = -1;
        if (a.logp) a.logp[p * a.draws + i] = none;
      }
    meet(ctas);  // (its results are read by the others)
    return;
  }

  Row r;
  r.best = key_score(best);
  r.best_wide = static_cast<double>(r.best);
  r.steps = greedy ? 0.0 : 64.0 * 1.4426950408889634074 / static_cast<double>(set.temperature);
  r.one = ldexp(1.0, min(51, __clzll(static_cast<long long>(len)) - 2));  // sums of all weights fit 63 bits
  r.least = set.min_p > 0.0f ? fmin(static_cast<double>(set.min_p), 1.0) * r.one : 0.0;
  r.reach = greedy ? 0.0f : (kReach + 1.0f) * set.temperature;
  // bins over what the scores reach, but no further than weights do
  const float span = fminf(r.best - low, kReach * set.temperature);
  r.bins = span > 0.0f ? static_cast<float>(kBins - 1) / span : 0.0f;
  if (threadIdx.x < 64) s.table[threadIdx.x] = exp2(threadIdx.x / 64.0) * r.one;
  __syncthreads();
  // what stays: scores above `cut_score`, and those that equal it up to the place `cut_at`
  Wide cut = greedy ? best : 0;
  // (without a branch: what lies behind the reach of weights, -inf above all, computes something and gets 0)
  auto weight = [&](float y) KS_INLINE {
    const Wide w = whole(scaled_weight(r, s.table, y));
    return r.best - y > r.reach ? 0ull : w;
  };

  // ---- cuts ----
  bool counted = false;  // the histogram over all candidates is there, over the cluster
  const int mine = kBins / ctas, per = (mine + kThreads - 1) / kThreads;  // bins of this CTA, and of a thread
  const unsigned* m_count = ctas == 1 ? s.count : s.m_count;
  auto m_sum = [&](int i) KS_INLINE { return ctas == 1 ? (static_cast<Wide>(s.high[i]) << 32) + s.low[i] : s.m_sum[i]; };
  // histogram of the candidates that `digit` gives a bin (-1: none), and this CTA's share of it over the cluster
  auto histogram = [&](bool clear, auto digit) KS_INLINE {
    if (clear) {
      for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = s.low[i] = s.high[i] = 0;
      __syncthreads();
    }
    each([&](int64_t i, const float (&y)[V]) KS_INLINE {
      Wide w[V];
#pragma unroll
      for (int v = 0; v < V; ++v) w[v] = weight(y[v]);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int d = digit(i + v, y[v]);
        if (w[v] == 0 || d < 0) continue;
        atomicAdd(&s.count[d], 1u);
        // 64 bits in two additions of 32: who sees the low one wrap carries
        const unsigned add = static_cast<unsigned>(w[v]), was = atomicAdd(&s.low[d], add);
        const unsigned up = static_cast<unsigned>(w[v] >> 32) + (was + add < was ? 1u : 0u);
        if (up) atomicAdd(&s.high[d], up);
      }
    });
    meet(ctas);
    Wide c = 0, w = 0;
    if (ctas > 1)
      for (int i = threadIdx.x; i < mine; i += kThreads) {
        unsigned bc = 0;
        Wide bw = 0;
        for (int o = 0; o < ctas; ++o) {
          bc += *of_rank(&s.count[rank * mine + i], o, ctas);
          bw += (static_cast<Wide>(*of_rank(&s.high[rank * mine + i], o, ctas)) << 32) + *of_rank(&s.low[rank * mine + i], o, ctas);
        }
        s.m_count[i] = bc;
        s.m_sum[i] = bw;
        c += bc;
        w += bw;
      }
    else
      for (int i = threadIdx.x; i < mine; i += kThreads) {
        c += m_count[i];
        w += m_sum(i);
      }
    Wide total_c, total_w;
    block_scan2(c, w, s.warp2, total_c, total_w);
    if (threadIdx.x == 0) {
      s.share_count = total_c;
      s.share_sum = total_w;
    }
    meet(ctas);
  };
  // The front of `n` candidates (n > 0), or else the shortest whose weights sum to `part` of `of` (0: of all), as a cut; the
  // sum of its weights, 0 where nothing is cut.
  auto find_cut = [&](Wide n, double part, Wide of) KS_INLINE -> Wide {
    const Wide outer = cut;  // what an earlier cut leaves
    if (!counted) {
      histogram(false, [&](int64_t, float y) KS_INLINE { return bin_of(r, y); });
      counted = true;
    }
    Wide base_count = 0, base_sum = 0, prefix = 0;
    int bin0 = 0, owner = 0;
    double target = 0.0;
    for (int level = 0;; ++level) {
      // the CTA whose share of the bins holds the last candidate that stays
      Wide c = base_count, w = base_sum, own_c = 0, own_w = 0, all_c = 0, all_w = 0;
      for (int o = 0; o < ctas; ++o) {
        all_c += *of_rank(&s.share_count, o, ctas);
        all_w += *of_rank(&s.share_sum, o, ctas);
      }
      if (level == 0) {
        target = fmax(part * static_cast<double>(of > 0 ? of : all_w), 1.0);  // (weights are whole numbers: the best one stays)
        if (n > 0 ? all_c <= n : static_cast<double>(of > 0 ? of : all_w) <= target) {
          meet(ctas);
          return 0;
        }
      }
      owner = ctas - 1;
      for (int o = 0; o < ctas; ++o) {
        own_c = c;
        own_w = w;
        c += *of_rank(&s.share_count, o, ctas);
        w += *of_rank(&s.share_sum, o, ctas);
        if (n > 0 ? c >= n : static_cast<double>(w) >= target) {
          owner = o;
          break;
        }
      }
      if (rank == owner) {
        Wide bc = 0, bw = 0, total_c, total_w;
        for (int q = 0; q < per; ++q) {
          const int i = threadIdx.x * per + q;
          if (i < mine) {
            bc += m_count[i];
            bw += m_sum(i);
          }
        }
        block_scan2(bc, bw, s.warp2, total_c, total_w);
        bc += own_c;
        bw += own_w;
        for (int q = 0; q < per; ++q) {
          const int i = threadIdx.x * per + q;
          if (i >= mine) break;
          const bool starts = n > 0 ? bc < n : static_cast<double>(bw) < target;
          const bool ends = n > 0 ? bc + m_count[i] >= n : static_cast<double>(bw + m_sum(i)) >= target;
          if (m_count[i] > 0 && starts && ends) {
            s.bin = rank * mine + i;
            s.held = m_count[i];
            s.before_count = bc;
            s.before_sum = bw;
          }
          bc += m_count[i];
          bw += m_sum(i);
        }
      }
      meet(ctas);
      const int bin = *of_rank(&s.bin, owner, ctas);
      const unsigned held = *of_rank(&s.held, owner, ctas);
      base_count = *of_rank(&s.before_count, owner, ctas);
      base_sum = *of_rank(&s.before_sum, owner, ctas);
      const int shift_now = 64 - kDigit * level;  // of the digits that are fixed
      if (level == 0) bin0 = bin;
      else prefix |= static_cast<Wide>(kBins - 1 - bin) << (shift_now > 0 ? shift_now : 0);
      auto member = [&](Wide key, float y) KS_INLINE {
        return bin_of(r, y) == bin0 && key >= outer && (level == 0 || (key >> (shift_now > 0 ? shift_now : 0)) == (prefix >> (shift_now > 0 ? shift_now : 0)));
      };
      if (held <= kList) {
        unsigned* n_list = of_rank(&s.listed, owner, ctas);
        Wide* list = of_rank(&s.list[0], owner, ctas);
        each([&](int64_t i, const float (&y)[V]) KS_INLINE {
#pragma unroll
          for (int v = 0; v < V; ++v) {
            if (bin_of(r, y[v]) != bin0) continue;
            const Wide key = key_of(i + v, y[v]);
            if (member(key, y[v]) && weight(y[v]) > 0) list[atomicAdd(n_list, 1u)] = key;
          }
        });
        meet(ctas);
        if (rank == owner) {
          const int n_held = static_cast<int>(s.listed);
          sort_list<kThreads>(s.list, n_held);
          constexpr int kEach = kList / kThreads;
          Wide w2[kEach], sum2 = 0, total;
#pragma unroll
          for (int q = 0; q < kEach; ++q) {
            const int i = threadIdx.x * kEach + q;
            w2[q] = i < n_held ? weight(key_score(s.list[i])) : 0;
            sum2 += w2[q];
          }
          Wide bw = block_scan(sum2, s.warp, total) + base_sum;
#pragma unroll
          for (int q = 0; q < kEach; ++q) {
            const int i = threadIdx.x * kEach + q;
            if (i < n_held && (n > 0 ? base_count + i + 1 == n
                                     : static_cast<double>(bw) < target && (static_cast<double>(bw + w2[q]) >= target || i + 1 == n_held))) {
              s.cut = s.list[i];
              s.cut_sum = bw + w2[q];
            }
            bw += w2[q];
          }
          if (threadIdx.x == 0) s.listed = 0;
        }
        meet(ctas);
        cut = *of_rank(&s.cut, owner, ctas);
        return *of_rank(&s.cut_sum, owner, ctas);
      }
      // too many to sort: by the next bits of (score, index)
      counted = false;
      const int next = shift_now - kDigit > 0 ? shift_now - kDigit : 0;
      const int width = shift_now - next;
      histogram(true, [&](int64_t i, float y) KS_INLINE {
        const Wide key = key_of(i, y);
        if (!member(key, y)) return -1;
        return kBins - 1 - static_cast<int>((key >> next) & ((1u << width) - 1));
      });
    }
  };
  if (!greedy) {
    const Wide sum = set.top_k > 0 ? find_cut(static_cast<Wide>(set.top_k), 1.0, 0) : 0;
    if (set.top_p < 1.0f) {  // of what top-k leaves
      if (sum > 0 && !counted) {  // (narrowed down: the histogram is that of one bin)
        const Wide outer = cut;
        histogram(true, [&](int64_t i, float y) KS_INLINE { return key_of(i, y) >= outer ? bin_of(r, y) : -1; });
        counted = true;
      }
      find_cut(0, fmax(static_cast<double>(set.top_p), 0.0), sum);
    }
  }

  // ---- the sum of what stays, then the draws, in the order of the indices ----
  const float cut_score = cut > 0 ? key_score(cut) : none;
  const unsigned cut_at = cut > 0 ? static_cast<unsigned>(key_index(cut)) : 0xFFFFFFFFu;
  auto stays = [&](int64_t i, float y) KS_INLINE -> Wide {
    const bool in = y > cut_score || (y == cut_score && static_cast<unsigned>(i - shift) <= cut_at);
    const double w = scaled_weight(r, s.table, y);
    return in && !(r.best - y > r.reach) && (greedy || w >= r.least) ? (greedy ? 1ull : whole(w)) : 0ull;
  };
  const int entries = tiles * kWarps;  // a tile's parts by warp, in the order of the indices
  __syncthreads();  // (the list is read)
  for (int tile = 0; tile < tiles; ++tile) {
    Wide own = 0;
    int64_t at = place(tile, warp, 0);
    uint4 next = get(tile, warp, 0);
#pragma unroll 1
    for (int q = 0; q < loads && at - lane * V < last; ++q, at += 32 * V) {
      float y[V];
      unpack(next, y, T{});
      if (q + 1 < loads) next = get(tile, warp, q + 1);
      // (where a cut leaves nothing of a warp's scores there is nothing to compute)
      float most = y[0];
#pragma unroll
      for (int v = 1; v < V; ++v) most = fmaxf(most, y[v]);
      if (!__any_sync(0xFFFFFFFFu, most >= cut_score && most > none)) continue;
#pragma unroll
      for (int v = 0; v < V; ++v) own += stays(at + v, y[v]);
    }
    own = warp_sum(own);
    if (lane == 0) s.list[tile * kWarps + warp] = own;
  }
  __syncthreads();
  {  // sums up to an entry's end
    const int per_thread = (entries + kThreads - 1) / kThreads;
    Wide own = 0, total;
    for (int e = 0; e < per_thread; ++e)
      if (static_cast<int>(threadIdx.x) * per_thread + e < entries) own += s.list[threadIdx.x * per_thread + e];
    Wide upto = block_scan(own, s.warp, total);
    for (int e = 0; e < per_thread; ++e)
      if (static_cast<int>(threadIdx.x) * per_thread + e < entries) s.list[threadIdx.x * per_thread + e] = upto += s.list[threadIdx.x * per_thread + e];
    if (threadIdx.x == 0) s.total = total;
  }
  meet(ctas);
  Wide all = 0, before = 0;
  for (int o = 0; o < ctas; ++o) {
    const Wide t = *of_rank(&s.total, o, ctas);
    if (o < rank) before += t;
    all += t;
  }
  for (int q_draw = warp; q_draw < a.draws; q_draw += kWarps) {
    const float u = a.u[p * a.draws + q_draw];
    Wide target = static_cast<Wide>(static_cast<double>(u > 0.0f ? u : 0.0f) * static_cast<double>(all));
    if (u >= 1.0f || target >= all) target = all - 1;
    if (target < before || target - before >= s.total) continue;
    target -= before;
    int lo = 0, hi = entries - 1;  // the first entry whose end is behind the target
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (s.list[mid] > target) hi = mid;
      else lo = mid + 1;
    }
    target -= lo > 0 ? s.list[lo - 1] : 0;
    const int tile = lo / kWarps, w_slot = lo % kWarps;
#pragma unroll 1
    for (int q = 0; q < loads; ++q) {
      float y[V];
      unpack(get(tile, w_slot, q), y, T{});
      const int64_t i0 = place(tile, w_slot, q);
      Wide w[V], own = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        w[v] = stays(i0 + v, y[v]);
        own += w[v];
      }
      const Wide row_total = warp_sum(own);
      if (target >= row_total) {
        target -= row_total;
        continue;
      }
      Wide from = warp_scan(own, lane) - own;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (target >= from && target < from + w[v]) {
          a.idx[p * a.draws + q_draw] = static_cast<int32_t>(i0 + v - shift);
          if (a.logp) {
            const double d = y[v] == r.best ? 0.0 : (static_cast<double>(y[v]) - r.best_wide) / static_cast<double>(set.temperature);
            a.logp[p * a.draws + q_draw] = static_cast<float>(d - log(static_cast<double>(all) / (greedy ? 1.0 : r.one)));
          }
        }
        from += w[v];
      }
      break;
    }
  }
  meet(ctas);  // (its sum is read by the others)
}

template <typename T, int kThreads>
cudaError_t launch_as(const SampleArgs& a, int ctas, int held_loads, cudaStream_t stream) {
  const void* kernel = reinterpret_cast<const void*>(&sample_kernel<T, kThreads>);
  cudaError_t e = ensure_dynamic_smem(kernel, kHeldLoads * kThreads * 16);
  if (e == cudaSuccess && ctas > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(a.p * ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(held_loads) * kThreads * 16;
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = static_cast<unsigned>(ctas);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T, kThreads>, a, ctas, held_loads);
}

constexpr int kManyThreads = 256, kFewThreads = 512;
constexpr int64_t kManyRows = 296;

template <typename T>
cudaError_t launch_type(const SampleArgs& a, cudaStream_t stream) {
  constexpr int64_t kV = 16 / sizeof(T);
  const int64_t len = std::max<int64_t>(1, a.seg_off ? a.c / a.p : a.c);  // (of segments the mean)
  // (a stretch is rounded up to whole warps' loads and may begin within one; four CTAs an SM keep 28 KB each)
  if (a.p >= kManyRows) {
    const int64_t loads = (2 * len + 64 * kV + kManyThreads * kV - 1) / (kManyThreads * kV);
    return launch_as<T, kManyThreads>(a, 1, static_cast<int>(len > 7 * kManyThreads * kV ? 0 : std::min<int64_t>(7, loads)), stream);
  }
  int ctas = 1;
  while (ctas < kMaxCtas && kFewThreads * kV * kHeldLoads * ctas < len) ctas *= 2;
  // few rows: more CTAs each, while they have a thousand scores and more
  while (ctas < kMaxCtas && a.p * ctas * 2 <= 148 && len / (2 * ctas) >= 1024) ctas *= 2;
  if (a.p * ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  const int64_t each = (a.seg_off ? 2 * len : len + ctas - 1) / ctas + 64 * kV;
  const int64_t loads = std::min<int64_t>(kHeldLoads, (each + kFewThreads * kV - 1) / (kFewThreads * kV));
  return launch_as<T, kFewThreads>(a, ctas, static_cast<int>(loads), stream);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, int score_type, cudaStream_t stream, int64_t* launches) {
  ++*launches;
  switch (score_type) {
    case KS_F32: return launch_type<float>(a, stream);
    case KS_BF16: return launch_type<__nv_bfloat16>(a, stream);
    default: return launch_type<__half>(a, stream);
  }
}

}  // namespace ks
