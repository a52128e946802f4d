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
// The sums of weights that top-p's histogram needs are first estimated in 32 bits; one pass with the weights themselves then
// sums up what lies surely in front of the cut and lists the candidates of the few bins around it, which are sorted. Bins that
// hold more than a list are estimated again in 1,024 bins of their own (64 x 500,000 scores: 659 us without, 257 so). Where
// the estimate was not good enough, or candidates share a score, the exact histogram is made.
//
// A short front (top-k of some hundred) needs no histogram: the k-th largest of the maxima of 128 parts of the row bounds the
// k-th score from below, so that little more than k candidates are listed, sorted, cut, and drawn from in the list.
//
// A row of a call with few rows belongs to a cluster of up to 16 CTAs, each with a stretch of it; their results meet in shared
// memory. Where there are rows for the whole machine a CTA takes a row by itself. Stretches that fit are kept in shared memory
// (short rows by four CTAs an SM), others read again in every phase by two CTAs an SM, which is what stays in L2. Rows of up to
// 256 scores belong to a warp each (short_rows_kernel).
//
// What bounds it: instructions. 1,024 x 60,000 fp32 scores with top-p take 357 us where reading them takes 38: three passes, of
// which the one with the weights (20 operations in 64 bits and the sums) takes half; the issue slots are 66 % busy, the fp64
// pipe 12 %. With top-k 50 110 us, without cuts 195. The phases are one kernel of 64 registers a thread, for 1,024 threads an SM, which
// spills (fp32 scores 88 bytes of stores and 120 of loads, 16-bit ones 312 and 572). Few rows are bound by the phases' latency: one of
// 60,000 scores 12 us with top-k, 29 with top-p.
#include <algorithm>
#include <cmath>
#include <type_traits>

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
constexpr int kParts = 128;        // of a CTA's scores, whose maxima bound a short front
constexpr int kShort = 512, kShortParts = 112;  // the longest front that is drawn from a list, and its share of a CTA's parts
constexpr int kHeldLoads = 8;      // 16-byte loads that a thread keeps at most
constexpr int kShortRow = 256;     // scores of a row that a warp takes
constexpr int kEntries = 1024;     // sums over stretches of a row that a CTA keeps
constexpr float kReach = 36.05f;   // (best - x) / t behind which every weight rounds to 0 (51 bits)
constexpr int kTable = 256;        // powers of two within one octave
constexpr int kDigit = 10;         // bits of (score, index) that a bin is narrowed down by

struct Row {
  float best;
  float reach;        // scores further below the best one have no weight
  float bins;         // bins a unit of score
  double best_wide;
  double steps;       // 256ths of a power of two a unit of score
  double one;         // weight of the best score, 2^s
  double least;       // weights below do not stay (min-p)
};

// Weight of a score within reach in units of 2^-s, before it is rounded: 2^(n / 256) from a table of 256 (times 2^s) and the
// exponent, times the exponential of what is left, at most ln 2 / 512, by its series (P. T. P. Tang's table-driven method, ACM
// TOMS 15, 1989). The first term that is left out is below 2^-54. The best score's weight is exact, also where it is infinite.
template <typename Table>
__device__ __forceinline__ double scaled_weight(const Row& r, const Table& table, float x) {
  constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: adding it rounds to a whole number in the low word
  constexpr double kL = 0.69314718055994530942 / kTable;
  const double z = (static_cast<double>(x) - r.best_wide) * r.steps, m = z + kRound;
  const int n = __double2loint(m);
  const double f = z - (m - kRound);
  double e = fma(f, kL * kL * kL * kL / 24.0, kL * kL * kL / 6.0);
  e = fma(f, e, kL * kL / 2.0);
  e = fma(f, e, kL);
  e = fma(f, e, 1.0);
  const double w = table[n & (kTable - 1)] * e;
  const double v = __hiloint2double(__double2hiint(w) + ((n >> 8) << 20), __double2loint(w));
  return x == r.best ? r.one : v;
}
__device__ __forceinline__ Row row_of(const ks_sampling& set, bool greedy, float best, int len) {
  Row r;
  r.best = best;
  r.best_wide = static_cast<double>(best);
  r.steps = greedy ? 0.0 : kTable * 1.4426950408889634074 / static_cast<double>(set.temperature);
  r.one = ldexp(1.0, min(51, __clzll(static_cast<long long>(len)) - 2));  // sums of all weights fit 63 bits
  r.least = set.min_p > 0.0f ? fmin(static_cast<double>(set.min_p), 1.0) * r.one : 0.0;
  // (finite, so that it leaves out -inf at any temperature)
  r.reach = greedy ? 0.0f : fminf((kReach + 1.0f) * set.temperature, 3.402823466e38f);
  r.bins = 0.0f;
  return r;
}
__device__ __forceinline__ double power(int i, double one) { return exp2(static_cast<double>(i) / kTable) * one; }
// rounded; w <= 2^51, so that the sum's low bits are the whole number
__device__ __forceinline__ Wide whole(double w) {
  return static_cast<Wide>(__double_as_longlong(w + 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
}

// (adding 2^23 rounds to a whole number in the low bits)
__device__ __forceinline__ int bin_of(const Row& r, float x) {
  return static_cast<int>(__float_as_uint(fminf((r.best - x) * r.bins, static_cast<float>(kBins - 1)) + 8388608.0f) & (kBins - 1));
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

template <int kWarps>
struct Shared {
  double table[kTable];
  alignas(16) unsigned low[kBins], high[kBins];  // of a bin's count or sum
  Wide merged[kBins / 2];            // this CTA's share of the bins, over the cluster
  Wide list[kList];
  Wide warp[kWarps];
  // what the cluster's other CTAs read
  Wide best;
  float least[kWarps], min, bound;
  alignas(16) float part[kParts];
  Wide share, before, total, cut, front, window[2];
  int bin, first_bin, last_bin;
  unsigned listed;
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

// Bitonic sorts, descending. Of a warp's keys, E neighbours a lane:
template <int E, typename Key>
__device__ __forceinline__ void sort_warp(Key (&x)[E], int lane) {
#pragma unroll
  for (int k = 2; k <= 32 * E; k *= 2)
#pragma unroll
    for (int j = k / 2; j > 0; j /= 2)
#pragma unroll
      for (int q = 0; q < E; ++q) {
        const int at = lane * E + q;
        const bool down = (at & k) == 0;
        if (j >= E) {
          const Key y = __shfl_xor_sync(0xFFFFFFFFu, x[q], j / E);
          if (((at & j) == 0) == down == (y > x[q])) x[q] = y;
        } else if ((q & j) == 0) {
          const Key u = x[q], v = x[q | j];
          if ((u < v) == down) {
            x[q] = v;
            x[q | j] = u;
          }
        }
      }
}
template <int E>
__device__ __forceinline__ void sort_short(Wide* list, int n) {
  Wide x[E];
#pragma unroll
  for (int q = 0; q < E; ++q) x[q] = static_cast<int>(threadIdx.x) * E + q < n ? list[threadIdx.x * E + q] : 0;
  sort_warp<E>(x, threadIdx.x);
#pragma unroll
  for (int q = 0; q < E; ++q) list[threadIdx.x * E + q] = x[q];
}
// Of a block's `size` keys (a power of two) by the warps that have some, partners in other warps through `list`.
template <int E>
__device__ __forceinline__ void sort_long(Wide* list, int n, int size) {
  Wide x[E];
  const int first = threadIdx.x * E;
  const bool mine = first < size;
#pragma unroll
  for (int q = 0; q < E; ++q) x[q] = first + q < n ? list[first + q] : 0;
#pragma unroll 1
  for (int k = 2; k <= size; k *= 2) {
#pragma unroll 1
    for (int j = k / 2; j >= E; j /= 2) {
      const bool far = j >= 32 * E;
      if (far) {
        __syncthreads();
        if (mine)
#pragma unroll
          for (int q = 0; q < E; ++q) list[first + q] = x[q];
        __syncthreads();
      }
      if (mine)
#pragma unroll
        for (int q = 0; q < E; ++q) {
          const int at = first + q;
          const Wide y = far ? list[at ^ j] : __shfl_xor_sync(0xFFFFFFFFu, x[q], j / E);
          if (((at & j) == 0) == ((at & k) == 0) == (y > x[q])) x[q] = y;
        }
    }
#pragma unroll
    for (int j = E / 2; j > 0; j /= 2)
      if (j < k)
#pragma unroll
        for (int q = 0; q < E; ++q)
          if ((q & j) == 0) {
            const Wide u = x[q], v = x[q | j];
            if ((u < v) == (((first + q) & k) == 0)) {
              x[q] = v;
              x[q | j] = u;
            }
          }
  }
  __syncthreads();
  if (mine)
#pragma unroll
    for (int q = 0; q < E; ++q) list[first + q] = x[q];
}
// The block's list of n <= kList keys. Up to 128 by one warp: the others' turns at the loops of a sort that they have no part in
// took most of its time (22 keys: 6,100 clocks by all, about 1,100 by one).
template <int kThreads>
__device__ __noinline__ void sort_list(Wide* list, int n) {
  __syncthreads();
  if (n <= 128) {
    if (threadIdx.x < 32) {
      if (n <= 32) sort_short<1>(list, n);
      else if (n <= 64) sort_short<2>(list, n);
      else sort_short<4>(list, n);
    }
  } else if (n <= 256) {
    sort_long<1>(list, n, 256);
  } else if (n <= 512) {
    sort_long<512 / kThreads>(list, n, 512);
  } else {
    sort_long<kList / kThreads>(list, n, kList);
  }
  __syncthreads();
}

// The scores of one load, with what is no number as -inf and of the two zeros one.
__device__ __forceinline__ float normal(float y) { return fmaxf(y + 0.0f, __int_as_float(0xFF800000)); }
template <typename T, int V>
__device__ __forceinline__ void unpack_as_is(const uint4& w, float (&y)[V]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (V == 4) {
      y[i] = __uint_as_float(u[i]);
    } else if constexpr (is_bf16<T>) {
      y[2 * i] = __uint_as_float(u[i] << 16);
      y[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
      y[2 * i] = f.x;
      y[2 * i + 1] = f.y;
    }
  }
}
template <typename T, int V>
__device__ __forceinline__ void unpack(const uint4& w, float (&y)[V]) {
  unpack_as_is<T, V>(w, y);
#pragma unroll
  for (int v = 0; v < V; ++v) y[v] = normal(y[v]);
}
// The load of scores at a place of which some lie outside [shift, last): those as -inf.
template <typename T>
__device__ __noinline__ uint4 fetch_edge(const T* base, uint32_t at, uint32_t shift, uint32_t last) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      const uint32_t e = at + i;
      u[i] = e >= shift && e < last ? __float_as_uint(base[e]) : 0xFF800000u;
    } else {
      constexpr uint32_t kNone = is_bf16<T> ? 0xFF80u : 0xFC00u;
      const uint32_t e = at + 2 * i;
      const uint32_t lo = e >= shift && e < last ? *reinterpret_cast<const uint16_t*>(base + e) : kNone;
      const uint32_t hi = e + 1 >= shift && e + 1 < last ? *reinterpret_cast<const uint16_t*>(base + e + 1) : kNone;
      u[i] = lo | (hi << 16);
    }
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// ---- short rows ----

struct Powers {
  double one;
  __device__ __forceinline__ double operator[](int i) const { return power(i, one); }
};

// A row of up to 32 * E scores by one warp, without a barrier, E neighbours a lane: the best one, the cuts from a sorted copy where
// there are cuts, the sums up to each score, which are searched. The same weights and sums as sample_kernel's, so the same draws.
template <typename T, int E>
__device__ __noinline__ void short_row(const SampleArgs& a, int64_t p, const T* row, int len, const ks_sampling& set, Wide* upto) {
  const int lane = threadIdx.x % 32, first = lane * E;
  const float none = __int_as_float(0xFF800000);
  auto place = [](int i) KS_INLINE { return i + i / E; };  // (no two lanes' in one bank)
  float y[E];
  Wide best = 0;
#pragma unroll
  for (int q = 0; q < E; ++q) y[q] = first + q < len ? normal(to_float(row[first + q])) : none;
  auto key = [&](int q) KS_INLINE -> Wide { return y[q] > none ? make_key(y[q], first + q) : 0; };
#pragma unroll
  for (int q = 0; q < E; ++q) best = max(best, key(q));
#pragma unroll
  for (int d = 16; d > 0; d /= 2) best = max(best, __shfl_xor_sync(0xFFFFFFFFu, best, d));
  if (best == 0) {  // nothing has weight
    for (int q = lane; q < a.draws; q += 32) {
      a.idx[p * a.draws + q] = -1;
      if (a.logp) a.logp[p * a.draws + q] = none;
    }
    return;
  }
  const bool greedy = !(set.temperature > 0.0f);
  const Row r = row_of(set, greedy, key_score(best), len);
  const Powers powers{r.one};
  Wide cut = greedy ? best : 0;  // what stays has this key or a larger one
  const bool some = set.top_k > 0 && set.top_k < len, front = set.top_p < 1.0f;
  if (!greedy && (some || front)) {
    Wide x[E];
#pragma unroll
    for (int q = 0; q < E; ++q) x[q] = key(q);
    sort_warp<E>(x, lane);
    if (some) {
      Wide mine = 0;
#pragma unroll
      for (int q = 0; q < E; ++q)
        if (q == (set.top_k - 1) % E) mine = x[q];
      cut = __shfl_sync(0xFFFFFFFFu, mine, (set.top_k - 1) / E);
    }
    if (front) {
      Wide w[E], sum = 0;
#pragma unroll
      for (int q = 0; q < E; ++q) {
        const float v = key_score(x[q]);
        w[q] = x[q] < cut || r.best - v > r.reach ? 0 : whole(scaled_weight(r, powers, v));
        sum += w[q];
      }
      const Wide end = warp_scan(sum, lane), total = __shfl_sync(0xFFFFFFFFu, end, 31);
      const Wide target = max(1ull, static_cast<Wide>(ceil(fmax(static_cast<double>(set.top_p), 0.0) * static_cast<double>(total))));
      Wide before = end - sum, last = 0;
#pragma unroll
      for (int q = 0; q < E; ++q) {
        if (before < target && before + w[q] >= target) last = x[q];
        before += w[q];
      }
      const unsigned who = __ballot_sync(0xFFFFFFFFu, last > 0);
      if (who) cut = __shfl_sync(0xFFFFFFFFu, last, __ffs(who) - 1);
    }
  }
  Wide w[E], sum = 0;
#pragma unroll
  for (int q = 0; q < E; ++q) {
    const double exact = scaled_weight(r, powers, y[q]);
    const bool stays = key(q) >= cut && !(r.best - y[q] > r.reach) && (greedy || exact >= r.least);
    w[q] = stays ? greedy ? 1 : whole(exact) : 0;
    sum += w[q];
  }
  Wide end = warp_scan(sum, lane);
  const Wide all = __shfl_sync(0xFFFFFFFFu, end, 31);
  end -= sum;
#pragma unroll
  for (int q = 0; q < E; ++q) upto[place(first + q)] = end += w[q];
  __syncwarp();
  for (int q = lane; q < a.draws; q += 32) {
    const float u = a.u[p * a.draws + q];
    Wide goal = static_cast<Wide>(static_cast<double>(u > 0.0f ? u : 0.0f) * static_cast<double>(all));
    if (u >= 1.0f || goal >= all) goal = all - 1;
    int lo = 0;  // the first whose end is behind the goal
#pragma unroll
    for (int step = 16 * E; step > 0; step /= 2)
      if (upto[place(lo + step - 1)] <= goal) lo += step;
    a.idx[p * a.draws + q] = lo;
    if (a.logp) {
      const float v = normal(to_float(row[lo]));
      const double d = v == r.best ? 0.0 : (static_cast<double>(v) - r.best_wide) / static_cast<double>(set.temperature);
      a.logp[p * a.draws + q] = static_cast<float>(d - log(static_cast<double>(all) / (greedy ? 1.0 : r.one)));
    }
  }
}

constexpr int kShortWarps = 4;
constexpr int kShortPlaces = kShortRow + 32;
// Rows of up to kShortRow scores by a warp each; others are left.
template <typename T>
__global__ void __launch_bounds__(32 * kShortWarps) short_rows_kernel(const __grid_constant__ SampleArgs a) {
  static_assert(kShortRow == 32 * 8, "the longest row has eight scores a lane");
  __shared__ Wide s[kShortWarps][kShortPlaces];
  next_may_start();
  wait_for_last();
  const int64_t p = static_cast<int64_t>(blockIdx.x) * kShortWarps + threadIdx.x / 32;
  if (p >= a.p) return;
  const int64_t begin = a.seg_off ? a.seg_off[p] : p * a.ld;
  const int64_t scores = a.seg_off ? a.seg_off[p + 1] - begin : a.c;
  if (scores > kShortRow) return;
  const int len = static_cast<int>(scores);
  const T* row = static_cast<const T*>(a.scores) + begin;
  const ks_sampling set = a.params ? a.params[p] : a.all;
  Wide* mine = s[threadIdx.x / 32];
  if (len <= 32) short_row<T, 1>(a, p, row, len, set, mine);
  else if (len <= 64) short_row<T, 2>(a, p, row, len, set, mine);
  else if (len <= 128) short_row<T, 4>(a, p, row, len, set, mine);
  else short_row<T, 8>(a, p, row, len, set, mine);
}

template <typename T, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) sample_kernel(const __grid_constant__ SampleArgs a, int ctas, int held_loads, int done) {
  constexpr int kWarps = kThreads / 32;
  __shared__ Shared<kWarps> s;
  extern __shared__ uint4 s_held[];  // [held_loads][threads]
  constexpr int V = 16 / static_cast<int>(sizeof(T));  // scores a load
  next_may_start();
  wait_for_last();
  const int rank = ctas == 1 ? 0 : static_cast<int>(blockIdx.x) % ctas;
  const int64_t p = blockIdx.x / ctas;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t begin = a.seg_off ? a.seg_off[p] : p * a.ld;
  const int len = static_cast<int>(a.seg_off ? max(a.seg_off[p + 1] - begin, static_cast<int64_t>(0)) : a.c);
  const T* row = static_cast<const T*>(a.scores) + begin;
  const ks_sampling set = a.params ? a.params[p] : a.all;
  const float none = __int_as_float(0xFF800000);
  if (len <= done) return;  // (a short row, drawn from by short_rows_kernel)

  // This CTA's stretch of the row, in places that are counted from the last 16-byte boundary at or before its first score. It
  // is kept in shared memory where it fits, one tile, else read again in every phase, in tiles that are few enough for the
  // sums over their warps' parts to be kept.
  const int shift = static_cast<int>(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
  const T* base = row - shift;
  // (a row has less than 2^31 scores: places fit 32 bits)
  const uint32_t places = static_cast<uint32_t>(len) + shift;
  const uint32_t chunk = (places / ctas + 32 * V) / (32 * V) * (32 * V);
  const uint64_t begin_at = static_cast<uint64_t>(rank) * chunk;
  const uint32_t first = begin_at < places ? static_cast<uint32_t>(begin_at) : places;
  const uint32_t last = chunk < places - first ? first + chunk : places;
  const uint32_t all_loads = (last - first + kThreads * V - 1) / (kThreads * V);
  const bool held = all_loads <= static_cast<uint32_t>(held_loads);
  const uint32_t least_loads = (all_loads + kEntries / kWarps - 1) / (kEntries / kWarps);
  const int loads = static_cast<int>(held ? all_loads : least_loads > kHeldLoads ? least_loads : kHeldLoads);
  const int tiles = loads > 0 ? static_cast<int>((all_loads + loads - 1) / loads) : 0;
  // loads at places from `shift` to here lie inside
  const uint32_t inner = last >= static_cast<uint32_t>(shift) + V ? last - shift - V + 1 : 0;

  auto fetch = [&](uint32_t at) KS_INLINE {
    return at - shift < inner ? *reinterpret_cast<const uint4*>(base + at) : fetch_edge(base, at, shift, last);
  };
  // Place of a load: those of a warp are neighbours, and warps follow one another in a tile.
  auto place = [&](int tile, int w, int q) KS_INLINE {
    return first + ((static_cast<uint32_t>(tile) * kWarps + w) * loads + q) * (32 * V) + lane * V;
  };
  auto get = [&](uint32_t at, int w, int q) KS_INLINE { return held ? s_held[q * kThreads + w * 32 + lane] : fetch(at); };
  auto key_of = [&](uint32_t at, float y) KS_INLINE { return make_key(y, static_cast<int>(at - shift)); };
  // f(place, scores) for all loads of this thread, as they are or with what is no number as -inf
  auto each_load = [&](auto as_is, auto f) KS_INLINE {
    for (int tile = 0; tile < tiles; ++tile) {
      uint32_t at = place(tile, warp, 0);
      const uint32_t lane0 = at - lane * V;
      if (lane0 >= last) break;
      const int mine = min(loads, static_cast<int>((last - lane0 + 32 * V - 1) / (32 * V)));
      uint4 next = get(at, warp, 0);
#pragma unroll 1
      for (int q = 0; q < mine; ++q, at += 32 * V) {
        float y[V];
        if constexpr (decltype(as_is)::value) unpack_as_is<T, V>(next, y);
        else unpack<T, V>(next, y);
        if (q + 1 < mine) next = get(at + 32 * V, warp, q + 1);  // on its way while these are worked on
        f(at, y);
      }
    }
  };
  auto each = [&](auto f) KS_INLINE { each_load(std::false_type{}, f); };

  // ---- the best candidate, and the least score that is a number ----
  float top = none, low = __int_as_float(0x7F800000);
  for (int tile = 0; tile < tiles; ++tile)
    for (int q0 = 0; q0 < loads; q0 += 4) {
      const uint32_t at = place(tile, warp, q0);
      uint4 w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q0 + q < loads) w[q] = fetch(at + q * (32 * V));
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q0 + q >= loads) break;
        if (held) s_held[(q0 + q) * kThreads + threadIdx.x] = w[q];
        float y[V];
        unpack<T, V>(w[q], y);
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
    each([&](uint32_t i, const float (&y)[V]) KS_INLINE {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (y[v] == top) at = min(at, i + v - shift);
    });
    best = make_key(top, static_cast<int>(at));
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) {
    const Wide u = __shfl_xor_sync(0xFFFFFFFFu, best, d);
    best = u > best ? u : best;
    low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, d));
  }
  // the maxima of the parts, and the one that as many of them reach as the CTA's share of a short front has candidates
  const int share = (min(set.top_k, kShort) + ctas - 1) / ctas;
  const bool short_front = !greedy && set.top_k > 0 && set.top_k <= kShort && share <= kShortParts;
  if (short_front) {
    constexpr int kEach = kThreads / kParts;
    float most = top;
#pragma unroll
    for (int d = 1; d < kEach; d *= 2) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
    if (threadIdx.x % kEach == 0) s.part[threadIdx.x / kEach] = most;
  }
  if (lane == 0) {
    s.warp[warp] = best;
    s.least[warp] = low;
  }
  __syncthreads();
  if (short_front && warp == 1) {
    static_assert(kParts == 4 * 32, "four parts a lane");
    const float4 f = *reinterpret_cast<const float4*>(&s.part[4 * lane]);
    float x[4] = {f.x, f.y, f.z, f.w};
    sort_warp<4>(x, lane);
    const int at = share - 1;
    if (lane == at / 4) s.bound = at % 4 == 0 ? x[0] : at % 4 == 1 ? x[1] : at % 4 == 2 ? x[2] : x[3];
  }
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

  Row r = row_of(set, greedy, key_score(best), len);
  // bins over what the scores reach, but no further than weights do
  const float span = fminf(r.best - low, kReach * set.temperature);
  r.bins = span > 0.0f ? static_cast<float>(kBins - 1) / span : 0.0f;
  if (threadIdx.x < kTable) s.table[threadIdx.x] = power(threadIdx.x, r.one);
  __syncthreads();
  // ---- a short front ----
  if (short_front) {
    float bound = __int_as_float(0x7F800000);
    for (int o = 0; o < ctas; ++o) bound = fminf(bound, *of_rank(&s.bound, o, ctas));
    unsigned* n_list = of_rank(&s.listed, 0, ctas);
    Wide* list = of_rank(&s.list[0], 0, ctas);
    each([&](uint32_t i, const float (&y)[V]) KS_INLINE {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!(y[v] >= bound) || !(y[v] > none)) continue;
        const unsigned at = atomicAdd(n_list, 1u);
        if (at < kList) list[at] = key_of(i + v, y[v]);
      }
    });
    meet(ctas);
    const unsigned listed = *n_list;
    if (listed <= kList) {
      if (rank == 0) {
        const int n = min(static_cast<int>(listed), set.top_k);
        sort_list<kThreads>(s.list, static_cast<int>(listed));
        constexpr int kEach = kShort / kThreads;
        Wide w[kEach], sum = 0, all;
        bool enough[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int i = threadIdx.x * kEach + e;
          const float y = key_score(i < n ? s.list[i] : best);
          const double exact = scaled_weight(r, s.table, y);
          enough[e] = exact >= r.least;
          w[e] = i < n && !(r.best - y > r.reach) ? whole(exact) : 0;
          sum += w[e];
        }
        Wide b = block_scan(sum, s.warp, all);
        const Wide target = set.top_p < 1.0f ? max(1ull, static_cast<Wide>(ceil(fmax(static_cast<double>(set.top_p), 0.0) * static_cast<double>(all)))) : all;
        Wide place_of[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int i = threadIdx.x * kEach + e;
          const bool in = w[e] > 0 && b < target && enough[e];
          b += w[e];
          if (i < kShort) s.merged[i] = in ? w[e] : 0;
          place_of[e] = in ? ~((static_cast<Wide>(static_cast<unsigned>(key_index(s.list[i]))) << 32) | static_cast<unsigned>(i)) : 0;
        }
        // the weights that each candidate has, in the order of the indices
        Wide* scores = reinterpret_cast<Wide*>(s.low);  // (kept by place in the sorted front)
#pragma unroll
        for (int e = 0; e < kEach; ++e) scores[threadIdx.x * kEach + e] = threadIdx.x * kEach + e < n ? s.list[threadIdx.x * kEach + e] : 0;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kEach; ++e) s.list[threadIdx.x * kEach + e] = place_of[e];
        __syncthreads();
        sort_list<kThreads>(s.list, n);
        sum = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int i = threadIdx.x * kEach + e;
          const Wide key = i < n ? s.list[i] : 0;
          w[e] = key > 0 ? s.merged[static_cast<unsigned>(~key)] : 0;
          sum += w[e];
        }
        Wide upto = block_scan(sum, s.warp, all);
        Wide* ends = reinterpret_cast<Wide*>(s.low) + kShort;
#pragma unroll
        for (int e = 0; e < kEach; ++e) ends[threadIdx.x * kEach + e] = upto += w[e];
        __syncthreads();
        for (int q = threadIdx.x; q < a.draws; q += kThreads) {
          const float u = a.u[p * a.draws + q];
          Wide goal = static_cast<Wide>(static_cast<double>(u > 0.0f ? u : 0.0f) * static_cast<double>(all));
          if (u >= 1.0f || goal >= all) goal = all - 1;
          int lo = 0, hi = n - 1;  // the first whose end is behind the goal
          while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (ends[mid] > goal) hi = mid;
            else lo = mid + 1;
          }
          const Wide key = scores[static_cast<unsigned>(~s.list[lo])];
          const float y = key_score(key);
          a.idx[p * a.draws + q] = key_index(key);
          if (a.logp) {
            const double d = y == r.best ? 0.0 : (static_cast<double>(y) - r.best_wide) / static_cast<double>(set.temperature);
            a.logp[p * a.draws + q] = static_cast<float>(d - log(static_cast<double>(all) / r.one));
          }
        }
      }
      meet(ctas);  // (the number is read by the others)
      return;
    }
    meet(ctas);  // (the number is read)
  }

  // what stays: scores above `cut_score`, and of those that equal it the ones up to `cut_at`
  float cut_score = greedy ? r.best : none;
  unsigned cut_at = greedy ? static_cast<unsigned>(key_index(best)) : 0xFFFFFFFFu;
  auto inside = [&](uint32_t i, float y) KS_INLINE {
    return y > cut_score || (y == cut_score && i - shift <= cut_at);
  };
  // (without a branch: what lies behind the reach of weights, -inf above all, computes something and gets 0)
  auto weight = [&](float y) KS_INLINE {
    const Wide w = whole(scaled_weight(r, s.table, y));
    return r.best - y > r.reach ? 0ull : w;
  };

  // ---- cuts ----
  const int mine = kBins / ctas, per = (mine + kThreads - 1) / kThreads;  // bins of this CTA, and of a thread
  auto bin_sum = [&](int i) KS_INLINE { return ctas == 1 ? (static_cast<Wide>(s.high[i]) << 32) + s.low[i] : s.merged[i]; };
  // Leaves the shortest front of what stays that holds `part` of its candidates' sum, or (`counts`) `n` candidates; the cut is
  // the first candidate in the order up to which the bins, then the sorted ones of a bin, reach that.
  auto find_cut = [&](auto counts, Wide n, double part) KS_INLINE {
    constexpr bool kCounts = decltype(counts)::value;
    Wide before = 0, target = n, prefix = 0;
    int bin0 = 0;
    for (int level = 0;; ++level) {
      const int fixed = level == 0 ? 64 : max(0, 64 - kDigit * (level - 1));  // bits of (score, index) above are `prefix`'s
      const int next = max(0, fixed - kDigit);
      auto member = [&](Wide key, float y) KS_INLINE {
        return level == 0 || (bin_of(r, y) == bin0 && (level == 1 || (key >> fixed) == (prefix >> fixed)));
      };
      for (int i = threadIdx.x; i < kBins; i += kThreads) s.low[i] = s.high[i] = 0;
      if (threadIdx.x == 0) s.listed = 0;
      __syncthreads();
      each([&](uint32_t i, const float (&y)[V]) KS_INLINE {
        bool in[V];
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = y[v] > none;
        if (cut_score > none) {  // (where an earlier cut leaves nothing of a warp's scores there is nothing to compute)
          bool any = false;
#pragma unroll
          for (int v = 0; v < V; ++v) {
            in[v] = inside(i + v, y[v]);
            any = any || in[v];
          }
          if (!__any_sync(0xFFFFFFFFu, any)) return;
        }
        Wide w[V];
        int bin[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          w[v] = kCounts ? 1ull : weight(y[v]);
          bin[v] = bin_of(r, y[v]);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (!in[v]) continue;
          int d = bin[v];
          if (level > 0) {
            const Wide key = key_of(i + v, y[v]);
            if (!member(key, y[v])) continue;
            d = kBins - 1 - static_cast<int>((key >> next) & ((1u << (fixed - next)) - 1));
          }
          // 64 bits in two additions of 32: who sees the low one wrap carries
          const unsigned add = static_cast<unsigned>(w[v]), was = atomicAdd(&s.low[d], add);
          if (!kCounts) {
            const unsigned up = static_cast<unsigned>(w[v] >> 32) + (was + add < was ? 1u : 0u);
            if (up) atomicAdd(&s.high[d], up);
          }
        }
      });
      meet(ctas);
      Wide own = 0, share;
      for (int i = threadIdx.x; i < mine; i += kThreads) {
        Wide b = 0;
        if (ctas == 1) {
          b = bin_sum(i);
        } else {
          for (int o = 0; o < ctas; ++o)
            b += (static_cast<Wide>(*of_rank(&s.high[rank * mine + i], o, ctas)) << 32) + *of_rank(&s.low[rank * mine + i], o, ctas);
          s.merged[i] = b;
        }
        own += b;
      }
      block_scan(own, s.warp, share);
      if (threadIdx.x == 0) s.share = share;
      meet(ctas);
      // the CTA whose share of the bins holds the last candidate that stays
      Wide reached = before, own_before = before;
      int owner = -1;
      for (int o = 0; o < ctas; ++o) {
        const Wide next_share = *of_rank(&s.share, o, ctas);
        if (level == 0) own_before += next_share;  // (the sum of all)
      }
      if (level == 0) {
        const Wide all = own_before;
        if (!kCounts) target = max(1ull, static_cast<Wide>(ceil(part * static_cast<double>(all))));
        if (all <= target) {
          meet(ctas);
          return;
        }
      }
      for (int o = 0; o < ctas && owner < 0; ++o) {
        own_before = reached;
        reached += *of_rank(&s.share, o, ctas);
        if (reached >= target) owner = o;
      }
      if (rank == owner) {
        Wide mine_sum = 0, total;
        for (int q = 0; q < per; ++q)
          if (static_cast<int>(threadIdx.x) * per + q < mine) mine_sum += bin_sum(threadIdx.x * per + q);
        Wide b = block_scan(mine_sum, s.warp, total) + own_before;
        for (int q = 0; q < per && static_cast<int>(threadIdx.x) * per + q < mine; ++q) {
          const int i = threadIdx.x * per + q;
          const Wide e = b + bin_sum(i);
          if (b < target && e >= target) {
            s.bin = rank * mine + i;
            s.before = b;
          }
          b = e;
        }
      }
      meet(ctas);
      const int bin = *of_rank(&s.bin, owner, ctas);
      before = *of_rank(&s.before, owner, ctas);
      if (level == 0) bin0 = bin;
      else prefix |= static_cast<Wide>(kBins - 1 - bin) << next;
      // the bin's candidates, if they are few enough to be sorted
      const int fixed_now = level == 0 ? 64 : next;
      unsigned* n_list = of_rank(&s.listed, owner, ctas);
      Wide* list = of_rank(&s.list[0], owner, ctas);
      each([&](uint32_t i, const float (&y)[V]) KS_INLINE {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (bin_of(r, y[v]) != bin0 || !(y[v] > none)) continue;
          const Wide key = key_of(i + v, y[v]);
          if (!inside(i + v, y[v]) || (level > 0 && (key >> fixed_now) != (prefix >> fixed_now))) continue;
          if (!kCounts && weight(y[v]) == 0) continue;
          const unsigned at = atomicAdd(n_list, 1u);
          if (at < kList) list[at] = key;
        }
      });
      meet(ctas);
      const unsigned listed = *n_list;
      if (listed > kList) {  // too many: by the next bits of (score, index)
        meet(ctas);  // (the number is read)
        continue;
      }
      if (rank == owner) {
        sort_list<kThreads>(s.list, static_cast<int>(listed));
        constexpr int kEach = kList / kThreads;
        Wide w[kEach], sum = 0, total;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
          const unsigned i = threadIdx.x * kEach + q;
          w[q] = i >= listed ? 0 : kCounts ? 1 : weight(key_score(s.list[i]));
          sum += w[q];
        }
        Wide b = block_scan(sum, s.warp, total) + before;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
          if (b < target && b + w[q] >= target) s.cut = s.list[threadIdx.x * kEach + q];
          b += w[q];
        }
      }
      meet(ctas);
      const Wide cut = *of_rank(&s.cut, owner, ctas);
      cut_score = key_score(cut);
      cut_at = static_cast<unsigned>(key_index(cut));
      return;
    }
  };
  Wide* ends = s.list;   // sums of the stretches of this CTA, then up to their ends
  bool summed = false;   // they are there
  // The cut of top-p by an estimate; false: it did not serve.
  auto estimated_cut = [&](double part) KS_INLINE -> bool {
    const float octaves = 1.4426950408889634f / set.temperature;
    const bool cuts = cut_score > none;  // an earlier cut leaves some
    // The bins [first0, last0] of the first histogram, where they hold more candidates than can be listed, in bins of their own.
    bool fine = false;
    int first0 = 0, last0 = 0;
    float origin = 0.0f, scale = 0.0f;
    auto fine_bin = [&](float y, int d) KS_INLINE {
      const float f = fminf(fmaxf((r.best - y - origin) * scale, 0.0f), static_cast<float>(kBins - 1));
      return d < first0 ? -1 : d > last0 ? kBins : static_cast<int>(f);
    };
    Wide all = 0, base = 0;
    int first_bin = -1, last_bin = -1;
    for (;;) {
      for (int i = threadIdx.x; i < kBins; i += kThreads) s.low[i] = s.high[i] = 0;
      if (threadIdx.x == 0) s.listed = 0;
      __syncthreads();
      auto estimate = [&](auto is_fine) KS_INLINE {
        each_load(std::true_type{}, [&](uint32_t i, const float (&y)[V]) KS_INLINE {
          unsigned add[V];
          int d[V];
#pragma unroll
          for (int v = 0; v < V; ++v) {
            // The weight times 2^30 (with 2^22, which needs no conversion, 16-bit scores that share a value are all rounded the same
            // way, and the estimate failed for one row in 20). The relative error of 53 octaves in fp32 is below 2^-18. What is no
            // number, or -inf, adds 0.
            const float below = y[v] - r.best;
            float w;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(below * octaves));
            add[v] = __float2uint_rn(w * 1073741824.0f);
            d[v] = __float_as_uint(fminf(-below * r.bins, static_cast<float>(kBins - 1)) + 8388608.0f) & (kBins - 1);
          }
          if (cuts)
#pragma unroll
            for (int v = 0; v < V; ++v)
              if (!inside(i + v, y[v])) add[v] = 0;
          if constexpr (decltype(is_fine)::value) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
              d[v] = fine_bin(y[v], d[v]);
              if (d[v] < 0 || d[v] >= kBins) add[v] = 0;
            }
          }
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (add[v] > 0) {
              const unsigned was = atomicAdd(&s.low[d[v]], add[v]);
              if (was + add[v] < was) atomicAdd(&s.high[d[v]], 1u);
            }
        });
      };
      if (fine) estimate(std::true_type{});
      else estimate(std::false_type{});
      meet(ctas);
      Wide own = 0, share;
      for (int i = threadIdx.x; i < mine; i += kThreads) {
        Wide b = 0;
        if (ctas == 1) {
          b = bin_sum(i);
        } else {
          for (int o = 0; o < ctas; ++o)
            b += (static_cast<Wide>(*of_rank(&s.high[rank * mine + i], o, ctas)) << 32) + *of_rank(&s.low[rank * mine + i], o, ctas);
          s.merged[i] = b;
        }
        own += b;
      }
      block_scan(own, s.warp, share);
      if (threadIdx.x == 0) s.share = share;
      meet(ctas);
      Wide before = base;
      for (int o = 0; o < ctas; ++o) {
        const Wide t = *of_rank(&s.share, o, ctas);
        if (o < rank) before += t;
        if (!fine) all += t;
      }
      // the bins in which the sum reaches a little less and a little more than the part
      const double goal = part * static_cast<double>(all);
      const Wide least = static_cast<Wide>(goal * (1.0 - 1.0 / 8192)), most = min(all, static_cast<Wide>(goal * (1.0 + 1.0 / 8192)) + 1);
      if (threadIdx.x == 0) s.first_bin = s.last_bin = -1;
      Wide mine_sum = 0, total;
      for (int q = 0; q < per; ++q)
        if (static_cast<int>(threadIdx.x) * per + q < mine) mine_sum += bin_sum(threadIdx.x * per + q);
      Wide b = block_scan(mine_sum, s.warp, total) + before;
      for (int q = 0; q < per && static_cast<int>(threadIdx.x) * per + q < mine; ++q) {
        const int i = threadIdx.x * per + q;
        const Wide e = b + bin_sum(i);
        if (b <= least && e > least) {
          s.first_bin = rank * mine + i;
          if (!fine) s.window[0] = b;
        }
        if (b < most && e >= most) {
          s.last_bin = rank * mine + i;
          if (!fine) s.window[1] = e;
        }
        b = e;
      }
      meet(ctas);
      first_bin = last_bin = -1;
      Wide up_to = 0;
      for (int o = 0; o < ctas; ++o) {
        const int f = *of_rank(&s.first_bin, o, ctas), l = *of_rank(&s.last_bin, o, ctas);
        first_bin = max(first_bin, f);
        last_bin = max(last_bin, l);
        if (!fine && f >= 0) base = *of_rank(&s.window[0], o, ctas);
        if (!fine && l >= 0) up_to = *of_rank(&s.window[1], o, ctas);
      }
      if (first_bin < 0 || last_bin < 0) {  // (all threads find the same)
        meet(ctas);
        return false;
      }
      // no more candidates than their sum has of the least of their weights (the last bin has no end)
      const float end = (static_cast<float>(last_bin) + 0.5f) / r.bins, lightest = exp2f(-end * octaves) * 1073741824.0f;
      if (fine || last_bin == kBins - 1 || static_cast<float>(up_to - base) <= kList * lightest) break;
      fine = true;
      first0 = first_bin;
      last0 = last_bin;
      origin = (static_cast<float>(first_bin) - 0.5f) / r.bins;
      scale = kBins * r.bins / static_cast<float>(last_bin - first_bin + 1);
    }
    // the weights: of all, of what lies in front of those bins (by stretches what min-p lets stay), and who lies in them
    unsigned* n_list = of_rank(&s.listed, 0, ctas);
    Wide* list = of_rank(&s.list[0], 0, ctas);
    ends = reinterpret_cast<Wide*>(s.low);
    const bool least_counts = r.least > 0.0;
    Wide sum = 0, front = 0;
    auto weigh = [&](auto is_fine) KS_INLINE {
      for (int tile = 0; tile < tiles; ++tile) {
        Wide stretch = 0;
        uint32_t at = place(tile, warp, 0);
        const uint32_t lane0 = at - lane * V;
        const int steps = lane0 >= last ? 0 : min(loads, static_cast<int>((last - lane0 + 32 * V - 1) / (32 * V)));
        uint4 next = make_uint4(0, 0, 0, 0);
        if (steps > 0) next = get(at, warp, 0);
#pragma unroll 1
        for (int q = 0; q < steps; ++q, at += 32 * V) {
          float y[V];
          unpack_as_is<T, V>(next, y);
          if (q + 1 < steps) next = get(at + 32 * V, warp, q + 1);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const double exact = scaled_weight(r, s.table, y[v]);
            bool in = r.best - y[v] <= r.reach;  // (not so of what is no number)
            if (cuts) in = in && inside(at + v, y[v]);
            const Wide w = in ? whole(exact) : 0;
            int bin = bin_of(r, y[v]);
            if constexpr (decltype(is_fine)::value) bin = fine_bin(y[v], bin);
            sum += w;
            if (bin < first_bin) {
              if (!least_counts) stretch += w;
              else front += w, stretch += exact >= r.least ? w : 0;
            } else if (bin <= last_bin && w > 0) {
              const unsigned to = atomicAdd(n_list, 1u);
              if (to < kList) list[to] = key_of(at + v, normal(y[v]));
            }
          }
        }
        if (!least_counts) front += stretch;
        stretch = warp_sum(stretch);
        if (lane == 0) ends[tile * kWarps + warp] = stretch;
      }
    };
    if (fine) weigh(std::true_type{});
    else weigh(std::false_type{});
    Wide block_sum, block_front;
    block_scan(sum, s.warp, block_sum);
    block_scan(front, s.warp, block_front);
    if (threadIdx.x == 0) {
      s.share = block_sum;
      s.front = block_front;
      s.cut = 0;
    }
    meet(ctas);
    const unsigned listed = *n_list;
    if (rank == 0) {
      all = front = 0;
      for (int o = 0; o < ctas; ++o) {
        all += *of_rank(&s.share, o, ctas);
        front += *of_rank(&s.front, o, ctas);
      }
      const Wide target = max(1ull, static_cast<Wide>(ceil(part * static_cast<double>(all))));
      if (listed <= kList && front < target) {
        sort_list<kThreads>(s.list, static_cast<int>(listed));
        constexpr int kEach = kList / kThreads;
        Wide w[kEach];
        sum = 0;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
          const unsigned i = threadIdx.x * kEach + q;
          w[q] = i >= listed ? 0 : weight(key_score(s.list[i]));
          sum += w[q];
        }
        Wide total, e = block_scan(sum, s.warp, total) + front;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
          if (e < target && e + w[q] >= target) s.cut = s.list[threadIdx.x * kEach + q];
          e += w[q];
        }
      }
    }
    meet(ctas);
    const Wide cut = *of_rank(&s.cut, 0, ctas);
    if (cut == 0) {
      ends = s.list;
      meet(ctas);  // (it is read)
      return false;
    }
    cut_score = key_score(cut);
    cut_at = static_cast<unsigned>(key_index(cut));
    // of the candidates listed those that stay belong to stretches too
    for (unsigned i = threadIdx.x; i < listed; i += kThreads) {
      const Wide key = list[i];
      const uint32_t at = static_cast<uint32_t>(key_index(key)) + shift;
      if (key < cut || at < first || at >= last) continue;
      const double exact = scaled_weight(r, s.table, key_score(key));
      if (exact >= r.least) atomicAdd(&ends[(at - first) / (32 * V) / loads], whole(exact));
    }
    __syncthreads();
    summed = true;
    return true;
  };
  if (!greedy && set.top_k > 0) find_cut(std::true_type{}, static_cast<Wide>(set.top_k), 0.0);
  if (!greedy && set.top_p < 1.0f) {
    const double part = fmax(static_cast<double>(set.top_p), 0.0);
    // (an infinite score's distance to itself is no number: the estimate is for others)
    if (!(r.best < __int_as_float(0x7F800000)) || !estimated_cut(part)) find_cut(std::false_type{}, 0, part);
  }

  // ---- the sum of what stays, then the draws, in the order of the indices ----
  auto stays = [&](uint32_t i, float y) KS_INLINE -> Wide {
    const double w = scaled_weight(r, s.table, y);
    return inside(i, y) && !(r.best - y > r.reach) && (greedy || w >= r.least) ? (greedy ? 1ull : whole(w)) : 0ull;
  };
  const int entries = tiles * kWarps;  // a tile's parts by warp, in the order of the indices
  __syncthreads();  // (the list is read)
  for (int tile = 0; tile < tiles && !summed; ++tile) {
    Wide own = 0;
    uint32_t at = place(tile, warp, 0);
    const uint32_t lane0 = at - lane * V;
    const int mine = lane0 >= last ? 0 : min(loads, static_cast<int>((last - lane0 + 32 * V - 1) / (32 * V)));
    uint4 next = make_uint4(0, 0, 0, 0);
    if (mine > 0) next = get(at, warp, 0);
#pragma unroll 1
    for (int q = 0; q < mine; ++q, at += 32 * V) {
      float y[V];
      unpack<T, V>(next, y);
      if (q + 1 < mine) next = get(at + 32 * V, warp, q + 1);
      // (where a cut leaves nothing of a warp's scores there is nothing to compute)
      float most = y[0];
#pragma unroll
      for (int v = 1; v < V; ++v) most = fmaxf(most, y[v]);
      if (!__any_sync(0xFFFFFFFFu, most >= cut_score && most > none)) continue;
#pragma unroll
      for (int v = 0; v < V; ++v) own += stays(at + v, y[v]);
    }
    own = warp_sum(own);
    if (lane == 0) ends[tile * kWarps + warp] = own;
  }
  __syncthreads();
  {  // sums up to an entry's end
    const int per_thread = (entries + kThreads - 1) / kThreads;
    Wide own = 0, total;
    for (int e = 0; e < per_thread; ++e)
      if (static_cast<int>(threadIdx.x) * per_thread + e < entries) own += ends[threadIdx.x * per_thread + e];
    Wide upto = block_scan(own, s.warp, total);
    for (int e = 0; e < per_thread; ++e)
      if (static_cast<int>(threadIdx.x) * per_thread + e < entries) ends[threadIdx.x * per_thread + e] = upto += ends[threadIdx.x * per_thread + e];
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
      if (ends[mid] > target) hi = mid;
      else lo = mid + 1;
    }
    target -= lo > 0 ? ends[lo - 1] : 0;
    const int tile = lo / kWarps, w_slot = lo % kWarps;
#pragma unroll 1
    for (int q = 0; q < loads; ++q) {
      float y[V];
      const uint32_t i0 = place(tile, w_slot, q);
      unpack<T, V>(get(i0, w_slot, q), y);
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
cudaError_t launch_as(const SampleArgs& a, int ctas, int held_loads, int done, cudaStream_t stream) {
  const void* kernel = reinterpret_cast<const void*>(&sample_kernel<T, kThreads>);
  cudaError_t e = ensure_dynamic_smem(kernel, kHeldLoads * kThreads * 16);
  if (e == cudaSuccess && ctas > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  return launch_following(&sample_kernel<T, kThreads>, dim3(static_cast<unsigned>(a.p * ctas)), kThreads,
                          static_cast<size_t>(held_loads) * kThreads * 16, ctas, stream, a, ctas, held_loads, done);
}

constexpr int kSmall = 256, kLarge = 512;  // threads of a CTA
constexpr int64_t kManyRows = 296;

template <typename T>
cudaError_t launch_type(const SampleArgs& a, cudaStream_t stream, int64_t* launches) {
  constexpr int64_t kV = 16 / sizeof(T);
  const int64_t len = std::max<int64_t>(1, a.seg_off ? a.c / a.p : a.c);  // (of segments the mean)
  // Short rows by a warp each: all of a call, or those of many segments or of segments that are short on the average, in a launch of
  // their own (4,096 rows of 32 scores with top-k: 60 us by CTAs, 6 by warps; of 256 scores 60 and 26. Warps of the other
  // kernel's CTAs instead of a launch: no gain, its code grows). Of segments the offsets alone say how long they are, and a replayed
  // graph may find others than the call was made with: both kernels follow, whatever their total is said to be.
  const bool all_short = !a.seg_off && a.c <= kShortRow, some_short = a.seg_off && (a.p >= kManyRows || len <= kShortRow);
  if (all_short || some_short) {
    if (a.p > INT32_MAX) return cudaErrorInvalidConfiguration;
    const cudaError_t e = launch_following(&short_rows_kernel<T>, dim3(static_cast<unsigned>((a.p + kShortWarps - 1) / kShortWarps)),
                                           32 * kShortWarps, 0, 0, stream, a);
    ++*launches;
    if (e != cudaSuccess || all_short) return e;
  }
  const int done = some_short ? kShortRow : -1;
  ++*launches;
  if (a.p >= kManyRows) {
    // rows that four CTAs an SM keep (28 KB each; segments are of all lengths), else what is in work at a time stays in L2
    constexpr int64_t kKept = 7;
    if (len <= kKept * kSmall * kV)
      return launch_as<T, kSmall>(a, 1, static_cast<int>(a.seg_off ? kKept : std::min(kKept, (len + 64 * kV) / (kSmall * kV) + 1)), done, stream);
    return launch_as<T, kLarge>(a, 1, 0, done, stream);
  }
  // Few rows: a cluster each, while all of its CTAs can run at once (two an SM; clusters of 16 on half of that) and have 5,000 scores and
  // more. 64 x 131,072 fp32 scores, top-p: 81 us by 4 CTAs a row, 123 by 8, in two waves, that keep their scores; 290 x 60,000: 104 by
  // one, 138 by 2, 213 by 4; 8 x 8,192, top-k: 10 by one, 11 by 2 or 4, 20 by 8.
  int ctas = 1;
  while (ctas < kMaxCtas && a.p * ctas * 2 <= (ctas < 8 ? 296 : 148) && len / (2 * ctas) >= 5000) ctas *= 2;
  const int64_t each = (a.seg_off ? 2 * len : len + ctas - 1) / ctas + 64 * kV;
  int64_t loads = (each + kLarge * kV - 1) / (kLarge * kV);
  if (loads > kHeldLoads) loads = a.seg_off ? kHeldLoads : 0;
  return launch_as<T, kLarge>(a, ctas, static_cast<int>(loads), done, stream);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, int score_type, cudaStream_t stream, int64_t* launches) {
  switch (score_type) {
    case KS_F32: return launch_type<float>(a, stream, launches);
    case KS_BF16: return launch_type<__nv_bfloat16>(a, stream, launches);
    default: return launch_type<__half>(a, stream, launches);
  }
}

}  // namespace ks
