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
// A row belongs to a cluster of 1 to 16 CTAs that keep its scores in shared memory, each thread its own (rows longer than the
// cluster holds are read again in every phase), so that a row is read from memory once. The CTAs' results meet there too.
#include <algorithm>
#include <cmath>

#include "ks_e4m3.cuh"
#include "ks_internal.h"
#include "ks_tcgen.cuh"
#include "ks_topk.cuh"

namespace ks {
namespace {

using Wide = unsigned long long;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kList = 1024;        // candidates of a bin that are sorted
constexpr int kMaxCtas = 16;       // of a cluster
constexpr int kLoads = 8;          // 16-byte loads that a thread keeps: two CTAs an SM
constexpr float kReach = 36.05f;   // (best - x) / t behind which every weight rounds to 0 (51 bits)
constexpr int kDigit = 11;         // bits of (score, index) that a bin is narrowed down by

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
__device__ __forceinline__ Wide block_scan(Wide v, Wide* s_warp, Wide& total) {
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
__device__ __forceinline__ void block_scan2(Wide& v, Wide& w, Wide (*s_warp)[kWarps], Wide& total_v, Wide& total_w) {
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
      if (j > 32 || j == 1) __syncthreads();
      else __syncwarp();
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleArgs a, int ctas, int loads) {
  __shared__ Shared s;
  extern __shared__ uint4 s_held[];  // [loads][threads]
  constexpr int V = 16 / static_cast<int>(sizeof(T));  // scores a load
  const int rank = ctas == 1 ? 0 : static_cast<int>(blockIdx.x) % ctas;
  const int64_t p = blockIdx.x / ctas;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t begin = a.seg_off ? a.seg_off[p] : p * a.ld;
  const int len = static_cast<int>(a.seg_off ? a.seg_off[p + 1] - begin : a.c);
  const T* row = static_cast<const T*>(a.scores) + begin;
  const ks_sampling set = a.params ? a.params[p] : a.all;
  const float none = __int_as_float(0xFF800000);

  // This CTA's stretch of the row, in places that are counted from the last 16-byte boundary at or before its first score.
  const int shift = static_cast<int>(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
  const T* base = row - shift;
  const int64_t places = static_cast<int64_t>(len) + shift;
  const int64_t chunk = ((places + ctas - 1) / ctas + 32 * V - 1) / (32 * V) * (32 * V);
  const int64_t first = rank * chunk, last = first + chunk < places ? first + chunk : places;
  const int held = kThreads * V * loads;
  const int tiles = first < last ? static_cast<int>((last - first + held - 1) / held) : 0;

  // The V scores from a place of this CTA's on; what lies outside its stretch, and what is no number, as -inf, and of the two
  // zeros one.
  auto fetch = [&](int64_t at) {
    uint4 w;
    T t[V];
    if (at >= shift && at + V <= last) {
      w = __ldg(reinterpret_cast<const uint4*>(base + at));
      memcpy(t, &w, 16);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) t[v] = at + v >= shift && at + v < last ? base[at + v] : from_float<T>(none);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float y = to_float(t[v]) + 0.0f;
      t[v] = from_float<T>(y == y ? y : none);
    }
    memcpy(&w, t, 16);
    return w;
  };
  auto score = [&](const uint4& w, int v) {
    T t[V];
    memcpy(t, &w, 16);
    return to_float(t[v]);
  };
  // Place of a thread's load in a tile: the loads of a warp are neighbours, and warps follow one another.
  auto place = [&](int tile, int q) { return first + static_cast<int64_t>(tile) * held + (static_cast<int64_t>(warp) * loads + q) * (32 * V) + lane * V; };
  auto get = [&](int tile, int q) { return tiles == 1 ? s_held[q * kThreads + threadIdx.x] : fetch(place(tile, q)); };
  auto key_of = [&](int64_t at, float y) { return make_key(y, static_cast<int>(at - shift)); };
  // f(place, score) for all scores of this thread that are not -inf
  auto each = [&](auto f) {
    for (int tile = 0; tile < tiles; ++tile)
#pragma unroll 1
      for (int q = 0; q < loads; ++q) {
        const int64_t at = place(tile, q);
        if (at - lane * V >= last) break;
        const uint4 w = get(tile, q);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float y = score(w, v);
          if (y > none) f(at + v, y);
        }
      }
  };

  // ---- the best candidate, and the least score that is a number ----
  float top = none, low = __int_as_float(0x7F800000);
  for (int tile = 0; tile < tiles; ++tile) {
    uint4 w[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q)
      if (q < loads) w[q] = fetch(place(tile, q));
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      if (q >= loads) break;
      if (tiles == 1) s_held[q * kThreads + threadIdx.x] = w[q];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float y = score(w[q], v);
        top = fmaxf(top, y);
        if (y > none) low = fminf(low, y);
      }
    }
  }
  // Temperature 0 is the limit of small ones: the best candidate alone, of several that share its score the first.
  const bool greedy = !(set.temperature > 0.0f);
  Wide best = top > none ? make_key(top, 0) : 0;
  if (greedy && top > none) {
    unsigned at = 0xFFFFFFFFu;
    each([&](int64_t i, float y) {
      if (y == top) at = min(at, static_cast<unsigned>(i - shift));
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
  auto weight = [&](float y) { return whole(scaled_weight(r, s.table, y)); };

  // ---- cuts ----
  bool counted = false;  // the histogram over all candidates is there, over the cluster
  const int mine = kBins / ctas, per = (mine + kThreads - 1) / kThreads;  // bins of this CTA, and of a thread
  const unsigned* m_count = ctas == 1 ? s.count : s.m_count;
  auto m_sum = [&](int i) { return ctas == 1 ? (static_cast<Wide>(s.high[i]) << 32) + s.low[i] : s.m_sum[i]; };
  // histogram of the candidates that `digit` gives a bin (-1: none), and this CTA's share of it over the cluster
  auto histogram = [&](bool clear, auto digit) {
    if (clear) {
      for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = s.low[i] = s.high[i] = 0;
      __syncthreads();
    }
    each([&](int64_t i, float y) {
      if (r.best - y > r.reach) return;
      const Wide w = weight(y);
      if (w == 0) return;
      const int d = digit(i, y);
      if (d < 0) return;
      atomicAdd(&s.count[d], 1u);
      // 64 bits in two additions of 32: who sees the low one wrap carries
      const unsigned add = static_cast<unsigned>(w), was = atomicAdd(&s.low[d], add);
      const unsigned up = static_cast<unsigned>(w >> 32) + (was + add < was ? 1u : 0u);
      if (up) atomicAdd(&s.high[d], up);
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
  auto find_cut = [&](Wide n, double part, Wide of) -> Wide {
    const Wide outer = cut;  // what an earlier cut leaves
    if (!counted) {
      histogram(false, [&](int64_t, float y) { return bin_of(r, y); });
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
      auto member = [&](Wide key, float y) {
        return bin_of(r, y) == bin0 && key >= outer && (level == 0 || (key >> (shift_now > 0 ? shift_now : 0)) == (prefix >> (shift_now > 0 ? shift_now : 0)));
      };
      if (held <= kList) {
        unsigned* n_list = of_rank(&s.listed, owner, ctas);
        Wide* list = of_rank(&s.list[0], owner, ctas);
        each([&](int64_t i, float y) {
          const Wide key = key_of(i, y);
          if (!member(key, y) || r.best - y > r.reach || weight(y) == 0) return;
          list[atomicAdd(n_list, 1u)] = key;
        });
        meet(ctas);
        if (rank == owner) {
          const int n_held = static_cast<int>(s.listed);
          sort_list(s.list, n_held);
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
      histogram(true, [&](int64_t i, float y) {
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
        histogram(true, [&](int64_t i, float y) { return key_of(i, y) >= outer ? bin_of(r, y) : -1; });
        counted = true;
      }
      find_cut(0, fmax(static_cast<double>(set.top_p), 0.0), sum);
    }
  }

  // ---- the sum of what stays, then the draws, in the order of the indices ----
  const float cut_score = cut > 0 ? key_score(cut) : none;
  const unsigned cut_at = cut > 0 ? static_cast<unsigned>(key_index(cut)) : 0xFFFFFFFFu;
  auto stays = [&](int64_t i, float y) -> Wide {
    if (!(y > cut_score) && !(y == cut_score && y > none && static_cast<unsigned>(i - shift) <= cut_at)) return 0;
    if (greedy) return 1;
    if (r.best - y > r.reach) return 0;
    const double w = scaled_weight(r, s.table, y);
    return w >= r.least ? whole(w) : 0;
  };
  Wide sum = 0;
  each([&](int64_t i, float y) { sum += stays(i, y); });
  const Wide warp_total = warp_sum(sum);
  Wide total;
  Wide below = block_scan(lane == 0 ? warp_total : 0, s.warp, total);  // of the warps before
  below = __shfl_sync(0xFFFFFFFFu, below, 0);
  if (threadIdx.x == 0) s.total = total;
  meet(ctas);
  Wide all = 0, before = 0;
  for (int o = 0; o < ctas; ++o) {
    const Wide t = *of_rank(&s.total, o, ctas);
    if (o < rank) before += t;
    all += t;
  }
  // lane q has draw q
  Wide at = ~0ull;
  if (lane < a.draws) {
    const float u = a.u[p * a.draws + lane];
    at = static_cast<Wide>(static_cast<double>(u > 0.0f ? u : 0.0f) * static_cast<double>(all));
    if (u >= 1.0f || at >= all) at = all - 1;
  }
  const double log_all = log(static_cast<double>(all) / (greedy ? 1.0 : r.one));
  auto resolve = [&](int tile, Wide from, Wide to) {  // the draws that fall to this warp's scores of a tile
    unsigned hits = __ballot_sync(0xFFFFFFFFu, at >= from && at < to);
    while (hits) {
      const int q_draw = __ffs(hits) - 1;
      hits &= hits - 1;
      const Wide target = __shfl_sync(0xFFFFFFFFu, at, q_draw);
      Wide done = from;
#pragma unroll 1
      for (int q = 0; q < loads; ++q) {
        const uint4 raw = get(tile, q);
        const int64_t i0 = place(tile, q);
        Wide w[V], own = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          w[v] = stays(i0 + v, score(raw, v));
          own += w[v];
        }
        const Wide in = warp_scan(own, lane), row_total = __shfl_sync(0xFFFFFFFFu, in, 31);
        if (target < done + row_total) {
          Wide lo = done + in - own;
#pragma unroll
          for (int v = 0; v < V; ++v) {
            if (target >= lo && target < lo + w[v]) {
              const float y = score(raw, v);
              a.idx[p * a.draws + q_draw] = static_cast<int32_t>(i0 + v - shift);
              if (a.logp) {
                const double d = y == r.best ? 0.0 : (static_cast<double>(y) - r.best_wide) / static_cast<double>(set.temperature);
                a.logp[p * a.draws + q_draw] = static_cast<float>(d - log_all);
              }
            }
            lo += w[v];
          }
          break;
        }
        done += row_total;
      }
    }
  };
  if (tiles == 1) {
    resolve(0, before + below, before + below + warp_total);
  } else {
    Wide from = before;
    for (int tile = 0; tile < tiles; ++tile) {
      Wide own = 0;
#pragma unroll 1
      for (int q = 0; q < loads; ++q) {
        const uint4 raw = fetch(place(tile, q));
#pragma unroll
        for (int v = 0; v < V; ++v) own += stays(place(tile, q) + v, score(raw, v));
      }
      own = warp_sum(own);
      Wide b = block_scan(lane == 0 ? own : 0, s.warp, total);
      b = __shfl_sync(0xFFFFFFFFu, b, 0);
      resolve(tile, from + b, from + b + own);
      from += total;
    }
  }
  meet(ctas);  // (its sum is read by the others)
}

template <typename T>
cudaError_t launch_type(const SampleArgs& a, cudaStream_t stream) {
  constexpr int64_t kLoad = kThreads * (16 / sizeof(T));  // scores of one load of a CTA
  const int64_t len = std::max<int64_t>(1, a.seg_off ? a.c / a.p : a.c);  // (of segments the mean)
  int ctas = 1;
  while (ctas < kMaxCtas && kLoad * kLoads * ctas < len) ctas *= 2;
  // few rows: more CTAs each, while they have a thousand scores and more
  while (ctas < kMaxCtas && a.p * ctas * 2 <= 148 && len / (2 * ctas) >= 1024) ctas *= 2;
  // (a stretch is rounded up to whole warps' loads and may begin within one)
  const int64_t each = (len + ctas - 1) / ctas + 64 * (16 / sizeof(T));
  const int loads = static_cast<int>(std::min<int64_t>(kLoads, (each + kLoad - 1) / kLoad));
  if (a.p * ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  const void* kernel = reinterpret_cast<const void*>(&sample_kernel<T>);
  cudaError_t e = ensure_dynamic_smem(kernel, kLoads * kThreads * 16);
  if (e == cudaSuccess && ctas > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(a.p * ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(loads) * kThreads * 16;
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = static_cast<unsigned>(ctas);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a, ctas, loads);
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
