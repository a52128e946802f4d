// Draws from the softmax of scores with temperature, top-k, top-p and min-p (ks_sample).
//
// A score's weight exp((x - best) / t) is held as a whole number of 2^-s of the best one's, with 64-bit sums. Sums of whole
// numbers do not depend on the order they are taken in, so the cuts and the draws do not depend on how a row is shared out;
// and what a rounding of 2^-s moves at a border lies far below what 32 bits of a weight would (a draw among 100,000 equal
// candidates meets a border within 2^-24 once in 100 times).
//
// The candidates that stay are the front of the order (score descending, index ascending), so top-k and top-p are each a
// place in it: the last score that stays, and how many of those that share it do. A histogram over the distance to the best
// score narrows it down to one bin, histograms over the bits of that bin's scores to one score.
#include <algorithm>
#include <cmath>

#include "ks_e4m3.cuh"
#include "ks_internal.h"
#include "ks_topk.cuh"

namespace ks {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr float kBinsPerUnit = 56.0f;  // bins a factor of e: weights end at 52 bits, 36.05 units, 2,019 bins

using Wide = unsigned long long;

// The place in the order where a row is cut: scores above `key` stay, of those that equal it the first `ties`.
struct Cut {
  unsigned key;
  unsigned ties;
};

struct Row {
  float best, per_t;  // bins a unit of score
  double inv_t;
  double one;         // weight of the best score, 2^s
  double least;       // weights below do not stay (min-p)
};

template <typename T>
__device__ __forceinline__ float score_at(const T* row, int64_t i) {
  const float v = to_float(row[i]) + 0.0f;  // (of the two zeros one)
  return v == v ? v : __int_as_float(0xFF800000);
}

// weight in units of 2^-s, and whether min-p lets it stay
__device__ __forceinline__ Wide weight(const Row& r, float x) {
  if (x == r.best) return static_cast<Wide>(r.one);
  const double w = exp((static_cast<double>(x) - static_cast<double>(r.best)) * r.inv_t) * r.one;
  return w >= r.least ? static_cast<Wide>(__double2ll_rn(w)) : 0ull;
}
__device__ __forceinline__ Wide weight_any(const Row& r, float x) {
  if (x == r.best) return static_cast<Wide>(r.one);
  return static_cast<Wide>(__double2ll_rn(exp((static_cast<double>(x) - static_cast<double>(r.best)) * r.inv_t) * r.one));
}

__device__ __forceinline__ int bin_of(const Row& r, float x) {
  return static_cast<int>(fminf((r.best - x) * r.per_t, static_cast<float>(kBins - 1)));
}

__device__ __forceinline__ Wide warp_scan(Wide v, int lane) {  // inclusive
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const Wide u = __shfl_up_sync(0xFFFFFFFFu, v, d);
    if (lane >= d) v += u;
  }
  return v;
}

// Exclusive sum over the block's threads; the block's in `total`.
__device__ __forceinline__ Wide block_scan(Wide v, Wide* s_warp, Wide& total) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const Wide in = warp_scan(v, lane);
  __syncthreads();
  if (lane == 31) s_warp[warp] = in;
  __syncthreads();
  Wide before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += s_warp[w];
    total += s_warp[w];
  }
  return before + in - v;
}

struct Shared {
  unsigned count[kBins];
  Wide sum[kBins];
  Wide warp[kWarps];
  float warp_f[kWarps];
  int bin;
  Wide before_count, before_sum;
};

// The place where the order's front of `n` candidates (n > 0), or else the shortest whose weights sum to `part` of all
// (of those above `first`), ends. False: nothing is cut.
template <typename T>
__device__ bool find_cut(const T* row, int64_t len, const Row& r, Wide n, double part, const Cut* first, Cut& cut, Shared& s) {
  unsigned prefix = 0;
  int bin0 = 0;
  Wide before_count = 0, before_sum = 0;
  double target = 0.0;
  const int shifts[4] = {0, 21, 10, 0};
  const int bits[4] = {0, 11, 11, 10};
  for (int level = 0; level < 4; ++level) {
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
      s.count[i] = 0;
      s.sum[i] = 0;
    }
    __syncthreads();
    Wide ties_before = 0;
    for (int64_t i0 = 0; i0 < len; i0 += kThreads) {
      const int64_t i = i0 + threadIdx.x;
      const float x = i < len ? score_at(row, i) : __int_as_float(0xFF800000);
      const unsigned key = sortable(x);
      Wide w = i < len ? weight_any(r, x) : 0;
      if (first) {  // the candidates that the first cut leaves: ties by their order
        Wide total;
        const Wide before = block_scan(w > 0 && key == first->key, s.warp, total) + ties_before;
        ties_before += total;
        if (key < first->key || (key == first->key && before >= first->ties)) w = 0;
      }
      if (w == 0) continue;
      const int bin = bin_of(r, x);
      int digit = bin;
      if (level > 0) {
        if (bin != bin0 || (level > 1 && (key >> (shifts[level] + bits[level])) != (prefix >> (shifts[level] + bits[level])))) continue;
        digit = (1 << bits[level]) - 1 - ((key >> shifts[level]) & ((1 << bits[level]) - 1));  // the largest scores first
      }
      atomicAdd(&s.count[digit], 1u);
      atomicAdd(&s.sum[digit], w);
    }
    __syncthreads();
    // four bins a thread
    Wide c[4], w[4], tc = 0, tw = 0, total_c, total_w;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      c[q] = s.count[threadIdx.x * 4 + q];
      w[q] = s.sum[threadIdx.x * 4 + q];
      tc += c[q];
      tw += w[q];
    }
    Wide bc = block_scan(tc, s.warp, total_c) + before_count;
    Wide bw = block_scan(tw, s.warp, total_w) + before_sum;
    if (level == 0) {
      target = fmax(part * static_cast<double>(total_w), 1.0);  // (weights are whole numbers: the best one stays)
      if (n > 0 ? total_c <= n : static_cast<double>(total_w) <= target) return false;
      __syncthreads();
      if (threadIdx.x == 0) s.bin = -1;
      __syncthreads();
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {  // the bin with the last candidate that stays
      const bool starts = n > 0 ? bc < n : static_cast<double>(bw) < target;
      const bool ends = n > 0 ? bc + c[q] >= n : !(static_cast<double>(bw + w[q]) < target);
      if (c[q] > 0 && starts && ends) {
        s.bin = threadIdx.x * 4 + q;
        s.before_count = bc;
        s.before_sum = bw;
      }
      bc += c[q];
      bw += w[q];
    }
    __syncthreads();
    before_count = s.before_count;
    before_sum = s.before_sum;
    const int at = s.bin;
    if (level == 0) bin0 = at;
    else prefix |= static_cast<unsigned>((1 << bits[level]) - 1 - at) << shifts[level];
    if (level == 3) {
      cut.key = prefix;
      const Wide have = s.count[at], each = s.sum[at] / have;
      Wide m = n > 0 ? n - before_count : static_cast<Wide>(ceil((target - static_cast<double>(before_sum)) / static_cast<double>(each)));
      cut.ties = static_cast<unsigned>(m < 1 ? 1 : m > have ? have : m);
    }
    __syncthreads();
  }
  return true;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const __grid_constant__ SampleArgs a) {
  __shared__ Shared s;
  const int64_t p = blockIdx.x;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t begin = a.seg_off ? a.seg_off[p] : p * a.ld;
  const int64_t len = a.seg_off ? a.seg_off[p + 1] - begin : a.c;
  const T* row = static_cast<const T*>(a.scores) + begin;
  const ks_sampling set = a.params ? a.params[p] : a.all;
  const float none = __int_as_float(0xFF800000);

  float best = none;
  for (int64_t i = threadIdx.x; i < len; i += kThreads) best = fmaxf(best, score_at(row, i));
#pragma unroll
  for (int d = 1; d < 32; d *= 2) best = fmaxf(best, __shfl_xor_sync(0xFFFFFFFFu, best, d));
  if (lane == 0) s.warp_f[warp] = best;
  __syncthreads();
  for (int w = 0; w < kWarps; ++w) best = fmaxf(best, s.warp_f[w]);
  for (int i = threadIdx.x; i < a.draws; i += kThreads) {
    a.idx[p * a.draws + i] = -1;
    if (a.logp) a.logp[p * a.draws + i] = none;
  }
  if (best == none) return;
  __syncthreads();

  // Temperature 0 is the limit of small ones: the best score alone, and of several that share it the first.
  const bool greedy = !(set.temperature > 0.0f);
  Row r;
  r.best = best;
  r.inv_t = greedy ? 0.0 : 1.0 / static_cast<double>(set.temperature);
  r.per_t = greedy ? 0.0f : kBinsPerUnit / set.temperature;
  r.one = ldexp(1.0, min(52, __clzll(len) - 2));  // sums of all weights fit 63 bits
  r.least = set.min_p > 0.0f ? fmin(static_cast<double>(set.min_p), 1.0) * r.one : 0.0;
  Cut cut{0, 0xFFFFFFFFu}, cut_p;
  bool cuts = false;
  if (greedy) {
    cut = Cut{sortable(best), 1};
    cuts = true;
  } else {
    if (set.top_k > 0) cuts = find_cut(row, len, r, static_cast<Wide>(set.top_k), 1.0, static_cast<const Cut*>(nullptr), cut, s);
    if (set.top_p < 1.0f && find_cut(row, len, r, 0, fmax(static_cast<double>(set.top_p), 0.0), cuts ? &cut : nullptr, cut_p, s)) {
      cut = cut_p;
      cuts = true;
    }
  }
  // twice over the row in the order of the indices: the sum of what stays, then the draws
  Wide all = 0;
  for (int pass = 0; pass < 2; ++pass) {
    Wide ties_before = 0, sum_before = 0;
    for (int64_t i0 = 0; i0 < len; i0 += kThreads) {
      const int64_t i = i0 + threadIdx.x;
      const float x = i < len ? score_at(row, i) : none;
      const unsigned key = sortable(x);
      Wide w = x > none && (!cuts || key >= cut.key) ? weight(r, x) : 0;
      Wide total;
      if (cuts) {
        const Wide before = block_scan(w > 0 && key == cut.key, s.warp, total) + ties_before;
        ties_before += total;
        if (key == cut.key && before >= cut.ties) w = 0;
      }
      const Wide lo = block_scan(w, s.warp, total) + sum_before;
      sum_before += total;
      if (pass == 1 && w > 0) {
        for (int q = 0; q < a.draws; ++q) {
          const float u = a.u[p * a.draws + q];
          Wide at = static_cast<Wide>(static_cast<double>(u > 0.0f ? u : 0.0f) * static_cast<double>(all));
          at = at < all ? at : all - 1;
          if (at >= lo && at < lo + w) {
            a.idx[p * a.draws + q] = static_cast<int32_t>(i);
            if (a.logp) {
              const double d = x == r.best ? 0.0 : (static_cast<double>(x) - static_cast<double>(r.best)) * r.inv_t;
              a.logp[p * a.draws + q] = static_cast<float>(d - log(static_cast<double>(all) / r.one));
            }
          }
        }
      }
    }
    all = sum_before;
  }
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, int score_type, cudaStream_t stream, int64_t* launches) {
  const unsigned grid = static_cast<unsigned>(a.p);
  switch (score_type) {
    case KS_F32: sample_kernel<float><<<grid, kThreads, 0, stream>>>(a); break;
    case KS_BF16: sample_kernel<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(a); break;
    default: sample_kernel<__half><<<grid, kThreads, 0, stream>>>(a);
  }
  ++*launches;
  return cudaGetLastError();
}

}  // namespace ks
