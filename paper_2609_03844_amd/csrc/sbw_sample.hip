// Sampling with temperature, top-k, top-p and min-p (sbw_step.h).  Part of sbw_library.hip.
//
// What the filters keep is a beginning of the row's order (larger first, equal ones by column): top-k by count, top-p by
// the sum of weights before a logit, min-p by its own weight.  Weights are e_v = exp((x_v - m) / T) relative to the row's
// largest logit m.  Of the kept ones the token is the first with the largest x_v / T + G_v, G_v the sampler's Gumbel noise of
// column v under the row's seed.
//
// Where top-p ends goes by sums of weights.  A small top-k sums doubles, in the lanes' order.  One workgroup a row sums whole
// numbers of 2^-F, exact in any order.  The steps for wide rows hold a weight in fp32, and a row's sum like that of the log
// probabilities; the sums in front of a bin are of whole numbers of 2^-61 of it, exact in any order, and doubles within a bin.
#include "sbw_step.h"

#include <algorithm>

namespace sbw {
namespace {

// The parameters of a call: of each row where there is an array, else of all.
struct Filters {
  const float *inv_ts, *top_ps, *min_ps;
  const int32_t* top_ks;
  float inv_t, top_p, min_p;
  int32_t top_k;
};
struct RowFilter {
  float inv_t, top_p, min_p;
  uint32_t top_k;          // V where it is off
};
__device__ __forceinline__ RowFilter row_filter(const Filters& f, int64_t b, uint32_t V) {
  RowFilter r{f.inv_ts != nullptr ? f.inv_ts[b] : f.inv_t, f.top_ps != nullptr ? f.top_ps[b] : f.top_p,
              f.min_ps != nullptr ? f.min_ps[b] : f.min_p, 0u};
  const int32_t k = f.top_ks != nullptr ? f.top_ks[b] : f.top_k;
  r.top_k = k > 0 && static_cast<uint32_t>(k) < V ? static_cast<uint32_t>(k) : V;
  r.top_p = r.top_p < 1.0f ? fmaxf(r.top_p, 0.0f) : 1.0f;   // its share of a sum is taken as a whole number without a sign
  r.min_p = r.min_p > 0.0f ? fminf(r.min_p, 1.0f) : 0.0f;
  return r;
}

// Bits behind the binary point of a weight: the sum of a row's stays below 2^63.
__host__ __device__ inline int weight_bits(uint32_t V) {
  int bits = 0;
  while (bits < 32 && (uint64_t{1} << bits) < V) ++bits;
  return 62 - bits;
}

// A row's kept logits: above `key`, and of those that equal it the ones up to `last`; none below `least`.
struct Kept {
  uint32_t key, last;
  float least;
  __device__ __forceinline__ bool operator()(float x, uint32_t v) const {
    const uint32_t k = order_key(x);
    return (k > key || (k == key && v <= last)) && x >= least;
  }
};
// The smallest float at or above x.
__device__ __forceinline__ float float_from(double x) {
  const float f = static_cast<float>(x);
  if (static_cast<double>(f) >= x || f != f) return f;
  return logit_of_key(order_key(f) + 1u);
}

constexpr int kAnyThreads = 1024;
constexpr uint32_t kDigits = 256;
struct AnyRow {
  uint64_t mass[kDigits], sums[kAnyThreads / kWave];
  uint32_t count[kDigits], digit;
  uint64_t above;          // counts or masses of larger digits
};

__device__ __forceinline__ uint64_t wave_sum64(uint64_t x) {
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ uint64_t wave_most64(uint64_t x) {
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) x = max(x, static_cast<uint64_t>(__shfl_xor(x, d)));
  return x;
}

// A row of any kind by one workgroup (1 x 32000 fp32 of a spread of 3: 330 us where a top-k of 1025 and top-p both cut), which reads it once for each step: the largest logit; four digits
// of the key where top-k ends, four of the one where top-p ends, four of a column where equal logits are parted; the
// weights and the draw.
template <typename T>
__device__ __noinline__ void sample_any_row(const T* row, uint32_t V, RowFilter f, uint64_t row_seed, int32_t* token_at,
                                            float* logprob_at, AnyRow& s) {
  constexpr int kWaves = kAnyThreads / kWave;
  const uint32_t tid = threadIdx.x, wave = tid / kWave;
  const int bits = weight_bits(V);
  const double unit = static_cast<double>(uint64_t{1} << bits);
  // the workgroup's sum or largest, in every lane
  const auto join = [&](uint64_t x, bool most) {
    x = most ? wave_most64(x) : wave_sum64(x);
    __syncthreads();
    if (tid % kWave == 0) s.sums[wave] = x;
    __syncthreads();
    x = s.sums[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) x = most ? max(x, s.sums[w]) : x + s.sums[w];
    return x;
  };
  const auto write = [&](int32_t token, float logprob) {
    if (tid == 0) {
      *token_at = token;
      if (logprob_at != nullptr) *logprob_at = logprob;
    }
  };
  if (!(f.inv_t > 0.0f) || isinf(f.inv_t)) {
    write(-1, __uint_as_float(0x7FC00000u));
    return;
  }
  uint64_t first = 0;
  for (uint32_t v = tid; v < V; v += kAnyThreads)
    first = max(first, static_cast<uint64_t>(order_key(logit_of(row[v]))) << 32 | ~v);
  first = join(first, true);
  const uint32_t highest = static_cast<uint32_t>(first >> 32);
  const float m = logit_of_key(highest);
  if (highest == kLowestKey || !(fabsf(m) < INFINITY)) {
    write(static_cast<int32_t>(~static_cast<uint32_t>(first)), highest == kLowestKey ? -INFINITY : __uint_as_float(0x7FC00000u));
    return;
  }
  const double inv_t = static_cast<double>(f.inv_t);
  const auto weight = [&](float x) -> uint64_t {
    return static_cast<uint64_t>(exp((static_cast<double>(x) - static_cast<double>(m)) * inv_t) * unit);
  };
  // The largest digits first, down to the key at which `target` is reached; its logits' number and the sum above
  // it.  limit, equal: only keys above limit, and `equal` logits at it, take part.
  uint32_t key = 0, equal = 0;
  uint64_t above = 0;
  const auto select = [&](bool by_mass, uint64_t target, uint32_t limit, uint32_t at_limit) {
    key = 0;
    above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      for (uint32_t i = tid; i < kDigits; i += kAnyThreads) s.mass[i] = 0, s.count[i] = 0;
      __syncthreads();
      const uint64_t high = shift == 24 ? 0 : ~uint64_t{0} << (shift + 8);
      for (uint32_t v = tid; v < V; v += kAnyThreads) {
        const float x = logit_of(row[v]);
        const uint32_t k = order_key(x);
        if (((k ^ key) & high) != 0 || k <= limit) continue;
        atomicAdd(&s.count[k >> shift & 255u], 1u);
        if (by_mass) atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[k >> shift & 255u]), weight(x));
      }
      __syncthreads();
      if (tid == 0) {
        if (at_limit != 0 && ((limit ^ key) & high) == 0) {
          s.count[limit >> shift & 255u] += at_limit;
          s.mass[limit >> shift & 255u] += at_limit * weight(logit_of_key(limit));
        }
        uint64_t sum = above;
        uint32_t d = 255, lowest = 0;
        while (lowest < 255 && s.count[lowest] == 0) ++lowest;   // never past the last digit that holds any
        for (; d > lowest; --d) {
          const uint64_t more = by_mass ? s.mass[d] : s.count[d];
          if (s.count[d] != 0 && sum + more >= target) break;
          sum += more;
        }
        s.digit = d;
        s.above = sum;
      }
      __syncthreads();
      key |= s.digit << shift;
      above = s.above;
      equal = s.count[s.digit];
    }
  };
  uint32_t kept_equal = 0;
  bool cut = false;
  if (f.top_k < V) {
    select(false, f.top_k, 0u, 0u);
    kept_equal = f.top_k - static_cast<uint32_t>(above);
    cut = true;
  }
  if (f.top_p < 1.0f) {
    const uint32_t limit = cut ? key : 0u, at_limit = cut ? kept_equal : 0u;
    uint64_t total = 0;
    for (uint32_t v = tid; v < V; v += kAnyThreads) {
      const float x = logit_of(row[v]);
      if (order_key(x) > limit) total += weight(x);
    }
    total = join(total, false);
    if (at_limit != 0) total += at_limit * weight(logit_of_key(limit));
    // kept while the sum before is below top_p of the total
    const uint64_t target = max(uint64_t{1}, static_cast<uint64_t>(ceil(static_cast<double>(f.top_p) * static_cast<double>(total))));
    select(true, target, limit, at_limit);
    const uint64_t of_one = max(uint64_t{1}, weight(logit_of_key(key)));
    const uint64_t wanted = target > above ? (target - above + of_one - 1) / of_one : 1;
    kept_equal = wanted < equal ? static_cast<uint32_t>(wanted) : equal;
    cut = true;
  }
  Kept kept{cut ? key : 0u, V, -INFINITY};
  if (f.min_p > 0.0f) kept.least = float_from(static_cast<double>(m) + log(static_cast<double>(f.min_p)) / inv_t);
  if (cut) {
    // the last column of the equal logits that are kept
    uint64_t of_key = 0;
    for (uint32_t v = tid; v < V; v += kAnyThreads) of_key += order_key(logit_of(row[v])) == key;
    of_key = join(of_key, false);
    if (kept_equal < of_key) {
      uint32_t column = 0, left = kept_equal;
      for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (uint32_t i = tid; i < kDigits; i += kAnyThreads) s.count[i] = 0;
        __syncthreads();
        const uint64_t high = shift == 24 ? 0 : ~uint64_t{0} << (shift + 8);
        for (uint32_t v = tid; v < V; v += kAnyThreads)
          if (((v ^ column) & high) == 0 && order_key(logit_of(row[v])) == key) atomicAdd(&s.count[v >> shift & 255u], 1u);
        __syncthreads();
        if (tid == 0) {
          uint32_t d = 0, sum = 0;
          while (d < 255 && sum + s.count[d] < left) sum += s.count[d++];
          s.digit = d;
          s.above = sum;
        }
        __syncthreads();
        column |= s.digit << shift;
        left -= static_cast<uint32_t>(s.above);
      }
      kept.last = column;
    }
  }
  const Key seed = key_of(row_seed);
  uint64_t total = 0, best = 0;
  for (uint32_t q = tid; q * 4 < V; q += kAnyThreads) {
    bool some = false;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) some |= q * 4 + e < V && kept(logit_of(row[q * 4 + e]), q * 4 + e);
    if (!some) continue;
    const Block draw = philox_block(q, seed);
    const uint32_t word[4] = {draw.w0, draw.w1, draw.w2, draw.w3};
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      const uint32_t v = q * 4 + e;
      if (v >= V) continue;
      const float x = logit_of(row[v]);
      if (!kept(x, v)) continue;
      total += weight(x);
      best = max(best, static_cast<uint64_t>(order_key(x * f.inv_t + gumbel_of(word[e]))) << 32 | ~v);
    }
  }
  total = join(total, false);
  best = join(best, true);
  const uint32_t token = ~static_cast<uint32_t>(best);
  write(static_cast<int32_t>(token), static_cast<float>((static_cast<double>(logit_of(row[token])) - static_cast<double>(m)) * inv_t -
                                                        log(static_cast<double>(total) / unit)));
}

template <typename T>
__global__ void __launch_bounds__(kAnyThreads)
sample_any_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, Filters filters,
                  const uint64_t* __restrict__ seeds, int32_t* __restrict__ tokens, float* __restrict__ logprobs) {
  __shared__ AnyRow s;
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    sample_any_row(logits + b * row_stride, V, row_filter(filters, b, V), seeds[b], tokens + b,
                   logprobs != nullptr ? logprobs + b : nullptr, s);
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Long rows.  One pass over the logits leaves each part's largest logit and sum of weights, and each group's largest logit,
// from which later steps see what they need not read again.  A row with a small top-k is finished from its
// k first logits, in order, by one workgroup.  Any other row is wide: where top-p or a large top-k ends is found from a
// histogram of the weights (or the number) of the logits that can be near, in kBins bins by their distance from the largest;
// bins in front of the one where it ends are kept whole, and the logits of that one are listed and put in order.  All
// workgroups share the wide rows' logits in both steps.
// ---------------------------------------------------------------------------
constexpr uint32_t kSmallTop = SelectionSize<false>::kT;   // top-k that a row's first logits in order are gathered for
constexpr uint32_t kQuarterTop = 64;            // of them by 256 lanes, the others by 1024 (sample_small_kernel)
// As many keys a lane as a row of 160000 logits has groups (200 of 256 x 152064 29 us with 8, 24 so).
struct SampledSize : SelectionSize<true> {
  static constexpr int kHeld = 20;
};
constexpr uint32_t kBins = 2048;
constexpr uint32_t kListed = SelectionSize<false>::kList;

struct PartBest {
  uint64_t best;                                // score's key << 32 | ~column, of the kept ones of a part
  double total;                                 // their weights' sum
};

// How a row is sampled.
struct WidePlan {
  bool small, plain;          // a small top-k; a row with a distribution
  bool by_count, cut, slow;   // the histogram counts; there is one; the row is left to one workgroup
  float m, c, scale, least;   // largest logit, score factor, bins per logit, min-p's floor
  float unit;                 // whole numbers of a weight of 1 in the histogram
  double S, target;           // sum of weights; of the histogram's units in front of where the filter ends
};
// The power of two that takes a sum to between 2^61 and 2^62.  A weight loses less than one of its whole numbers, so V of them
// less than V 2^-61 of the sum (whole numbers of 2^-30 of the largest weight lost V 2^-31 of that, far more than fp32 where a tail lies below).
__device__ __forceinline__ float unit_of(float S) { return __uint_as_float((127u + 61u + 127u - (__float_as_uint(S) >> 23)) << 23); }
__device__ __forceinline__ bool is_small(const RowFilter& f, uint32_t V) { return f.top_k <= kSmallTop && f.top_k < V; }
__device__ __forceinline__ WidePlan wide_plan(const RowFilter& f, uint32_t V, Stats r) {
  WidePlan p{};
  p.small = is_small(f, V);
  p.plain = f.inv_t > 0.0f && !isinf(f.inv_t) && fabsf(r.m) < INFINITY;
  p.m = r.m;
  p.c = score_factor(f.inv_t);
  p.S = r.S;
  p.unit = unit_of(r.S);
  p.by_count = f.top_k < V;
  p.cut = p.by_count || f.top_p < 1.0f;
  p.slow = (p.by_count && f.top_p < 1.0f) || !(fabsf(r.m * f.inv_t) < INFINITY);
  p.least = f.min_p > 0.0f ? float_from(static_cast<double>(r.m) + log(static_cast<double>(f.min_p)) / static_cast<double>(f.inv_t)) : -INFINITY;
  if (p.cut) {
    // logits so far below the largest that all of them together cannot reach what is left out lie behind the end
    const float left = p.by_count ? 0.25f / static_cast<float>(V)
                                  : fmaxf((1.0f - f.top_p) * r.S / static_cast<float>(V) * 0.999f, 1e-12f);
    p.scale = static_cast<float>(kBins) * f.inv_t / -logf(fminf(left, 0.5f));
    p.target = p.by_count ? static_cast<double>(f.top_k)
                          : ceil(static_cast<double>(f.top_p) * p.S * static_cast<double>(p.unit));
    if (!(p.scale > 1e-30f) || !(p.scale < 1e30f)) p.slow = true;
  }
  return p;
}
// A wide row between the steps, in the workspace (cleared by the first one).
struct WideRow {
  WidePlan plan;
  uint64_t bins[kBins];
  uint64_t list[kListed];                       // key << 32 | ~column
  uint32_t listed, unused;
};
// The bin of a logit (kBins and more: behind all); larger logits have smaller bins.
__device__ __forceinline__ uint32_t bin_of(const WidePlan& p, float x) {
  return static_cast<uint32_t>(fminf((p.m - x) * p.scale, 2.0f * kBins));
}
__device__ __forceinline__ float weight_of(const WidePlan& p, float x) { return __builtin_amdgcn_exp2f((x - p.m) * p.c); }

// The pass.  Workgroups and groups as in row_pass_kernel.  Bound by memory: 256 x 152064 fp32 25 us, 6.1 TB/s.
template <typename T, int kVecs, bool kStats, bool kTop>
__global__ void __launch_bounds__(kThreads)
sample_pass_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, Filters filters,
                   Stats* __restrict__ parts, Maxima maxima, WideRow* __restrict__ wide) {
  constexpr uint32_t kPer = kPerOf<T>;
  const uint32_t j0 = blockIdx.x * (kThreads * kVecs) + threadIdx.x;
  const bool whole = (blockIdx.x + 1) * (kThreads * kVecs) <= V / kPer;
  for (int64_t b = blockIdx.y; b < B; b += gridDim.y) {
    const T* row = logits + b * row_stride;
    typename VecOf<T>::Value x[kVecs];
#pragma unroll
    for (int u = 0; u < kVecs; ++u) x[u] = whole ? load_whole(row, j0 + u * kThreads) : load_any(row, V, j0 + u * kThreads);
    if (wide != nullptr) {
      for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < kBins; i += gridDim.x * kThreads) wide[b].bins[i] = 0;
      if (blockIdx.x == 0 && threadIdx.x == 0) wide[b].listed = 0;
    }
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < kVecs; ++u)
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e) m = larger(m, elem(x[u], e));
    const int64_t segment = b * gridDim.x + blockIdx.x;
    const uint32_t key = order_key(m);
    maxima.groups[segment * kThreads + threadIdx.x] = key;
    if (kTop) {
      const uint32_t of_block = row_largest(key);
      if (threadIdx.x % kBlockLanes == 0) maxima.blocks[segment * kBlocksOf + threadIdx.x / kBlockLanes] = of_block;
    }
    if (kStats) {
      m = wave_largest(m);
      const float base = m == -INFINITY ? 0.0f : m, c = score_factor(filters.inv_ts != nullptr ? filters.inv_ts[b] : filters.inv_t);
      float S = 0.0f;
#pragma unroll
      for (int u = 0; u < kVecs; ++u) {
        float of_vector = 0.0f;
#pragma unroll
        for (uint32_t e = 0; e < kPer; ++e) of_vector += __builtin_amdgcn_exp2f((elem(x[u], e) - base) * c);
        S += of_vector;
      }
      S = wave_sum(S);
      if (threadIdx.x % kWave == 0) parts[segment * (kThreads / kWave) + threadIdx.x / kWave] = Stats{m, S, 0.0f};
    }
  }
}

// The plans of wide rows, a wave each (in the steps that go by them it took 2 us of each workgroup).
__global__ void __launch_bounds__(kThreads)
sample_plan_kernel(int64_t B, uint32_t V, uint32_t segments, const Stats* __restrict__ parts, Filters filters, WideRow* __restrict__ wide) {
  const uint32_t count = segments * (kThreads / kWave);
  const int64_t b = static_cast<int64_t>(blockIdx.x) * (kThreads / kWave) + threadIdx.x / kWave;
  if (b >= B) return;
  const RowFilter f = row_filter(filters, b, V);
  if (is_small(f, V)) return;
  const WidePlan p = wide_plan(f, V, join_parts(parts + b * count, count, score_factor(f.inv_t)));
  if (threadIdx.x % kWave == 0) wide[b].plan = p;
}

// A small top-k: the first logits in order, their weights' sums, the draw among those that are kept; a lane for each.  Bound by
// dependent trips to memory, like any selection.  Us of a call with top-p, by 256 lanes and by 1024: 50 of 1 x 32000 fp32 13.3 and 14.2, of
// 64 x 128256 bf16 16.4 and 17.4; 100 17.1 and 15.9, 21.3 and 19.0; 256 22.7 and 16.4, 29.3 and 20.5; where rows differ 1024 take all
// (both, one after the other, 30 us of 256 requests).  Up to 1024 lanes' worth beats a histogram: 400 of 64 x 128256 21.6 and 48, 1000 28.5 and 50, of 256 x 152064 fp32 60 and 142; with top-p behind
// it no histogram serves, and one workgroup a row takes 235 for 1 x 32000, 650 for 64 x 128256.
template <typename T, int kVecs, typename Size>
__global__ void __launch_bounds__(Size::kT)
sample_small_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, uint32_t segments, Maxima maxima,
                    Filters filters, const uint64_t* __restrict__ seeds, int32_t* __restrict__ tokens, float* __restrict__ logprobs) {
  static_assert(Size::kT >= (Size::kSmall ? kQuarterTop : kSmallTop), "a lane for each of the first logits");
  constexpr int kWaves = Size::kT / kWave;
  __shared__ Selection<Size> s;
  __shared__ double sums[2][kWaves];
  __shared__ uint64_t bests[kWaves];
  const uint32_t tid = threadIdx.x, wave = tid / kWave;
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const RowFilter f = row_filter(filters, b, V);
    if (!is_small(f, V)) continue;
    const T* row = logits + b * row_stride;
    const Maxima of_row = row_maxima(maxima, b, segments);
    const uint64_t* best = select_row<T, kVecs, Size>(
        (const SBW_GLOBAL T*)row, V, (const SBW_GLOBAL uint32_t*)of_row.groups, (const SBW_GLOBAL uint32_t*)of_row.blocks,
        segments, f.top_k, (SBW_LDS Selection<Size>*)&s);
    const uint64_t first = best[0], mine = best[min(tid, f.top_k - 1)];
    const uint32_t highest = static_cast<uint32_t>(first >> 32), column = ~static_cast<uint32_t>(mine);
    const float m = logit_of_key(highest), x = logit_of_key(static_cast<uint32_t>(mine >> 32));
    const bool valid = f.inv_t > 0.0f && !isinf(f.inv_t);
    if (!valid || highest == kLowestKey || !(fabsf(m) < INFINITY)) {
      if (tid == 0) {
        tokens[b] = valid ? static_cast<int32_t>(~static_cast<uint32_t>(first)) : -1;
        if (logprobs != nullptr) logprobs[b] = valid && highest == kLowestKey ? -INFINITY : __uint_as_float(0x7FC00000u);
      }
      __syncthreads();
      continue;
    }
    const double inv_t = static_cast<double>(f.inv_t), score = (static_cast<double>(x) - static_cast<double>(m)) * inv_t;
    const double weight = tid < f.top_k ? exp(score) : 0.0;
    double upto = weight;                       // of the lanes up to this one
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const double before = __shfl_up(upto, d);
      if (tid % kWave >= static_cast<uint32_t>(d)) upto += before;
    }
    if (tid % kWave == kWave - 1) sums[0][wave] = upto;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w == static_cast<int>(wave)) upto += total;
      total += sums[0][w];
    }
    const float least = f.min_p > 0.0f ? float_from(static_cast<double>(m) + log(static_cast<double>(f.min_p)) / inv_t) : -INFINITY;
    const bool kept = tid < f.top_k && (tid == 0 || f.top_p >= 1.0f || upto - weight < static_cast<double>(f.top_p) * total) && x >= least;
    uint64_t drawn = 0;
    if (kept) {
      const Block words = philox_block(column / 4, key_of(seeds[b]));
      const uint32_t e = column % 4, word = e == 0 ? words.w0 : e == 1 ? words.w1 : e == 2 ? words.w2 : words.w3;
      drawn = static_cast<uint64_t>(order_key(x * f.inv_t + gumbel_of(word))) << 32 | ~column;
    }
    const uint64_t most = wave_most64(drawn);
    double of_kept = kept ? weight : 0.0;
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) of_kept += __shfl_xor(of_kept, d);
    if (tid % kWave == 0) {
      bests[wave] = most;
      sums[1][wave] = of_kept;
    }
    __syncthreads();
    uint64_t winner = bests[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) winner = max(winner, bests[w]);
    if (drawn == winner && kept) {
      double whole = 0.0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) whole += sums[1][w];
      tokens[b] = static_cast<int32_t>(column);
      if (logprobs != nullptr) logprobs[b] = static_cast<float>(score - log(whole));
    }
    __syncthreads();
  }
}

// The workgroup's groups that a step looks at, side by side; their number.
__device__ __forceinline__ uint32_t list_groups(bool some, uint16_t* list, uint32_t* counts) {
  const uint64_t mask = __ballot(some);
  if (threadIdx.x % kWave == 0) counts[threadIdx.x / kWave] = __popcll(mask);
  __syncthreads();
  uint32_t at = __popcll(mask & ((uint64_t{1} << threadIdx.x % kWave) - 1u)), total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) {
    if (w < static_cast<int>(threadIdx.x / kWave)) at += counts[w];
    total += counts[w];
  }
  if (some) list[at] = static_cast<uint16_t>(threadIdx.x);
  __syncthreads();
  return total;
}

// The histogram of a wide row with top-p or a large top-k.  Groups whose largest logit lies behind all bins are not read.  Bound by the
// atomics in LDS of neighbouring weights: 64 x 128256 bf16 12.6 us, 32 of 256 x 152064 fp32 among others 20.
template <typename T, int kVecs>
__global__ void __launch_bounds__(kThreads)
sample_bins_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, const uint32_t* __restrict__ groups,
                   Filters filters, WideRow* __restrict__ wide) {
  constexpr uint32_t kPer = kPerOf<T>;
  __shared__ uint64_t bins[kBins];
  __shared__ uint16_t listed[kThreads];
  __shared__ uint32_t counts[kThreads / kWave];
  const uint32_t j0 = blockIdx.x * (kThreads * kVecs);
  for (int64_t b = blockIdx.y; b < B; b += gridDim.y) {
    const RowFilter f = row_filter(filters, b, V);
    if (is_small(f, V) || (f.top_k >= V && f.top_p >= 1.0f)) continue;
    const WidePlan p = wide[b].plan;
    if (!p.plain || p.slow) continue;
    const T* row = logits + b * row_stride;
    const bool near = bin_of(p, logit_of_key(groups[(b * gridDim.x + blockIdx.x) * kThreads + threadIdx.x])) < kBins;
    const uint32_t items = list_groups(near, listed, counts) * kVecs;
    if (items == 0) continue;
    for (uint32_t i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
    __syncthreads();
#pragma unroll 2
    for (uint32_t i = threadIdx.x; i < items; i += kThreads) {
      const uint32_t j = j0 + listed[i / kVecs] + i % kVecs * kThreads;
      const auto x = load_any(row, V, j);
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e) {
        const float v = elem(x, e);
        const uint32_t bin = bin_of(p, v);
        if (bin >= kBins || j * kPer + e >= V) continue;
        const auto w = p.by_count ? 1ull : static_cast<unsigned long long>(weight_of(p, v) * p.unit);
        atomicAdd(reinterpret_cast<unsigned long long*>(&bins[bin]), w);
      }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kBins; i += kThreads)
      if (bins[i] != 0) atomicAdd(reinterpret_cast<unsigned long long*>(&wide[b].bins[i]), static_cast<unsigned long long>(bins[i]));
    __syncthreads();
  }
}

// The bin where the filter ends, and the sum in front of it, the same in every lane of the workgroup; kBins where it ends
// beyond all bins (a count may, and a sum by its rounding), which leaves the row to one workgroup.
struct CutBin {
  uint32_t bin;
  uint64_t before;
};
template <int kT>
__device__ __forceinline__ CutBin cut_bin(const uint64_t* bins, double target, uint64_t* sums, CutBin* found) {
  constexpr int kEach = kBins / kT, kWaves = kT / kWave;
  uint64_t own[kEach], total = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) total += own[i] = bins[threadIdx.x * kEach + i];
  uint64_t before = total;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const uint64_t n = __shfl_up(before, d);
    if (threadIdx.x % kWave >= static_cast<uint32_t>(d)) before += n;
  }
  if (threadIdx.x % kWave == kWave - 1) sums[threadIdx.x / kWave] = before;
  if (threadIdx.x == 0) *found = CutBin{kBins, 0};
  __syncthreads();
  before -= total;
#pragma unroll
  for (int w = 0; w < kWaves; ++w)
    if (w < static_cast<int>(threadIdx.x / kWave)) before += sums[w];
  const uint64_t wanted = max(uint64_t{1}, static_cast<uint64_t>(target));
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (before < wanted && before + own[i] >= wanted) *found = CutBin{threadIdx.x * kEach + i, before};
    before += own[i];
  }
  __syncthreads();
  return *found;
}

// The kept logits of a wide row: the largest score of those in front of the bin where the filter ends, their weights' sum,
// and the list of that bin's.  A kept logit's noise is first bounded from both sides by its draw's bits; only where its
// upper bound reaches the largest lower one so far, about one of a wave's vector, it is queued and its noise computed.  (All
// in registers and unrolled, without a queue, the code was as long as 32 logarithms and took 58 us for 64 x 128256.)
// The bin's logits gather in LDS first: one atomic a workgroup reserves their places (one for each logit: 24 us, so 16).
constexpr uint32_t kQueued = 1024, kCutListed = 1024;
template <typename T, int kVecs>
__global__ void __launch_bounds__(kThreads)
sample_wide_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, const uint32_t* __restrict__ groups,
                   Filters filters, const uint64_t* __restrict__ seeds,
                   WideRow* __restrict__ wide, PartBest* __restrict__ bests) {
  constexpr uint32_t kPer = kPerOf<T>;
  constexpr int kWaves = kThreads / kWave;
  __shared__ uint64_t sums[kWaves];
  __shared__ CutBin found;
  __shared__ uint16_t listed[kThreads];
  __shared__ uint32_t counts[kWaves];
  __shared__ uint32_t queued_column[kWaves][kQueued];
  __shared__ float queued_logit[kWaves][kQueued];
  __shared__ uint64_t cut_list[kCutListed];
  __shared__ uint32_t cut_listed, cut_place;
  const uint32_t tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, j0 = blockIdx.x * (kThreads * kVecs);
  for (int64_t b = blockIdx.y; b < B; b += gridDim.y) {
    const RowFilter f = row_filter(filters, b, V);
    if (is_small(f, V)) continue;
    const WidePlan p = wide[b].plan;
    if (!p.plain || p.slow) continue;
    const T* row = logits + b * row_stride;
    const float of_group = logit_of_key(groups[(b * gridDim.x + blockIdx.x) * kThreads + tid]);
    const CutBin cut = p.cut ? cut_bin<kThreads>(wide[b].bins, p.target, sums, &found) : CutBin{0, 0};
    // whatever stands this far below the largest cannot be drawn: the noise lies in (-2.82, 16.64)
    const float highest = p.m * f.inv_t, lowest = __builtin_fmaf(-fabsf(highest), 9.5367431640625e-7f, highest - 20.0f);
    const auto wanted = [&](float x) { return (!p.cut || bin_of(p, x) <= cut.bin) && x >= p.least; };
    const bool summed = p.cut || p.least > -INFINITY;     // else the sum of all is known
    const Key seed = key_of(seeds[b]);
    uint64_t best = 0;
    float total = 0.0f;                                   // of a lane's logits, in the order of the list
    float most = highest + kGumbelLo;                     // that the best score reaches
    uint32_t queue = 0;
    const auto flush = [&] {
      for (uint32_t i = lane; i < queue; i += kWave) {
        const uint32_t v = queued_column[wave][i];
        const Block words = philox_block(v / 4, seed);
        const uint32_t word = v % 4 == 0 ? words.w0 : v % 4 == 1 ? words.w1 : v % 4 == 2 ? words.w2 : words.w3;
        best = max(best, static_cast<uint64_t>(order_key(queued_logit[wave][i] * f.inv_t + gumbel_of(word))) << 32 | ~v);
      }
      queue = 0;
    };
    if (tid == 0) cut_listed = 0;
    const uint32_t items = list_groups(cut.bin < kBins && wanted(of_group), listed, counts) * kVecs;
    const auto vector_of = [&](uint32_t i) { return j0 + listed[min(i, items - 1) / kVecs] + min(i, items - 1) % kVecs * kThreads; };
    if (items > wave * kWave) {
      uint32_t j = vector_of(tid);
      auto next = load_any(row, V, j);
#pragma unroll 1
      for (uint32_t i0 = wave * kWave; i0 < items; i0 += kThreads) {
        const uint32_t i = i0 + lane, of_next = vector_of(i + kThreads);
        auto x = next;
        if (i0 + kThreads < items) next = load_any(row, V, of_next);
        if (i >= items) x = lowest_vec(typename VecOf<T>::Value{});
#pragma unroll
        for (uint32_t q = 0; q < kPer / 4; ++q) {
          float upper[4];
          bool any = false;
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e) {
            const uint32_t v = j * kPer + q * 4 + e;
            const float y = elem(x, q * 4 + e);
            bool kept = i < items && v < V && wanted(y);
            if (kept && p.cut && bin_of(p, y) == cut.bin) {
              const uint64_t entry = static_cast<uint64_t>(order_key(y)) << 32 | ~v;
              const uint32_t n = count_one(cut_listed);
              if (n < kCutListed) {
                cut_list[n] = entry;
              } else {
                const uint32_t at = atomicAdd(&wide[b].listed, 1u);
                if (at < kListed) wide[b].list[at] = entry;
              }
              kept = false;
            }
            if (summed && kept) total += weight_of(p, y);
            const bool drawn = kept && y * f.inv_t >= lowest;
            any |= drawn;
            upper[e] = drawn ? 0.0f : -INFINITY;
          }
          if (!__any(any)) continue;
          const Block words = philox_block(j * (kPer / 4) + q, seed);
          const uint32_t word[4] = {words.w0, words.w1, words.w2, words.w3};
          float lower = -INFINITY;
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e) {
            const float y = elem(x, q * 4 + e) * f.inv_t;
            const float above = __builtin_fmaf(-kNoiseBitsScale, noise_bits(word[e]), kNoiseBitsOffset);
            const bool drawn = upper[e] == 0.0f;
            upper[e] = drawn ? y + above : -INFINITY;
            lower = fmaxf(lower, drawn ? y + (above > kNoiseUpperRange ? above - kNoiseGap : kGumbelLo) : -INFINITY);
          }
          if (__any(lower > most)) most = fmaxf(most, wave_reduce(lower, -INFINITY, [](float a, float c) { return fmaxf(a, c); }));
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e) {
            const uint64_t can = __ballot(upper[e] >= most);
            if (can == 0) continue;
            if (queue + kWave > kQueued) flush();
            if (upper[e] >= most) {
              const uint32_t at = queue + __popcll(can & ((uint64_t{1} << lane) - 1u));
              queued_column[wave][at] = j * kPer + q * 4 + e;
              queued_logit[wave][at] = elem(x, q * 4 + e);
            }
            queue += __popcll(can);
          }
        }
        j = of_next;
      }
      flush();
    }
    best = wave_most64(best);
    if (summed) total = wave_sum(total);
    if (lane == 0) bests[(b * gridDim.x + blockIdx.x) * kWaves + wave] = PartBest{best, static_cast<double>(total)};
    __syncthreads();
    const uint32_t own = min(cut_listed, kCutListed);
    if (own != 0) {
      if (tid == 0) cut_place = atomicAdd(&wide[b].listed, own);
      __syncthreads();
      for (uint32_t i = tid; i < own; i += kThreads)
        if (cut_place + i < kListed) wide[b].list[cut_place + i] = cut_list[i];
    }
    __syncthreads();
  }
}

// The parts of a wide row joined, with the listed logits' share; rows that no other step took.  One workgroup a row: a chain of
// the bins' sums, the list's order and two sums over the lanes, 17 us whatever the number of rows.
template <typename T>
__global__ void __launch_bounds__(kAnyThreads)
sample_join_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, uint32_t segments,
                   Filters filters, const uint64_t* __restrict__ seeds, const WideRow* __restrict__ wide, const PartBest* __restrict__ bests,
                   int32_t* __restrict__ tokens, float* __restrict__ logprobs) {
  using Size = SelectionSize<false>;
  static_assert(Size::kT == kAnyThreads, "one workgroup");
  constexpr int kWaves = kAnyThreads / kWave;
  __shared__ union {
    Selection<Size> list;
    AnyRow any;
  } s;
  __shared__ uint64_t sums[kWaves], most[kWaves];
  __shared__ double weights[2][kWaves];
  __shared__ CutBin found;
  const uint32_t tid = threadIdx.x, wave = tid / kWave, count = segments * (kThreads / kWave);
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const RowFilter f = row_filter(filters, b, V);
    if (is_small(f, V)) continue;
    const T* row = logits + b * row_stride;
    const WidePlan p = wide[b].plan;
    const bool valid = f.inv_t > 0.0f && !isinf(f.inv_t);
    if (!valid || p.m == -INFINITY) {          // no parameter, or no logit
      if (tid == 0) {
        tokens[b] = valid ? 0 : -1;
        if (logprobs != nullptr) logprobs[b] = valid ? -INFINITY : __uint_as_float(0x7FC00000u);
      }
      continue;
    }
    bool alone = !p.plain || p.slow;
    CutBin cut{0, 0};
    uint32_t listed = 0;
    if (p.cut && !alone) {
      cut = cut_bin<kAnyThreads>(wide[b].bins, p.target, sums, &found);
      listed = wide[b].listed;
      alone = cut.bin == kBins || listed > kListed;
    }
    if (alone) {
      sample_any_row(row, V, f, seeds[b], tokens + b, logprobs != nullptr ? logprobs + b : nullptr, s.any);
      __syncthreads();
      continue;
    }
    const double inv_t = static_cast<double>(f.inv_t);
    uint64_t best = 0;
    double whole = 0.0;
    for (uint32_t i = tid; i < count; i += kAnyThreads) {
      const PartBest part = bests[b * count + i];
      best = max(best, part.best);
      whole += part.total;
    }
    double own = 0.0;                    // of the listed logits that are kept
    if (p.cut) {
      const double before = p.by_count ? 0.0 : static_cast<double>(cut.before) / static_cast<double>(p.unit), target = p.by_count ? 0.0 : static_cast<double>(f.top_p) * p.S;
      const uint32_t still = p.by_count ? f.top_k - static_cast<uint32_t>(cut.before) : listed;
      for (uint32_t i = tid; i < listed; i += kAnyThreads) s.list.list[i] = wide[b].list[i];
      __syncthreads();
      const uint64_t* in_order = sorted(listed, s.list);
      double sum = before;               // in front of the lanes' next logits
      for (uint32_t i0 = 0; i0 < listed; i0 += kAnyThreads) {
        const uint32_t i = i0 + tid;
        const uint64_t mine = i < listed ? in_order[i] : 0;
        const float x = logit_of_key(static_cast<uint32_t>(mine >> 32));
        const double weight = i < listed ? exp((static_cast<double>(x) - static_cast<double>(p.m)) * inv_t) : 0.0;
        double upto = weight;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
          const double n = __shfl_up(upto, d);
          if (tid % kWave >= static_cast<uint32_t>(d)) upto += n;
        }
        if (tid % kWave == kWave - 1) weights[0][wave] = upto;
        __syncthreads();
        double in_front = sum;
        for (int w = 0; w < kWaves; ++w) {
          if (w < static_cast<int>(wave)) in_front += weights[0][w];
          sum += weights[0][w];
        }
        const bool first = i == 0 && cut.before == 0;
        const bool kept = i < listed && x >= p.least && (p.by_count ? i < still : first || in_front + upto - weight < target);
        if (kept) {
          const uint32_t v = ~static_cast<uint32_t>(mine);
          const Block words = philox_block(v / 4, key_of(seeds[b]));
          const uint32_t word = v % 4 == 0 ? words.w0 : v % 4 == 1 ? words.w1 : v % 4 == 2 ? words.w2 : words.w3;
          best = max(best, static_cast<uint64_t>(order_key(x * f.inv_t + gumbel_of(word))) << 32 | ~v);
          own += weight;
        }
        __syncthreads();
      }
    }
    best = wave_most64(best);
    own += whole;
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) own += __shfl_xor(own, d);
    if (tid % kWave == 0) most[wave] = best, weights[1][wave] = own;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kWaves; ++w) {
        best = max(best, most[w]);
        own += weights[1][w];
      }
      const uint32_t token = min(~static_cast<uint32_t>(best), V - 1);
      tokens[b] = static_cast<int32_t>(token);
      if (logprobs != nullptr) {
        const bool all = !p.cut && f.min_p <= 0.0f;
        const double total = all ? p.S : own;
        logprobs[b] = static_cast<float>((static_cast<double>(logit_of(row[token])) - static_cast<double>(p.m)) * inv_t - log(total));
      }
    }
    __syncthreads();
  }
}

// Few short rows that nothing is cut from are left to one workgroup each.  Us so and in steps: 1 x 4096 fp32 12.7 and 15.2, 64 x 1024
// 11.3 and 17.2, 64 x 4096 14.2 and 16.7; but 64 x 8192 19.2 and 17.0, 512 x 1024 32 and 25.  With top-p, or a top-k of 50, one workgroup takes
// 80 and 140 us for a row of any of these lengths, the steps 24 and 13.
constexpr int64_t kShortSampled = 4096, kFewSampled = 128;

// The workspace: statistics of the pass, maxima, best scores, wide rows.  Its sizes go by B and V alone.
struct SampleSpace {
  bool longer;                  // long segments
  int64_t segments, parts, maxima, bests, wide, total;   // offsets in uint64 elements
};
constexpr int64_t kRowsAtOnce = 512;   // more rows take turns: a wide row's space is 49 KB
SampleSpace sample_space(int64_t B, int64_t V) {
  SampleSpace s{};
  B = std::min(B, kRowsAtOnce);
  // Long segments leave fewer parts to join and groups to look at, short ones fill the chip.  Us with top-p 0.9, short and long: 1 x 32000
  // fp32 24.4 and 27.9, 1 x 152064 bf16 28.2 and 29.2, 16 x 128256 39.0 and 32.0, 64 x 128256 78.9 and 46.8, 256 x 152064 fp32 243 and
  // 129.  A selection of up to 40 wants twice as many blocks.
  const int64_t of_long = (V + kLongSegment - 1) / kLongSegment;
  s.longer = B * of_long >= 256 && of_long * kBlocksOf >= 80;
  s.segments = s.longer ? of_long : (V + kShortSegment - 1) / kShortSegment;
  s.maxima = B * s.segments * kPartElems;
  s.bests = s.maxima + B * s.segments * kMaximaElems;
  s.wide = s.bests + B * s.segments * (kThreads / kWave) * static_cast<int64_t>(sizeof(PartBest) / 8);
  s.total = s.wide + B * static_cast<int64_t>(sizeof(WideRow) / 8);
  return s;
}

template <typename T, int kVecs>
void launch_long_rows(const T* logits, int64_t B, uint32_t V, int64_t row_stride, const Filters& filters, const uint64_t* seeds,
                      int32_t* tokens, float* logprobs, uint64_t* workspace, const SampleSpace& space, hipStream_t stream) {
  const bool all_small = filters.top_ks == nullptr && filters.top_k > 0 && filters.top_k <= static_cast<int32_t>(kSmallTop) &&
                         static_cast<uint32_t>(filters.top_k) < V;
  const bool any_small = all_small || filters.top_ks != nullptr;
  const bool any_cut = filters.top_ks != nullptr || filters.top_k > 0 || filters.top_ps != nullptr || filters.top_p < 1.0f;
  const auto segments = static_cast<uint32_t>(space.segments);
  const Maxima maxima = maxima_at(workspace + space.maxima, B, space.segments);
  auto* parts = reinterpret_cast<Stats*>(workspace);
  auto* bests = reinterpret_cast<PartBest*>(workspace + space.bests);
  auto* wide = reinterpret_cast<WideRow*>(workspace + space.wide);
  const dim3 grid(segments, static_cast<uint32_t>(B));
  const auto rows = static_cast<uint32_t>(grid_for(B));
  auto* pass = all_small ? sample_pass_kernel<T, kVecs, false, true>
               : any_small ? sample_pass_kernel<T, kVecs, true, true> : sample_pass_kernel<T, kVecs, true, false>;
  pass<<<grid, kThreads, 0, stream>>>(logits, B, V, row_stride, filters, parts, maxima, !all_small && any_cut ? wide : nullptr);
  if (!all_small) sample_plan_kernel<<<static_cast<uint32_t>((B + 3) / 4), kThreads, 0, stream>>>(B, V, segments, parts, filters, wide);
  if (any_small) {
    const bool quarter = all_small && filters.top_k <= static_cast<int32_t>(kQuarterTop);
    auto* small = quarter ? sample_small_kernel<T, kVecs, SampledSize> : sample_small_kernel<T, kVecs, SelectionSize<false>>;
    small<<<rows, quarter ? SampledSize::kT : kSmallTop, 0, stream>>>(logits, B, V, row_stride, segments, maxima, filters, seeds, tokens,
                                                                      logprobs);
  }
  if (all_small) return;
  if (any_cut) sample_bins_kernel<T, kVecs><<<grid, kThreads, 0, stream>>>(logits, B, V, row_stride, maxima.groups, filters, wide);
  sample_wide_kernel<T, kVecs><<<grid, kThreads, 0, stream>>>(logits, B, V, row_stride, maxima.groups, filters, seeds, wide, bests);
  sample_join_kernel<T><<<rows, kAnyThreads, 0, stream>>>(logits, B, V, row_stride, segments, filters, seeds, wide, bests, tokens, logprobs);
}

template <typename T>
void launch_sample(const void* logits_, int64_t B, uint32_t V, int64_t row_stride, const Filters& filters,
                   const uint64_t* seeds, int32_t* tokens, float* logprobs, uint64_t* workspace, hipStream_t stream) {
  const T* logits = static_cast<const T*>(logits_);
  const bool cuts = filters.top_ks != nullptr || (filters.top_k > 0 && static_cast<uint32_t>(filters.top_k) < V) ||
                    filters.top_ps != nullptr || filters.top_p < 1.0f;
  if (!cuts && V <= kShortSampled && B <= kFewSampled) {
    sample_any_kernel<T><<<static_cast<uint32_t>(grid_for(B)), kAnyThreads, 0, stream>>>(logits, B, V, row_stride, filters, seeds,
                                                                                        tokens, logprobs);
    return;
  }
  const SampleSpace space = sample_space(B, V);
  auto* launch = space.longer ? launch_long_rows<T, kLongVecs<T>> : launch_long_rows<T, kShortVecs<T>>;
  for (int64_t b = 0; b < B; b += kRowsAtOnce) {
    const auto from = [&](const auto* p) { return p != nullptr ? p + b : nullptr; };
    Filters of_rows = filters;
    of_rows.inv_ts = from(filters.inv_ts);
    of_rows.top_ps = from(filters.top_ps);
    of_rows.min_ps = from(filters.min_ps);
    of_rows.top_ks = from(filters.top_ks);
    launch(logits + b * row_stride, std::min(B - b, kRowsAtOnce), V, row_stride, of_rows, seeds + b, tokens + b,
           logprobs != nullptr ? logprobs + b : nullptr, workspace, space, stream);
  }
}

}  // namespace
}  // namespace sbw

extern "C" {

int64_t sbw_sample_tokens_workspace(int64_t B, int64_t V) {
  if (B <= 0 || V <= 0 || V > kMostColumns || B > INT64_MAX / 4 / V) return 0;
  return sample_space(B, V).total;
}

sbw_status_t sbw_sample_tokens(const void* logits, sbw_dtype_t dtype, int64_t B, int64_t V, int64_t row_stride,
                               const uint64_t* seeds, const float* inv_temperatures, float inv_temperature,
                               const int32_t* top_ks, int64_t top_k, const float* top_ps, float top_p,
                               const float* min_ps, float min_p, int32_t* tokens, float* logprobs, uint64_t* workspace,
                               void* stream) {
  sbw_status_t s = check_logits(logits, dtype, B, V, row_stride);
  if (s != SBW_OK) return s;
  if (inv_temperatures == nullptr && (!(inv_temperature > 0.0f) || isinf(inv_temperature))) return SBW_ERR_INVALID_ARG;
  if ((top_ps == nullptr && isnan(top_p)) || (min_ps == nullptr && isnan(min_p))) return SBW_ERR_INVALID_ARG;
  if (B == 0) return SBW_OK;
  if (seeds == nullptr || tokens == nullptr) return SBW_ERR_INVALID_ARG;
  if (workspace == nullptr && sbw_sample_tokens_workspace(B, V) > 0) return SBW_ERR_INVALID_ARG;
  s = check_device();
  if (s != SBW_OK) return s;
  const int64_t most = INT32_MAX;
  const Filters filters{inv_temperatures, top_ps, min_ps, top_ks, inv_temperature, top_p, min_p,
                        static_cast<int32_t>(top_k < 0 ? 0 : top_k < most ? top_k : most)};
  auto* launch = dtype == SBW_F32 ? launch_sample<float> : launch_sample<uint16_t>;
  launch(logits, B, static_cast<uint32_t>(V), row_stride, filters, seeds, tokens, logprobs, workspace, static_cast<hipStream_t>(stream));
  return after_launch();
}

}  // extern "C"
