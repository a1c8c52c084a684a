// Sampling with temperature, top-k, top-p and min-p (sbw_step.h).  Part of sbw_library.hip.
//
// What the filters keep is a beginning of the row's order (larger first, equal ones by column): top-k by count, top-p by
// the sum of weights before a logit, min-p by its own weight.  Weights are e_v = exp((x_v - m) / T) relative to the row's
// largest logit m, held as whole numbers of 2^-F, so that their sums are exact in any order.  Of the kept ones
// the token is the first with the largest x_v / T + G_v, G_v the sampler's Gumbel noise of column v under the
// row's seed.
#include "sbw_step.h"

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
  if (!(r.top_p < 1.0f)) r.top_p = 1.0f;
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
  uint64_t mass[kDigits], best[kAnyThreads / kWave], sums[kAnyThreads / kWave];
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

// A row of any kind by one workgroup, which reads it once for each step: the largest logit; four digits
// of the key where top-k ends, four of the one where top-p ends, four of a column where equal logits are parted; the
// weights and the draw.
template <typename T>
__global__ void __launch_bounds__(kAnyThreads)
sample_any_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, Filters filters,
                  const uint64_t* __restrict__ seeds, int32_t* __restrict__ tokens, float* __restrict__ logprobs) {
  constexpr int kWaves = kAnyThreads / kWave;
  __shared__ AnyRow s;
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
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const T* row = logits + b * row_stride;
    const RowFilter f = row_filter(filters, b, V);
    const auto write = [&](int32_t token, float logprob) {
      if (tid == 0) {
        tokens[b] = token;
        if (logprobs != nullptr) logprobs[b] = logprob;
      }
    };
    if (!(f.inv_t > 0.0f) || isinf(f.inv_t)) {
      write(-1, __uint_as_float(0x7FC00000u));
      continue;
    }
    uint64_t first = 0;
    for (uint32_t v = tid; v < V; v += kAnyThreads)
      first = max(first, static_cast<uint64_t>(order_key(logit_of(row[v]))) << 32 | ~v);
    first = join(first, true);
    const uint32_t highest = static_cast<uint32_t>(first >> 32);
    const float m = logit_of_key(highest);
    if (highest == kLowestKey || !(fabsf(m) < INFINITY)) {
      write(static_cast<int32_t>(~static_cast<uint32_t>(first)), highest == kLowestKey ? -INFINITY : __uint_as_float(0x7FC00000u));
      continue;
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
    const Key seed = key_of(seeds[b]);
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
}

template <typename T>
void launch_sample(const void* logits, int64_t B, uint32_t V, int64_t row_stride, const Filters& filters,
                   const uint64_t* seeds, int32_t* tokens, float* logprobs, hipStream_t stream) {
  sample_any_kernel<T><<<static_cast<uint32_t>(grid_for(B)), kAnyThreads, 0, stream>>>(
      static_cast<const T*>(logits), B, V, row_stride, filters, seeds, tokens, logprobs);
}

}  // namespace
}  // namespace sbw

extern "C" {

int64_t sbw_sample_tokens_workspace(int64_t B, int64_t V) {
  if (B <= 0 || V <= 0 || V > kMostColumns) return 0;
  return 0;
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
  launch(logits, B, static_cast<uint32_t>(V), row_stride, filters, seeds, tokens, logprobs, static_cast<hipStream_t>(stream));
  return after_launch();
}

}  // extern "C"
