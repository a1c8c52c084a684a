// Log probabilities of given tokens with entropy and the most likely alternatives, their
// gradient, and the k largest logits of a row (sbw_step.h).  Part of sbw_library.hip.
//
// With c = inv_temperature * log2(e) and a row's largest logit m, every sum runs over
// e_v = 2^((x_v - m) c), which lies in [0, 1]:
//   S = sum e_v,  A = sum e_v (x_v - m) c
//   lse = m * inv_temperature + ln S,  log p_t = (x_t - m) * inv_temperature - ln S,
//   entropy = ln S - ln 2 * A / S.
#include "sbw_step.h"

namespace sbw {
namespace {

constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / kWave;
constexpr int kMostTokens = SBW_STEP_MAX_TOKENS;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.693147180559945309417f;

__device__ __forceinline__ float logit_of(float x) { return x; }
__device__ __forceinline__ float logit_of(uint16_t x) {
  return __uint_as_float(static_cast<uint32_t>(x) << 16);
}

// The order of logits as unsigned integers: larger logits have larger keys, every NaN the
// largest, both zeros the same.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);   // -0 + 0 = +0
  const uint32_t key = b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
  return x != x ? 0xFFFFFFFFu : key;
}
__device__ __forceinline__ float logit_of_key(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// (x - m) * inv_t - ln_s; halved on the way, so that only a result beyond fp32 is infinite.
__device__ __forceinline__ float logprob_of(float x, float m, float inv_t, float ln_s) {
  return __builtin_fmaf((0.5f * x - 0.5f * m) * inv_t, 2.0f, -ln_s);
}

template <typename F>
__device__ __forceinline__ float wave_reduce(float v, F f) {
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) v = f(v, __shfl_xor(v, d));
  return v;
}

// The reduction of one value a thread over the workgroup, the same in every thread.
template <typename F>
__device__ __forceinline__ float row_reduce(float v, F f, float* slots) {
  v = wave_reduce(v, f);
  __syncthreads();
  if (threadIdx.x % kWave == 0) slots[threadIdx.x / kWave] = v;
  __syncthreads();
  v = slots[0];
  for (int w = 1; w < kRowWaves; ++w) v = f(v, slots[w]);
  return v;
}
__device__ __forceinline__ uint32_t row_count(uint32_t v, uint32_t* slots) {
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) v += __shfl_xor(v, d);
  __syncthreads();
  if (threadIdx.x % kWave == 0) slots[threadIdx.x / kWave] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < kRowWaves; ++w) v += slots[w];
  return v;
}

__device__ __forceinline__ float larger(float a, float b) { return a > b || a != a ? a : b; }
__device__ __forceinline__ float sum(float a, float b) { return a + b; }

// The k first logits of a row in order, as (key << 32 | ~column), in best[0 .. found).
// Bisection over the keys for the k-th largest, then the larger logits and as many equal
// ones, by column, as there is room for.
struct Selection {
  uint64_t raw[kMostTokens], best[kMostTokens];
  uint32_t slots[kRowWaves], taken;
};
template <typename T>
__device__ uint32_t select_row(const T* row, uint32_t V, uint32_t k, Selection& s) {
  k = k < V ? k : V;
  const uint32_t tid = threadIdx.x;
  uint32_t at = 0;      // the largest key with k logits at or above it
  for (uint32_t bit = 0x80000000u; bit != 0; bit >>= 1) {
    uint32_t c = 0;
    for (uint32_t v = tid; v < V; v += kRowThreads) c += order_key(logit_of(row[v])) >= (at | bit);
    if (row_count(c, s.slots) >= k) at |= bit;
  }
  if (tid == 0) s.taken = 0;
  __syncthreads();
  for (uint32_t v = tid; v < V; v += kRowThreads) {
    const uint32_t key = order_key(logit_of(row[v]));
    if (key > at) s.raw[atomicAdd(&s.taken, 1u)] = static_cast<uint64_t>(key) << 32 | ~v;
  }
  __syncthreads();
  uint32_t taken = s.taken;
  for (uint32_t v0 = 0; v0 < V && taken < k; v0 += kRowThreads) {
    const bool equal = v0 + tid < V && order_key(logit_of(row[v0 + tid])) == at;
    const uint64_t mask = __ballot(equal);
    __syncthreads();
    if (tid % kWave == 0) s.slots[tid / kWave] = __popcll(mask);
    __syncthreads();
    uint32_t before = taken;
    for (uint32_t w = 0; w < kRowWaves; ++w) {
      if (w < tid / kWave) before += s.slots[w];
      taken += s.slots[w];
    }
    before += __popcll(mask & ((uint64_t{1} << (tid % kWave)) - 1u));
    if (equal && before < k) s.raw[before] = static_cast<uint64_t>(at) << 32 | ~(v0 + tid);
  }
  __syncthreads();
  if (tid < k) {
    const uint64_t mine = s.raw[tid];
    uint32_t rank = 0;
    for (uint32_t i = 0; i < k; ++i) rank += s.raw[i] > mine;
    s.best[rank] = mine;
  }
  __syncthreads();
  return k;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
token_logprobs_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride,
                      const int32_t* __restrict__ tokens, uint32_t n, float inv_t, uint32_t top,
                      float* __restrict__ logprobs, float* __restrict__ lse,
                      float* __restrict__ entropy, float* __restrict__ stats,
                      int32_t* __restrict__ top_ids, float* __restrict__ top_logprobs) {
  __shared__ float slots[kRowWaves];
  __shared__ Selection s;
  const uint32_t tid = threadIdx.x;
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const T* row = logits + b * row_stride;
    float m = -INFINITY;
    for (uint32_t v = tid; v < V; v += kRowThreads) m = larger(logit_of(row[v]), m);
    m = row_reduce(m, larger, slots);
    const bool empty = m == -INFINITY;
    const float c = inv_t * kLog2e;
    float S = 0.0f, A = 0.0f;
    for (uint32_t v = tid; v < V; v += kRowThreads) {
      const float y = empty ? -INFINITY : (logit_of(row[v]) - m) * c;
      const float e = __builtin_amdgcn_exp2f(y);
      S += e;
      A = __builtin_fmaf(e, fmaxf(y, -1e30f), A);   // 0 * -inf is no part of the sum
    }
    S = row_reduce(S, sum, slots);
    A = row_reduce(A, sum, slots);
    const float ln_s = logf(S);
    if (tid == 0) {
      if (lse != nullptr) lse[b] = empty ? -INFINITY : __builtin_fmaf(m, inv_t, ln_s);
      if (entropy != nullptr) entropy[b] = empty ? 0.0f : ln_s - kLn2 * (A / S);
      if (stats != nullptr) stats[2 * b] = m, stats[2 * b + 1] = ln_s;
    }
    for (uint32_t j = tid; j < n; j += kRowThreads) {
      const int32_t t = tokens[b * n + j];
      const bool token = t >= 0 && static_cast<uint32_t>(t) < V;
      logprobs[b * n + j] = !token ? 0.0f : empty ? -INFINITY : logprob_of(logit_of(row[t]), m, inv_t, ln_s);
    }
    if (top == 0) continue;
    const uint32_t found = select_row(row, V, top, s);
    for (uint32_t j = tid; j < top; j += kRowThreads) {
      top_ids[b * top + j] = j < found ? static_cast<int32_t>(~static_cast<uint32_t>(s.best[j])) : -1;
      if (top_logprobs != nullptr) {
        const float x = j < found ? logit_of_key(static_cast<uint32_t>(s.best[j] >> 32)) : 0.0f;
        top_logprobs[b * top + j] = j >= found || empty ? -INFINITY : logprob_of(x, m, inv_t, ln_s);
      }
    }
    __syncthreads();
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
top_candidates_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride,
                      uint32_t vbase, uint32_t k, int32_t* __restrict__ ids,
                      float* __restrict__ values) {
  __shared__ Selection s;
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const uint32_t found = select_row(logits + b * row_stride, V, k, s);
    for (uint32_t j = threadIdx.x; j < k; j += kRowThreads) {
      ids[b * k + j] = j < found ? static_cast<int32_t>(vbase + ~static_cast<uint32_t>(s.best[j])) : -1;
      if (values != nullptr)
        values[b * k + j] = j < found ? logit_of_key(static_cast<uint32_t>(s.best[j] >> 32)) : -INFINITY;
    }
    __syncthreads();
  }
}

__device__ __forceinline__ void put_logit(float* p, float x) { *p = x; }
__device__ __forceinline__ void put_logit(uint16_t* p, float x) {
  *p = static_cast<uint16_t>(to_bf16x2(x, 0.0f));
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
token_logprobs_grad_kernel(const T* logits, int64_t B, uint32_t V, int64_t row_stride,
                           const int32_t* __restrict__ tokens, uint32_t n,
                           const float* __restrict__ stats, const float* __restrict__ entropy,
                           const float* __restrict__ grad_logprobs,
                           const float* __restrict__ grad_lse,
                           const float* __restrict__ grad_entropy, float inv_t, T* grad,
                           int64_t grad_stride) {
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const T* row = logits + b * row_stride;
    T* out = grad + b * grad_stride;
    const float m = stats[2 * b], ln_s = stats[2 * b + 1];
    const float gh = grad_entropy != nullptr ? grad_entropy[b] : 0.0f;
    float share = grad_lse != nullptr ? grad_lse[b] : 0.0f;
    if (grad_entropy != nullptr) share -= gh * entropy[b];
    const int32_t* ids = tokens + b * n;
    const float* g = grad_logprobs + b * n;
    if (grad_logprobs != nullptr)
      for (uint32_t j = 0; j < n; ++j)
        if (ids[j] >= 0 && static_cast<uint32_t>(ids[j]) < V) share -= g[j];
    for (uint32_t v = threadIdx.x; v < V; v += kRowThreads) {
      const float y = __builtin_fmaf(logit_of(row[v]) - m, inv_t, -ln_s);
      const float p = __builtin_amdgcn_exp2f(y * kLog2e);
      float d = p * __builtin_fmaf(-gh, fmaxf(y, -1e30f), share);
      if (grad_logprobs != nullptr)
        for (uint32_t j = 0; j < n; ++j)
          if (static_cast<uint32_t>(ids[j]) == v) d += g[j];
      put_logit(out + v, m == -INFINITY ? 0.0f : d * inv_t);
    }
  }
}

constexpr int64_t kMostColumns = kMaxTokenIds - 65536;   // column + a workgroup's stride fits 32 bits

sbw_status_t check_logits(const void* logits, sbw_dtype_t dtype, int64_t B, int64_t V, int64_t row_stride) {
  if (B < 0 || V < 0 || row_stride < V) return SBW_ERR_INVALID_ARG;
  if (dtype != SBW_F32 && dtype != SBW_BF16) return SBW_ERR_UNSUPPORTED;
  if (V > kMostColumns) return SBW_ERR_UNSUPPORTED;
  if (B == 0) return SBW_OK;
  if (V == 0 || logits == nullptr) return SBW_ERR_INVALID_ARG;
  if (B > INT64_MAX / 4 / row_stride) return SBW_ERR_UNSUPPORTED;
  return SBW_OK;
}
sbw_status_t check_most(int64_t count, int64_t least) {
  if (count < least) return SBW_ERR_INVALID_ARG;
  return count > kMostTokens ? SBW_ERR_UNSUPPORTED : SBW_OK;
}

}  // namespace
}  // namespace sbw

extern "C" {

int64_t sbw_token_logprobs_workspace(int64_t B, int64_t V, int64_t top) {
  (void)B, (void)V, (void)top;
  return 0;
}

int64_t sbw_top_candidates_workspace(int64_t B, int64_t V, int64_t k) {
  (void)B, (void)V, (void)k;
  return 0;
}

sbw_status_t sbw_token_logprobs(const void* logits, sbw_dtype_t dtype, int64_t B, int64_t V,
                                int64_t row_stride, const int32_t* tokens, int64_t n,
                                float inv_temperature, int64_t top, float* logprobs, float* lse,
                                float* entropy, float* stats, int32_t* top_ids,
                                float* top_logprobs, uint64_t* workspace, void* stream) {
  sbw_status_t s = check_most(n, 0);
  if (s == SBW_OK) s = check_most(top, 0);
  if (s == SBW_OK) s = check_logits(logits, dtype, B, V, row_stride);
  if (s != SBW_OK) return s;
  if (!(inv_temperature > 0.0f) || isinf(inv_temperature)) return SBW_ERR_INVALID_ARG;
  if (B == 0) return SBW_OK;
  if (n > 0 && (tokens == nullptr || logprobs == nullptr)) return SBW_ERR_INVALID_ARG;
  if (top > 0 && top_ids == nullptr) return SBW_ERR_INVALID_ARG;
  if (workspace == nullptr && sbw_token_logprobs_workspace(B, V, top) > 0) return SBW_ERR_INVALID_ARG;
  s = check_device();
  if (s != SBW_OK) return s;
  const auto st = static_cast<hipStream_t>(stream);
  const dim3 grid(static_cast<uint32_t>(grid_for(B)));
  if (dtype == SBW_F32)
    token_logprobs_kernel<float><<<grid, kRowThreads, 0, st>>>(
        static_cast<const float*>(logits), B, static_cast<uint32_t>(V), row_stride, tokens,
        static_cast<uint32_t>(n), inv_temperature, static_cast<uint32_t>(top), logprobs, lse, entropy,
        stats, top_ids, top_logprobs);
  else
    token_logprobs_kernel<uint16_t><<<grid, kRowThreads, 0, st>>>(
        static_cast<const uint16_t*>(logits), B, static_cast<uint32_t>(V), row_stride, tokens,
        static_cast<uint32_t>(n), inv_temperature, static_cast<uint32_t>(top), logprobs, lse, entropy,
        stats, top_ids, top_logprobs);
  return after_launch();
}

sbw_status_t sbw_token_logprobs_grad(const void* logits, sbw_dtype_t dtype, int64_t B, int64_t V,
                                     int64_t row_stride, const int32_t* tokens, int64_t n,
                                     const float* stats, const float* entropy,
                                     const float* grad_logprobs, const float* grad_lse,
                                     const float* grad_entropy, float inv_temperature, void* grad,
                                     int64_t grad_stride, void* stream) {
  sbw_status_t s = check_most(n, 0);
  if (s == SBW_OK) s = check_logits(logits, dtype, B, V, row_stride);
  if (s != SBW_OK) return s;
  if (!(inv_temperature > 0.0f) || isinf(inv_temperature)) return SBW_ERR_INVALID_ARG;
  if (grad_stride < V) return SBW_ERR_INVALID_ARG;
  if (B == 0) return SBW_OK;
  if (stats == nullptr || grad == nullptr || (n > 0 && grad_logprobs != nullptr && tokens == nullptr) ||
      (grad_entropy != nullptr && entropy == nullptr) || (grad == logits && grad_stride != row_stride))
    return SBW_ERR_INVALID_ARG;
  if (B > INT64_MAX / 4 / grad_stride) return SBW_ERR_UNSUPPORTED;
  s = check_device();
  if (s != SBW_OK) return s;
  const auto st = static_cast<hipStream_t>(stream);
  const dim3 grid(static_cast<uint32_t>(grid_for(B)));
  if (dtype == SBW_F32)
    token_logprobs_grad_kernel<float><<<grid, kRowThreads, 0, st>>>(
        static_cast<const float*>(logits), B, static_cast<uint32_t>(V), row_stride, tokens,
        static_cast<uint32_t>(n), stats, entropy, grad_logprobs, grad_lse, grad_entropy, inv_temperature,
        static_cast<float*>(grad), grad_stride);
  else
    token_logprobs_grad_kernel<uint16_t><<<grid, kRowThreads, 0, st>>>(
        static_cast<const uint16_t*>(logits), B, static_cast<uint32_t>(V), row_stride, tokens,
        static_cast<uint32_t>(n), stats, entropy, grad_logprobs, grad_lse, grad_entropy, inv_temperature,
        static_cast<uint16_t*>(grad), grad_stride);
  return after_launch();
}

sbw_status_t sbw_top_candidates(const void* logits, sbw_dtype_t dtype, int64_t B, int64_t V,
                                int64_t row_stride, int64_t v_offset, int64_t k, int32_t* ids,
                                float* values, uint64_t* workspace, void* stream) {
  sbw_status_t s = check_most(k, 1);
  if (s == SBW_OK) s = check_logits(logits, dtype, B, V, row_stride);
  if (s != SBW_OK) return s;
  if (v_offset < 0) return SBW_ERR_INVALID_ARG;
  if (!ids_fit(V, v_offset)) return SBW_ERR_UNSUPPORTED;
  if (B == 0) return SBW_OK;
  if (ids == nullptr) return SBW_ERR_INVALID_ARG;
  if (workspace == nullptr && sbw_top_candidates_workspace(B, V, k) > 0) return SBW_ERR_INVALID_ARG;
  s = check_device();
  if (s != SBW_OK) return s;
  const auto st = static_cast<hipStream_t>(stream);
  const dim3 grid(static_cast<uint32_t>(grid_for(B)));
  const auto vbase = static_cast<uint32_t>(v_offset);
  if (dtype == SBW_F32)
    top_candidates_kernel<float><<<grid, kRowThreads, 0, st>>>(
        static_cast<const float*>(logits), B, static_cast<uint32_t>(V), row_stride, vbase,
        static_cast<uint32_t>(k), ids, values);
  else
    top_candidates_kernel<uint16_t><<<grid, kRowThreads, 0, st>>>(
        static_cast<const uint16_t*>(logits), B, static_cast<uint32_t>(V), row_stride, vbase,
        static_cast<uint32_t>(k), ids, values);
  return after_launch();
}

}  // extern "C"
