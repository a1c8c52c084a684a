// Next-token logits by a head with 4-bit weights (sbw_step.h).  Part of sbw_library.hip.
#include "sbw_step.h"

namespace sbw {
namespace {

constexpr int64_t kMostHidden = 8192;

// One wave a logit: its lanes share the columns, eight weights a 32-bit word.
template <typename S, typename T>
__global__ void __launch_bounds__(kThreads)
head_logits_kernel(const uint16_t* __restrict__ hidden, int64_t B, uint32_t K, int64_t hidden_stride,
                   const uint8_t* __restrict__ codes, const S* __restrict__ scales, uint32_t group,
                   int64_t V, T* __restrict__ logits, int64_t row_stride) {
  const int64_t waves = static_cast<int64_t>(gridDim.x) * (kThreads / kWave);
  const uint32_t lane = threadIdx.x % kWave;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * (kThreads / kWave) + threadIdx.x / kWave; i < B * V;
       i += waves) {
    const int64_t b = i % B, v = i / B;
    float total = 0.0f;
    for (uint32_t c = lane; c < K / 2; c += kWave) {
      const uint32_t q = codes[v * (K / 2) + c];
      const uint16_t* h = hidden + b * hidden_stride + 2 * c;
      float d = logit_of(h[0]) * (static_cast<float>(q & 15u) - 8.0f);
      d = __builtin_fmaf(logit_of(h[1]), static_cast<float>(q >> 4) - 8.0f, d);
      total = __builtin_fmaf(d, logit_of(scales[v * (K / group) + 2 * c / group]), total);
    }
    total = wave_sum(total);
    if (lane == 0) put_logit(logits + b * row_stride + v, total);
  }
}

template <typename S, typename T>
void launch_head(const void* hidden, int64_t B, int64_t K, int64_t hidden_stride, const uint8_t* codes,
                 const void* scales, int64_t group, int64_t V, void* logits, int64_t row_stride,
                 hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(grid_for((B * V + 3) / 4)));
  head_logits_kernel<S, T><<<grid, kThreads, 0, stream>>>(
      static_cast<const uint16_t*>(hidden), B, static_cast<uint32_t>(K), hidden_stride, codes,
      static_cast<const S*>(scales), static_cast<uint32_t>(group), V, static_cast<T*>(logits), row_stride);
}

}  // namespace
}  // namespace sbw

extern "C" sbw_status_t sbw_head_logits(const void* hidden, int64_t B, int64_t K, int64_t hidden_stride,
                                        const uint8_t* codes, const void* scales, sbw_dtype_t scale_dtype,
                                        int64_t group, int64_t V, void* logits, sbw_dtype_t dtype,
                                        int64_t row_stride, void* stream) {
  if (B < 0 || V < 0 || K <= 0 || hidden_stride < K || row_stride < V) return SBW_ERR_INVALID_ARG;
  if (group != 32 && group != 64 && group != 128) return SBW_ERR_UNSUPPORTED;
  if (K % group != 0) return SBW_ERR_INVALID_ARG;
  if (K > kMostHidden || V > kMostColumns) return SBW_ERR_UNSUPPORTED;
  if ((dtype != SBW_F32 && dtype != SBW_BF16) || (scale_dtype != SBW_F32 && scale_dtype != SBW_BF16))
    return SBW_ERR_UNSUPPORTED;
  if (B == 0 || V == 0) return SBW_OK;
  if (hidden == nullptr || codes == nullptr || scales == nullptr || logits == nullptr)
    return SBW_ERR_INVALID_ARG;
  if (B > INT64_MAX / 4 / row_stride || B > INT64_MAX / 4 / hidden_stride) return SBW_ERR_UNSUPPORTED;
  const sbw_status_t s = check_device();
  if (s != SBW_OK) return s;
  const auto st = static_cast<hipStream_t>(stream);
  auto* launch = scale_dtype == SBW_F32
                     ? (dtype == SBW_F32 ? launch_head<float, float> : launch_head<float, uint16_t>)
                     : (dtype == SBW_F32 ? launch_head<uint16_t, float> : launch_head<uint16_t, uint16_t>);
  launch(hidden, B, K, hidden_stride, codes, scales, group, V, logits, row_stride, st);
  return after_launch();
}
