// Next-token logits by a head with 4-bit weights (sbw_step.h).  Part of sbw_library.hip.
#include "sbw_step.h"

namespace sbw {
namespace {

constexpr int64_t kMostHidden = 8192;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kChunk = 128;              // columns of a wave's 16-byte loads: 16 rows x 64 bytes
constexpr int kTileRows = 16;            // head rows of a matrix instruction
constexpr int kHeadWaves = 16;           // of a CU
constexpr uint32_t kSixteens = 0x41804180u;   // two bf16 16.0: or a 4-bit q into bits 3-6 for 16 + q
constexpr uint32_t kCodeBits = 0x00780078u;

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                 0, 0);
}

// Eight 4-bit codes as bf16 16 + q, in the order 0 4 1 5 2 6 3 7.  `sixteens` is kSixteens in a vector
// register: an instruction reads one scalar operand, and the mask is that one.
__device__ __forceinline__ u32x4 widened(uint32_t w, uint32_t sixteens) {
  return u32x4{((w << 3) & kCodeBits) | sixteens, ((w >> 1) & kCodeBits) | sixteens,
               ((w >> 5) & kCodeBits) | sixteens, ((w >> 9) & kCodeBits) | sixteens};
}
// Eight hidden values in the same order.
__device__ __forceinline__ u32x4 in_code_order(u32x4 h) {
  return u32x4{(h.x & 0xFFFFu) | h.z << 16, h.x >> 16 | (h.z & 0xFFFF0000u), (h.y & 0xFFFFu) | h.w << 16,
               h.y >> 16 | (h.w & 0xFFFF0000u)};
}

// A lane's 16 bytes hold 32 columns of one row, a quarter (lane / 16) of a chunk; word d its columns
// 8 d .. 8 d + 7.  A matrix instruction sums over the four quarters' words, so for groups smaller
// than a chunk the words are exchanged between quarters until each instruction's lie in one group.
// Instruction i then takes, in this quarter, word `d` of quarter `q`:
struct Source {
  uint32_t q, d;
};
template <int kGroup>
__device__ __forceinline__ Source source_of(uint32_t i, uint32_t quarter) {
  if (kGroup == 128) return Source{quarter, i};
  if (kGroup == 32) return Source{i, quarter};
  const bool upper = quarter >= 2;
  if (i < 2) return Source{upper ? quarter - 2 : quarter, upper ? i + 2 : i};
  return Source{upper ? quarter : quarter + 2, upper ? i : i - 2};
}
// Swap a's upper half (lanes 32-63) with b's lower half; a's odd quarters with b's even ones.
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
__device__ __forceinline__ void swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
template <int kGroup>
__device__ __forceinline__ void exchange(u32x4& w) {
  if (kGroup == 128) return;
  uint32_t w0 = w.x, w1 = w.y, w2 = w.z, w3 = w.w;
  swap32(w0, w2);
  swap32(w1, w3);
  if (kGroup == 32) {
    swap16(w0, w1);
    swap16(w2, w3);
  }
  w = u32x4{w0, w1, w2, w3};
}

// Logits of up to 16 hidden states (grid y) by tiles of kTiles * 16 head rows (grid x, in turn).
//
// The waves of a workgroup share the columns, kChunks chunks each, and keep their part of the hidden
// states in registers, so a head row streams through once: 16 bytes a lane, widened to 16 + q by one
// shift and one and-or for two codes, straight into the matrix instructions (hidden states as rows,
// head rows as columns).  Each group's sum starts at -24 times the sum of its hidden values, which leaves
// sum (q - 8) h: every product is exact and all sums are fp32.  A lane then holds four hidden states'
// sums for one head row, so a group's scale is one value a lane; a tile's scales are loaded side by side
// and handed out through LDS.  The waves' sums meet in LDS.
//
// Every 16 states read the head again (64 states of 128256 x 4096: 211 us, 16 of them 61).
//
// Bound by HBM, less what a tile's barrier, sums and stores leave uncovered: one state through 128256 x 4096 in
// groups of 128 49 us (5.5 TB/s), 16 states in groups of 64 59 us (5.1 TB/s; one state in
// those groups 53; all-zero states are faster, 59 where others took 66 in the same run), groups of 32 for
// one state 57 us, 32000 x 2048 9.5 us.  Measured and not
// kept: two tiles in registers (52 us against 50), eight waves with four chunks each in two
// workgroups a CU (56 against 50), non-temporal codes (53 against 49: two loads share a
// 128-byte line), neighbouring tiles to a workgroup (52), the sums shared by all waves (50).
template <typename S, typename T, int kGroup, int kChunks, int kTiles, int kMost>
__global__ void __launch_bounds__(kMost * kWave, 4)
head_logits_kernel(const uint16_t* __restrict__ hidden, int64_t B, uint32_t K, int64_t hidden_stride,
                   const uint8_t* __restrict__ codes, const S* __restrict__ scales, uint32_t V,
                   T* __restrict__ logits, int64_t row_stride, uint32_t waves) {
  constexpr int kGroups = kChunk / kGroup;           // groups of a chunk
  constexpr int kPerGroup = 4 / kGroups;             // matrix instructions of a group
  constexpr uint32_t kRows = kTiles * kTileRows;
  constexpr int kOwnScales = kRows * kChunks * kGroups / kWave;   // of a tile, that a lane loads
  static_assert(kOwnScales * kWave == kRows * kChunks * kGroups, "a tile's scales fill the lanes");
  __shared__ float sums[2][kMost][kTiles * kWave * 4];
  __shared__ float tile_scales[2][kRows * (kMost * kChunks * kGroups + 1)];
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, threads = waves * kWave;
  const uint32_t r = lane % 16, quarter = lane / 16;
  const int64_t b0 = static_cast<int64_t>(blockIdx.y) * 16;
  const uint32_t batch = static_cast<uint32_t>(B - b0 < 16 ? B - b0 : 16);

  // A tile starts at row v0: the last one at V - kRows, where it meets rows of the one before it.
  const uint32_t tiles = (V + kRows - 1) / kRows;
  const uint32_t last = V > kRows ? V - kRows : 0u;
  const uint32_t groups = K / kGroup, row_bytes = K / 2;
  uint32_t code_at[kTiles][kChunks];                 // from the tile's first row
#pragma unroll
  for (int q = 0; q < kChunks; ++q)
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
      // columns beyond the last meet hidden values of 0
      code_at[t][q] = min(t * kTileRows + r, V - 1) * row_bytes +
                      min((wave * kChunks + q) * (kChunk / 2) + quarter * 16, row_bytes - 16);
  u32x4 words[kTiles][kChunks];
  const auto load = [&](uint32_t tile) {
    const uint8_t* code = codes + static_cast<uint64_t>(min(tile * kRows, last)) * row_bytes;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int q = 0; q < kChunks; ++q) words[t][q] = *reinterpret_cast<const u32x4_memory*>(code + code_at[t][q]);
  };
  // The tile after `tile` in turn; past the end it is `tile` again, not nothing: with a branch around its
  // loads the compiler would wait for every load before each use.
  const auto next_of = [&](uint32_t tile) { return tile + gridDim.x < tiles ? tile + gridDim.x : tile; };
  const uint32_t of_tile = min(kRows, V) * groups;   // scales of a tile, side by side
  // a place for every group that the waves' chunks could hold, those beyond K with a scale of 0;
  // an odd stride: a column of 16 rows falls into 16 LDS banks
  const uint32_t scale_stride = waves * (kChunks * kGroups) | 1u;
  S own_scale[kOwnScales];
  const auto load_scales = [&](uint32_t tile) {
    const S* scale = scales + static_cast<uint64_t>(min(tile * kRows, last)) * groups;
#pragma unroll
    for (int i = 0; i < kOwnScales; ++i) own_scale[i] = scale[min(threadIdx.x + i * threads, of_tile - 1)];
  };
  const auto put_scales = [&](float* to) {
#pragma unroll
    for (int i = 0; i < kOwnScales; ++i) {
      const uint32_t n = threadIdx.x + i * threads;
      if (n < of_tile) to[n / groups * scale_stride + n % groups] = logit_of(own_scale[i]);
    }
  };

  load_scales(blockIdx.x);
  load(blockIdx.x);

  u32x4 h[kChunks][4];
  // held where there are few groups; else it is summed again by a second matrix instruction
  constexpr bool kHold = kChunks * kGroups <= 4 && kChunks <= 2;
  f32x4 base[kChunks][kGroups];
  const u32x4 minus24 = {0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u};
  // every load is made, from a place inside the states, so that all are on their way together
#pragma unroll
  for (int q = 0; q < kChunks; ++q)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Source at = source_of<kGroup>(i, quarter);
      const uint32_t k = (wave * kChunks + q) * kChunk + at.q * 32 + at.d * 8;
      h[q][i] = *reinterpret_cast<const u32x4_memory*>(hidden + (b0 + min(r, batch - 1)) * hidden_stride +
                                                       min(k, K - 8));
    }
  for (uint32_t i = threadIdx.x; i < kTiles * kWave * 4; i += threads)
    for (uint32_t n = waves; n < kMost; ++n) sums[0][n][i] = sums[1][n][i] = 0.0f;   // of no wave
  for (uint32_t i = threadIdx.x; i < kRows * scale_stride; i += threads)
    if (i % scale_stride >= groups) tile_scales[0][i] = tile_scales[1][i] = 0.0f;
  put_scales(tile_scales[0]);
  load_scales(next_of(blockIdx.x));
#pragma unroll
  for (int q = 0; q < kChunks; ++q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Source at = source_of<kGroup>(i, quarter);
      const bool some = r < batch && (wave * kChunks + q) * kChunk + at.q * 32 + at.d * 8 < K;
      const u32x4 x = in_code_order(h[q][i]);
      h[q][i] = u32x4{some ? x.x : 0u, some ? x.y : 0u, some ? x.z : 0u, some ? x.w : 0u};
    }
    if (!kHold) continue;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      base[q][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < kPerGroup; ++i) base[q][g] = mfma(h[q][g * kPerGroup + i], minus24, base[q][g]);
    }
  }
  uint32_t sixteens = kSixteens;
  asm volatile("" : "+v"(sixteens));
  __syncthreads();

  uint32_t turn = 0;
  for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      f32x4 total = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int q = 0; q < kChunks; ++q) {
        u32x4 w = words[t][q];
        exchange<kGroup>(w);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          const float scale = tile_scales[turn][(t * kTileRows + r) * scale_stride + (wave * kChunks + q) * kGroups + g];
          f32x4 of_group = {0.0f, 0.0f, 0.0f, 0.0f};
          if (kHold) {
            of_group = base[q][g];
          } else {
#pragma unroll
            for (int i = 0; i < kPerGroup; ++i) of_group = mfma(h[q][g * kPerGroup + i], minus24, of_group);
          }
#pragma unroll
          for (int i = 0; i < kPerGroup; ++i)
            of_group = mfma(h[q][g * kPerGroup + i], widened(word[g * kPerGroup + i], sixteens), of_group);
#pragma unroll
          for (int i = 0; i < 4; ++i) total[i] = __builtin_fmaf(of_group[i], scale, total[i]);
        }
      }
      *reinterpret_cast<f32x4*>(&sums[turn][wave][(t * kWave + lane) * 4]) = total;
    }
    __builtin_amdgcn_sched_barrier(0);   // into the registers just read, not into others to be copied later
    load(next_of(tile));
    __builtin_amdgcn_sched_barrier(0);
    put_scales(tile_scales[turn ^ 1]);
    load_scales(next_of(next_of(tile)));
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    const uint32_t v0 = min(tile * kRows, last);
    for (uint32_t i = threadIdx.x; i < kTiles * kWave * 4; i += threads) {
      // place i: head row (i / 4) % 16 of its 16, hidden state 4 * (i / 64 % 4) + i % 4
      const uint32_t b = i / 64 % 4 * 4 + i % 4;
      const uint32_t v = v0 + i / (kWave * 4) * kTileRows + i / 4 % 16;
      if (b >= batch || v >= V || v < tile * kRows) continue;
      float x = sums[turn][0][i];
#pragma unroll
      for (int n = 1; n < kMost; ++n) x += sums[turn][n][i];
      put_logit(logits + (b0 + b) * row_stride + v, x);
    }
    turn ^= 1;
  }
}

template <typename S, typename T, int kGroup, int kChunks, int kTiles, int kMost>
void launch_head_shape(const void* hidden, int64_t B, uint32_t K, int64_t hidden_stride, const uint8_t* codes,
                       const void* scales, uint32_t V, void* logits, int64_t row_stride, hipStream_t stream) {
  const uint32_t waves = (K + kChunks * kChunk - 1) / (kChunks * kChunk);
  const uint32_t tiles = (V + kTiles * kTileRows - 1) / (kTiles * kTileRows);
  const uint32_t resident = 256u * (kHeadWaves / waves);
  const dim3 grid(tiles < resident ? tiles : resident, static_cast<uint32_t>((B + 15) / 16));
  head_logits_kernel<S, T, kGroup, kChunks, kTiles, kMost><<<grid, waves * kWave, 0, stream>>>(
      static_cast<const uint16_t*>(hidden), B, K, hidden_stride, codes, static_cast<const S*>(scales), V,
      static_cast<T*>(logits), row_stride, waves);
}

// Few columns are shared by few waves, so that a CU holds up to 16 waves (their hidden states fill its registers)
// in 4, 2 or 1 workgroups: 16 where K is 1024, 2048, 4096 or 8192, as few as 9 between them (2304, 4608).  One state through
// 128256 rows in groups of 128, from a graph: K = 1024 16.5 us (4.3 TB/s), 2048 28.5-29.8 (4.7-4.9), 2304 31.3-32.8 (4.8-5.0),
// 2560 33.3 (5.2), 3584 45.7 (5.4), 4096 53-54 (5.2), 4608 63.8 (4.9), 5120 66.6 (5.3), 7168 88.1 (5.6), 8192 104.1 (5.4).
// The forms against each other: two chunks a wave with sums for 16 waves instead of 4, K = 1024, 20.5 us; instead of 8, 2048,
// 28.7.  Four chunks a wave: 1024 27.7, 2048 33.5, 3584 48.2, 4096 53.3, but 16 states in groups of 64 69.3 (two 61.4).  In
// groups of 32 four chunks need 6 vector registers more than there are (28 bytes of scratch a lane): K = 4608 107 us,
// 8192 152 (4.3 TB/s) where 4096 with two chunks takes 60 (5.5).
template <typename S, typename T, int kGroup>
void launch_head_group(const void* hidden, int64_t B, uint32_t K, int64_t hidden_stride, const uint8_t* codes,
                       const void* scales, uint32_t V, void* logits, int64_t row_stride, hipStream_t stream) {
  auto* launch = K <= 4 * 2 * kChunk    ? launch_head_shape<S, T, kGroup, 2, 2, 4>
                 : K <= 8 * 2 * kChunk  ? launch_head_shape<S, T, kGroup, 2, 2, 8>
                 : K <= 16 * 2 * kChunk ? launch_head_shape<S, T, kGroup, 2, 2, 16>
                                        : launch_head_shape<S, T, kGroup, 4, 1, 16>;
  launch(hidden, B, K, hidden_stride, codes, scales, V, logits, row_stride, stream);
}

template <typename S, typename T>
void launch_head(const void* hidden, int64_t B, int64_t K_, int64_t hidden_stride, const uint8_t* codes,
                 const void* scales, int64_t group, int64_t V_, void* logits, int64_t row_stride,
                 hipStream_t stream) {
  const auto K = static_cast<uint32_t>(K_), V = static_cast<uint32_t>(V_);
  if (group == 32)
    launch_head_group<S, T, 32>(hidden, B, K, hidden_stride, codes, scales, V, logits, row_stride, stream);
  else if (group == 64)
    launch_head_group<S, T, 64>(hidden, B, K, hidden_stride, codes, scales, V, logits, row_stride, stream);
  else
    launch_head_group<S, T, 128>(hidden, B, K, hidden_stride, codes, scales, V, logits, row_stride, stream);
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
  if (B > INT64_MAX / 4 / row_stride || B > INT64_MAX / 4 / hidden_stride || B > 16 * kMaxGridY)
    return SBW_ERR_UNSUPPORTED;
  const sbw_status_t s = check_device();
  if (s != SBW_OK) return s;
  const auto st = static_cast<hipStream_t>(stream);
  auto* launch = scale_dtype == SBW_F32
                     ? (dtype == SBW_F32 ? launch_head<float, float> : launch_head<float, uint16_t>)
                     : (dtype == SBW_F32 ? launch_head<uint16_t, float> : launch_head<uint16_t, uint16_t>);
  launch(hidden, B, K, hidden_stride, codes, scales, group, V, logits, row_stride, st);
  return after_launch();
}
