// Matrices in 8-bit floating point (e4m3) with a scale for each block of 128, and their product
// (sbw_step.h).  Part of sbw_library.hip.
#include "sbw_step.h"

namespace sbw {
namespace {

constexpr int kBlock = 128;                       // columns that share a scale
constexpr float kLargestCode = 448.0f;            // of e4m3
constexpr int64_t kMostStride = (1 << 23) - 1;    // of a matrix of codes: 256 rows lie within 2^31 bytes
constexpr int64_t kMostRows = (int64_t{1} << 30) - 1;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef u32x4 u32x4_bytes __attribute__((aligned(1)));
typedef u32x2 u32x2_bytes __attribute__((aligned(1)));

__host__ __device__ inline int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

// ---------------------------------------------------------------------------
// Quantisation.  A block's scale takes its largest finite magnitude to 448 or below; a code is its value
// times the reciprocal of the scale, rounded once to e4m3.  Powers of two as scales make both products exact.
// ---------------------------------------------------------------------------
struct BlockScale {
  float inverse;
  uint32_t stored;   // the exponent's byte, or the bits of an fp32 scale
};
template <bool kE8>
__device__ __forceinline__ BlockScale scale_of(uint32_t largest) {   // bits of a magnitude
  if constexpr (kE8) {
    // 2^e with 448 2^e = 1.75 2^(8+e) at or above the largest
    const int e = static_cast<int>(largest >> 23) - 135 + ((largest & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    const int bounded = max(e, -127);
    return BlockScale{__uint_as_float(static_cast<uint32_t>(127 - bounded) << 23), static_cast<uint32_t>(bounded + 127)};
  } else {
    const float scale = fmaxf(__uint_as_float(largest) / kLargestCode, 1.17549435e-38f);
    return BlockScale{1.0f / scale, __float_as_uint(scale)};
  }
}
template <bool kE8>
__device__ __forceinline__ void put_scale(void* scales, int64_t at, uint32_t stored) {
  if constexpr (kE8) static_cast<uint8_t*>(scales)[at] = static_cast<uint8_t>(stored);
  else static_cast<uint32_t*>(scales)[at] = stored;
}

// |x| as bits, 0 for an infinity or NaN
__device__ __forceinline__ uint32_t finite_size(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}
__device__ __forceinline__ float scaled_value(float x, float inverse) {
  return finite_size(x) == 0u && x != 0.0f ? __uint_as_float(0x7FC00000u) : x * inverse;
}
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d, float inverse) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled_value(a, inverse), scaled_value(b, inverse), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled_value(c, inverse), scaled_value(d, inverse), w, true);
  return static_cast<uint32_t>(w);
}

// Eight neighbours of a row; those from `columns` on are 0.
struct Eight {
  float x[8];
};
__device__ __forceinline__ Eight load_eight(const float* p, int64_t columns) {
  Eight v;
  if (columns >= 8) {
    const f32x4 lo = *reinterpret_cast<const f32x4_memory*>(p), hi = *reinterpret_cast<const f32x4_memory*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) v.x[e] = lo[e], v.x[e + 4] = hi[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v.x[e] = e < columns ? p[e] : 0.0f;
  }
  return v;
}
__device__ __forceinline__ Eight load_eight(const uint16_t* p, int64_t columns) {
  Eight v;
  if (columns >= 8) {
    const u32x4 w = *reinterpret_cast<const u32x4_memory*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v.x[2 * e] = __uint_as_float(w[e] << 16), v.x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v.x[e] = e < columns ? logit_of(p[e]) : 0.0f;
  }
  return v;
}

// Blocks of one row: sixteen lanes a block, eight values a lane.  `across` (a power of two, at most 16) of a
// workgroup's sixteen groups of lanes take neighbouring blocks of a row, the others the next rows.
template <typename T, bool kE8>
__global__ void __launch_bounds__(kThreads)
quantize_rows_kernel(const T* __restrict__ x, int64_t M, int64_t K, int64_t row_stride, uint32_t across,
                     uint8_t* __restrict__ codes, int64_t codes_stride, void* __restrict__ scales) {
  const uint32_t group = threadIdx.x / 16, at = threadIdx.x % 16 * 8;
  const int64_t block = static_cast<int64_t>(blockIdx.x) * across + group % across;
  const int64_t blocks = (K + kBlock - 1) / kBlock, column = block * kBlock + at;
  if (block >= blocks) return;                    // whole groups of sixteen lanes
  const int64_t rows = kThreads / 16 / across;    // of a workgroup
  for (int64_t row = blockIdx.y * rows + group / across; row < M; row += gridDim.y * rows) {
    const Eight v = load_eight(x + row * row_stride + column, K - column);
    uint32_t largest = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) largest = max(largest, finite_size(v.x[e]));
    const BlockScale s = scale_of<kE8>(row_largest(largest));
    const u32x2 w = {codes_of(v.x[0], v.x[1], v.x[2], v.x[3], s.inverse), codes_of(v.x[4], v.x[5], v.x[6], v.x[7], s.inverse)};
    uint8_t* to = codes + row * codes_stride + column;
    if (column + 8 <= K) {
      *reinterpret_cast<u32x2_bytes*>(to) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (column + e < K) to[e] = static_cast<uint8_t>(w[e / 4] >> e % 4 * 8);
    }
    if (at == 0) put_scale<kE8>(scales, row * blocks + block, s.stored);
  }
}

// What a call writes in one orientation; codes is null where it is not asked for.
struct Quantized {
  uint8_t* codes;
  int64_t stride;
  void* scales;
};

// Tiles of 128 x 128: blocks of 128 rows, and the transposed orientation.  A lane holds eight neighbouring
// columns of four neighbouring rows, twice, so that four rows' codes of a column make a word of LDS.
template <typename T, bool kE8, bool kSquare>
__global__ void __launch_bounds__(kThreads)
quantize_tiles_kernel(const T* __restrict__ x, int64_t M, int64_t K, int64_t row_stride, Quantized straight,
                      Quantized transposed) {
  constexpr uint32_t kStride = 33;                // words of a column in LDS: lanes 8 columns apart meet in pairs of banks
  __shared__ uint32_t turned[kBlock * kStride];
  __shared__ uint32_t largest_of[4][kBlock];
  const uint32_t lane16 = threadIdx.x % 16, group = threadIdx.x / 16, wave = threadIdx.x / kWave;
  const int64_t column = static_cast<int64_t>(blockIdx.x) * kBlock + lane16 * 8;
  const int64_t column_blocks = (K + kBlock - 1) / kBlock, row_blocks = (M + kBlock - 1) / kBlock;
  const auto row_of = [&](int i) { return static_cast<int64_t>(group * 4 + i / 4 * 64 + i % 4); };
  for (int64_t row_block = blockIdx.y; row_block < row_blocks; row_block += gridDim.y) {
    const int64_t row0 = row_block * kBlock;
    Eight v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = row0 + row_of(i);
      v[i] = load_eight(x + (row < M ? row : M - 1) * row_stride + min(column, K - 1), row < M ? K - column : 0);
    }
    BlockScale square;
    if (kSquare) {
      uint32_t largest = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) largest = max(largest, finite_size(v[i].x[e]));
      largest = wave_highest(largest);
      if (threadIdx.x % kWave == 0) largest_of[wave][0] = largest;
      __syncthreads();
      largest = max(max(largest_of[0][0], largest_of[1][0]), max(largest_of[2][0], largest_of[3][0]));
      square = scale_of<kE8>(largest);
      if (threadIdx.x == 0) {
        if (straight.codes != nullptr) put_scale<kE8>(straight.scales, row_block * column_blocks + blockIdx.x, square.stored);
        if (transposed.codes != nullptr) put_scale<kE8>(transposed.scales, blockIdx.x * row_blocks + row_block, square.stored);
      }
    }
    if (straight.codes != nullptr) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + row_of(i);
        BlockScale s = square;
        if (!kSquare) {
          uint32_t largest = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) largest = max(largest, finite_size(v[i].x[e]));
          s = scale_of<kE8>(row_largest(largest));
        }
        if (row >= M || column >= K) continue;
        const u32x2 w = {codes_of(v[i].x[0], v[i].x[1], v[i].x[2], v[i].x[3], s.inverse),
                         codes_of(v[i].x[4], v[i].x[5], v[i].x[6], v[i].x[7], s.inverse)};
        uint8_t* to = straight.codes + row * straight.stride + column;
        if (column + 8 <= K) {
          *reinterpret_cast<u32x2_bytes*>(to) = w;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (column + e < K) to[e] = static_cast<uint8_t>(w[e / 4] >> e % 4 * 8);
        }
        if (!kSquare && lane16 == 0) put_scale<kE8>(straight.scales, row * column_blocks + blockIdx.x, s.stored);
      }
    }
    if (transposed.codes != nullptr) {
      float inverse[8];
      if (!kSquare) {
        // a column's largest: a lane's eight rows, the wave's four groups of lanes, the four waves
        uint32_t largest[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          largest[e] = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) largest[e] = max(largest[e], finite_size(v[i].x[e]));
          largest[e] = max(largest[e], __shfl_xor(largest[e], 16));
          largest[e] = max(largest[e], __shfl_xor(largest[e], 32));
          if (threadIdx.x % kWave < 16) largest_of[wave][lane16 * 8 + e] = largest[e];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t c = lane16 * 8 + e;
          const BlockScale s = scale_of<kE8>(max(max(largest_of[0][c], largest_of[1][c]), max(largest_of[2][c], largest_of[3][c])));
          inverse[e] = s.inverse;
          if (group == 0 && column + e < K) put_scale<kE8>(transposed.scales, (column + e) * row_blocks + row_block, s.stored);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) inverse[e] = square.inverse;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          turned[(lane16 * 8 + e) * kStride + group + h * 16] =
              codes_of(v[4 * h].x[e], v[4 * h + 1].x[e], v[4 * h + 2].x[e], v[4 * h + 3].x[e], inverse[e]);
      __syncthreads();
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const uint32_t c = threadIdx.x / 8 + p * 32, part = threadIdx.x % 8;
        const int64_t to_row = static_cast<int64_t>(blockIdx.x) * kBlock + c, to_column = row0 + part * 16;
        if (to_row >= K || to_column >= M) continue;
        u32x4 w;
#pragma unroll
        for (int d = 0; d < 4; ++d) w[d] = turned[c * kStride + part * 4 + d];
        uint8_t* to = transposed.codes + to_row * transposed.stride + to_column;
        if (to_column + 16 <= M) {
          *reinterpret_cast<u32x4_bytes*>(to) = w;
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (to_column + e < M) to[e] = static_cast<uint8_t>(w[e / 4] >> e % 4 * 8);
        }
      }
    }
    __syncthreads();
  }
}

template <typename T, bool kE8>
void launch_quantize(const void* x_, int64_t M, int64_t K, int64_t row_stride, bool square, Quantized straight,
                     Quantized transposed, hipStream_t stream) {
  const T* x = static_cast<const T*>(x_);
  const int64_t blocks = blocks_of(K);
  if (!square && transposed.codes == nullptr) {
    uint32_t across = 1;
    while (across < 16 && across < blocks) across *= 2;
    const int64_t rows = 16 / across, groups = (M + rows - 1) / rows;
    const dim3 grid(static_cast<uint32_t>((blocks + across - 1) / across),
                    static_cast<uint32_t>(groups < kMaxGridY ? groups : kMaxGridY));
    quantize_rows_kernel<T, kE8><<<grid, kThreads, 0, stream>>>(x, M, K, row_stride, across, straight.codes,
                                                               straight.stride, straight.scales);
    return;
  }
  const int64_t row_blocks = blocks_of(M);
  const dim3 grid(static_cast<uint32_t>(blocks), static_cast<uint32_t>(row_blocks < kMaxGridY ? row_blocks : kMaxGridY));
  auto* kernel = square ? quantize_tiles_kernel<T, kE8, true> : quantize_tiles_kernel<T, kE8, false>;
  kernel<<<grid, kThreads, 0, stream>>>(x, M, K, row_stride, straight, transposed);
}

// ---------------------------------------------------------------------------
// Product.  out[m, n] = sum over blocks j of sa[m, j] sb[n, j] (sum over the block of a[m, k] b[n, k]).
//
// The matrix instructions of 8-bit floating point take eight neighbouring products of a row together: each is cut off,
// towards zero, 13 bits below the power of two of the largest of them, then they are added to an fp32 sum (measured with
// single products at every distance; of 16x16x32, 16x16x128 and 32x32x64 alike).  Of normally distributed rows
// that is 1.4e-5 of a result, a hundredth of what its rounding to bf16 takes, so a product of type bf16 takes
// them.  One of type fp32 takes those of bf16 instead, at half the rate, on codes widened in registers: products
// are exact then and every sum is fp32.
//
// Powers of two as scales go into the 8-bit instructions; other scales, and all in front of an fp32 result, multiply a
// block's sum, by one fma for each element and block.
// ---------------------------------------------------------------------------
// One side of a product: a row's codes, and its blocks' scales, those of row / block_rows.
struct Side {
  const uint8_t* codes;
  int64_t rows, stride;
  const void* scales;
  uint32_t row_shift;      // log2 of block_rows
};

// Sixteen codes of a row from column k on; 0 from column K on.
__device__ __forceinline__ u32x4 load_codes(const uint8_t* row, int64_t k, int64_t K) {
  if (k + 16 <= K) return *reinterpret_cast<const u32x4_bytes*>(row + k);
  u32x4 w = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (k + e < K) w[e / 4] |= static_cast<uint32_t>(row[k + e]) << e % 4 * 8;
  return w;
}
// 2^(e - 127)
__device__ __forceinline__ float power_of(uint32_t e) {
  return __uint_as_float(e == 0 ? 0x00400000u : e == 255 ? 0x7FC00000u : e << 23);
}
// A scale for the instructions (kRaw), or as the bits of an fp32 number.
template <bool kE8, bool kRaw>
__device__ __forceinline__ uint32_t load_scale(const Side& s, int64_t row, int64_t block, int64_t blocks) {
  const int64_t at = (min(row, s.rows - 1) >> s.row_shift) * blocks + block;
  if constexpr (!kE8) return static_cast<const uint32_t*>(s.scales)[at];
  else if constexpr (kRaw) return static_cast<const uint8_t*>(s.scales)[at];
  else return __float_as_uint(power_of(static_cast<const uint8_t*>(s.scales)[at]));
}

// A lane's 32 codes of a row (A and B alike): 64 columns of 32 rows in one instruction, or four of bf16.
struct Codes {
  u32x4 lo, hi;
};
__device__ __forceinline__ i32x8 as_operand(Codes c) {
  return i32x8{static_cast<int>(c.lo.x), static_cast<int>(c.lo.y), static_cast<int>(c.lo.z), static_cast<int>(c.lo.w),
               static_cast<int>(c.hi.x), static_cast<int>(c.hi.y), static_cast<int>(c.hi.z), static_cast<int>(c.hi.w)};
}
struct Widened {
  bf16x8 part[4];
};
__device__ __forceinline__ Widened widened(Codes c) {
  Widened w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const uint32_t four = i < 2 ? c.lo[2 * i + d] : c.hi[2 * (i - 2) + d];
      const bf16x2 first = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, 1.0f, false);
      const bf16x2 second = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, 1.0f, true);
      w.part[i][4 * d] = first.x, w.part[i][4 * d + 1] = first.y;
      w.part[i][4 * d + 2] = second.x, w.part[i][4 * d + 3] = second.y;
    }
  return w;
}

// Where a tile's 16-byte part c of row r stands in LDS: parts are permuted by the row, so that sixteen lanes
// that read one part of sixteen rows meet every bank once.
__device__ __forceinline__ uint32_t place_of(uint32_t r, uint32_t c) { return r * 8 + (c ^ (r >> 1 & 7u)); }

// Any sizes and alignments: tiles of 128 x 128 by four waves of 64 x 64, the next step's codes on their way in
// registers while this one's are multiplied.
template <typename Out, bool kE8>
__global__ void __launch_bounds__(kThreads)
product_any_kernel(Side a, Side b, int64_t K, Out* __restrict__ out, int64_t out_stride) {
  constexpr uint32_t kTile = 128;
  constexpr bool kExact = sizeof(Out) == 4, kInside = kE8 && !kExact;   // scales inside the instructions
  __shared__ u32x4 codes[2][2][kTile * 8];
  __shared__ uint32_t tile_scales[2][2][kTile];
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint32_t r32 = lane % 32, half = lane / 32;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * kTile, n0 = static_cast<int64_t>(blockIdx.x) * kTile;
  const int64_t blocks = (K + kBlock - 1) / kBlock;
  u32x4 held[2][4];
  uint32_t held_scale;
  const auto load = [&](int64_t block) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t r = threadIdx.x / 8 + i * 32, c = threadIdx.x % 8;
      const int64_t k = block * kBlock + c * 16;
      held[0][i] = load_codes(a.codes + min(m0 + r, a.rows - 1) * a.stride, k, K);
      held[1][i] = load_codes(b.codes + min(n0 + r, b.rows - 1) * b.stride, k, K);
    }
    held_scale = threadIdx.x < kTile ? load_scale<kE8, kInside>(a, m0 + threadIdx.x, block, blocks)
                                     : load_scale<kE8, kInside>(b, n0 + threadIdx.x - kTile, block, blocks);
  };
  const auto put = [&](uint32_t turn) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t r = threadIdx.x / 8 + i * 32, c = threadIdx.x % 8;
      codes[turn][0][place_of(r, c)] = held[0][i];
      codes[turn][1][place_of(r, c)] = held[1][i];
    }
    tile_scales[turn][threadIdx.x / kTile][threadIdx.x % kTile] = held_scale;
  };
  const uint32_t row_a = wave / 2 * 64, row_b = wave % 2 * 64;
  f32x16 total[2][2] = {};
  load(0);
  put(0);
  uint32_t turn = 0;
  for (int64_t block = 0; block < blocks; ++block, turn ^= 1) {
    __syncthreads();
    if (block + 1 < blocks) load(block + 1);
    f32x16 part[2][2] = {};
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const auto fragment = [&](uint32_t side, uint32_t row) {
        return Codes{codes[turn][side][place_of(row, kk * 4 + half * 2)],
                     codes[turn][side][place_of(row, kk * 4 + half * 2 + 1)]};
      };
      Codes x[2], y[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        x[t] = fragment(0, row_a + t * 32 + r32);
        y[t] = fragment(1, row_b + t * 32 + r32);
      }
      if constexpr (kExact) {
        Widened wx[2] = {widened(x[0]), widened(x[1])}, wy[2] = {widened(y[0]), widened(y[1])};
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              part[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wx[i].part[s], wy[j].part[s], part[i][j], 0, 0, 0);
        continue;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if constexpr (kInside)
            total[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                as_operand(x[i]), as_operand(y[j]), total[i][j], 0, 0, 0, tile_scales[turn][0][row_a + i * 32 + r32], 0,
                tile_scales[turn][1][row_b + j * 32 + r32]);
          else
            part[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(as_operand(x[i]), as_operand(y[j]), part[i][j],
                                                                         0, 0, 0, 0x7F7F7F7F, 0, 0x7F7F7F7F);
        }
    }
    if constexpr (!kInside) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float sb = __uint_as_float(tile_scales[turn][1][row_b + j * 32 + r32]);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float sa = __uint_as_float(tile_scales[turn][0][row_a + i * 32 + e / 4 * 8 + half * 4 + e % 4]);
            total[i][j][e] = __builtin_fmaf(part[i][j][e], sa * sb, total[i][j][e]);
          }
        }
    }
    if (block + 1 < blocks) put(turn ^ 1);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int64_t m = m0 + row_a + i * 32 + e / 4 * 8 + half * 4 + e % 4, n = n0 + row_b + j * 32 + r32;
        if (m < a.rows && n < b.rows) put_logit(out + m * out_stride + n, total[i][j][e]);
      }
}

template <typename Out, bool kE8>
void launch_product(Side a, Side b, int64_t K, void* out, int64_t out_stride, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(blocks_of(b.rows)), static_cast<uint32_t>(blocks_of(a.rows)));
  product_any_kernel<Out, kE8><<<grid, kThreads, 0, stream>>>(a, b, K, static_cast<Out*>(out), out_stride);
}

}  // namespace
}  // namespace sbw

extern "C" {

sbw_status_t sbw_quantize_fp8(const void* x, sbw_dtype_t dtype, int64_t M, int64_t K, int64_t row_stride,
                              int64_t block_rows, sbw_scale_t scale_type, uint8_t* codes, int64_t codes_stride,
                              void* scales, uint8_t* codes_t, int64_t codes_t_stride, void* scales_t, void* stream) {
  if (M < 0 || K < 0 || row_stride < K) return SBW_ERR_INVALID_ARG;
  if (block_rows != 1 && block_rows != kBlock) return SBW_ERR_UNSUPPORTED;
  if ((dtype != SBW_F32 && dtype != SBW_BF16) || (scale_type != SBW_SCALE_E8M0 && scale_type != SBW_SCALE_F32))
    return SBW_ERR_UNSUPPORTED;
  if ((codes != nullptr && codes_stride < K) || (codes_t != nullptr && codes_t_stride < M)) return SBW_ERR_INVALID_ARG;
  if (M > kMostRows || K > kMostRows) return SBW_ERR_UNSUPPORTED;
  if (M == 0 || K == 0) return SBW_OK;
  if (x == nullptr || (codes == nullptr && codes_t == nullptr) || (codes == nullptr) != (scales == nullptr) ||
      (codes_t == nullptr) != (scales_t == nullptr))
    return SBW_ERR_INVALID_ARG;
  if (M > INT64_MAX / 4 / row_stride || (codes != nullptr && M > INT64_MAX / codes_stride) ||
      (codes_t != nullptr && K > INT64_MAX / codes_t_stride))
    return SBW_ERR_UNSUPPORTED;
  const sbw_status_t s = check_device();
  if (s != SBW_OK) return s;
  const Quantized straight{codes, codes_stride, scales}, transposed{codes_t, codes_t_stride, scales_t};
  auto* launch = scale_type == SBW_SCALE_E8M0
                     ? (dtype == SBW_F32 ? launch_quantize<float, true> : launch_quantize<uint16_t, true>)
                     : (dtype == SBW_F32 ? launch_quantize<float, false> : launch_quantize<uint16_t, false>);
  launch(x, M, K, row_stride, block_rows != 1, straight, transposed, static_cast<hipStream_t>(stream));
  return after_launch();
}

int64_t sbw_matmul_fp8_workspace(int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || N <= 0 || K <= 0) return 0;
  return 0;
}

sbw_status_t sbw_matmul_fp8(const uint8_t* a, int64_t M, int64_t a_stride, const void* a_scales, int64_t a_block_rows,
                            const uint8_t* b, int64_t N, int64_t b_stride, const void* b_scales, int64_t b_block_rows,
                            int64_t K, sbw_scale_t scale_type, void* out, sbw_dtype_t dtype, int64_t out_stride,
                            uint64_t* workspace, void* stream) {
  if (M < 0 || N < 0 || K <= 0 || a_stride < K || b_stride < K || out_stride < N) return SBW_ERR_INVALID_ARG;
  if ((a_block_rows != 1 && a_block_rows != kBlock) || (b_block_rows != 1 && b_block_rows != kBlock))
    return SBW_ERR_UNSUPPORTED;
  if ((dtype != SBW_F32 && dtype != SBW_BF16) || (scale_type != SBW_SCALE_E8M0 && scale_type != SBW_SCALE_F32))
    return SBW_ERR_UNSUPPORTED;
  if (a_stride > kMostStride || b_stride > kMostStride) return SBW_ERR_UNSUPPORTED;
  if (M > kBlock * kMaxGridY || N > kMostRows) return SBW_ERR_UNSUPPORTED;
  if (M == 0 || N == 0) return SBW_OK;
  if (a == nullptr || b == nullptr || a_scales == nullptr || b_scales == nullptr || out == nullptr)
    return SBW_ERR_INVALID_ARG;
  if (M > INT64_MAX / 4 / out_stride) return SBW_ERR_UNSUPPORTED;
  if (workspace == nullptr && sbw_matmul_fp8_workspace(M, N, K) > 0) return SBW_ERR_INVALID_ARG;
  const sbw_status_t s = check_device();
  if (s != SBW_OK) return s;
  const Side left{a, M, a_stride, a_scales, a_block_rows == 1 ? 0u : 7u};
  const Side right{b, N, b_stride, b_scales, b_block_rows == 1 ? 0u : 7u};
  auto* launch = scale_type == SBW_SCALE_E8M0
                     ? (dtype == SBW_F32 ? launch_product<float, true> : launch_product<uint16_t, true>)
                     : (dtype == SBW_F32 ? launch_product<float, false> : launch_product<uint16_t, false>);
  launch(left, right, K, out, out_stride, static_cast<hipStream_t>(stream));
  return after_launch();
}

}  // extern "C"
