// Matrices in 8-bit floating point (e4m3) with a scale for each block of 128, and their product
// (sbw_step.h).  Part of sbw_library.hip.
#include "sbw_step.h"

#include <algorithm>

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
// Infinities and NaN become NaN.
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d, float inverse) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, w, true);
  return static_cast<uint32_t>(w);
}

// Eight neighbours of a row as they stand in memory; those from `columns` on are 0.  Sizes are magnitudes as integers, which
// order like them: of bf16 two to a word.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename T>
struct Eight;
template <>
struct Eight<float> {
  f32x4 lo, hi;
  static constexpr int kSizes = 8;       // words of sizes
  __device__ __forceinline__ float operator[](int e) const { return e < 4 ? lo[e] : hi[e - 4]; }
  __device__ __forceinline__ uint32_t size(int i) const { return __float_as_uint((*this)[i]) & 0x7FFFFFFFu; }
  static __device__ __forceinline__ uint32_t larger_size(uint32_t a, uint32_t b) { return max(a, b); }
  static __device__ __forceinline__ uint32_t bits_of(uint32_t size, int) { return size; }
  static __device__ __forceinline__ uint32_t largest(uint32_t size) { return size; }
};
template <>
struct Eight<uint16_t> {
  u32x4 w;
  static constexpr int kSizes = 4;
  __device__ __forceinline__ float operator[](int e) const { return __uint_as_float(e % 2 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16); }
  __device__ __forceinline__ uint32_t size(int i) const { return w[i] & 0x7FFF7FFFu; }
  static __device__ __forceinline__ uint32_t larger_size(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
  }
  static __device__ __forceinline__ uint32_t bits_of(uint32_t size, int e) { return e % 2 ? size & 0xFFFF0000u : size << 16; }
  static __device__ __forceinline__ uint32_t largest(uint32_t size) { return max(size & 0xFFFF0000u, size << 16); }
};
__device__ __forceinline__ Eight<float> load_eight(const float* p, int64_t columns) {
  if (columns >= 8) return Eight<float>{*reinterpret_cast<const f32x4_memory*>(p), *reinterpret_cast<const f32x4_memory*>(p + 4)};
  Eight<float> v{};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < columns) (e < 4 ? v.lo : v.hi)[e % 4] = p[e];
  return v;
}
__device__ __forceinline__ Eight<uint16_t> load_eight(const uint16_t* p, int64_t columns) {
  if (columns >= 8) return Eight<uint16_t>{*reinterpret_cast<const u32x4_memory*>(p)};
  Eight<uint16_t> v{};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < columns) v.w[e / 2] |= static_cast<uint32_t>(p[e]) << e % 2 * 16;
  return v;
}
// Bits of the largest magnitude; where that is no number, of the largest finite one.
template <typename T>
__device__ __forceinline__ uint32_t largest_size(const Eight<T>& v, bool finite) {
  uint32_t s = 0;
  if (finite) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s = max(s, finite_size(v[e]));
    return s;
  }
#pragma unroll
  for (int i = 0; i < Eight<T>::kSizes; ++i) s = Eight<T>::larger_size(s, v.size(i));
  return Eight<T>::largest(s);
}
template <typename T>
__device__ __forceinline__ void put_eight(uint8_t* to, int64_t columns, const Eight<T>& v, float inverse) {
  const u32x2 w = {codes_of(v[0], v[1], v[2], v[3], inverse), codes_of(v[4], v[5], v[6], v[7], inverse)};
  if (columns >= 8) {
    *reinterpret_cast<u32x2_bytes*>(to) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < columns) to[e] = static_cast<uint8_t>(w[e / 4] >> e % 4 * 8);
  }
}

// Blocks of one row: sixteen lanes a block, eight values a lane, kRowsEach rows on their way together.  `across` (a power of
// two, at most 16) of a workgroup's sixteen groups of lanes take neighbouring blocks of a row, the others the next rows.
// Bound by memory: 8192 x 4096 bf16 17 us, 5.9 TB/s (a row at a time 20.6).
constexpr int kRowsEach = 4;
template <typename T, bool kE8>
__global__ void __launch_bounds__(kThreads)
quantize_rows_kernel(const T* __restrict__ x, int64_t M, int64_t K, int64_t row_stride, uint32_t across,
                     uint8_t* __restrict__ codes, int64_t codes_stride, void* __restrict__ scales) {
  const uint32_t group = threadIdx.x / 16, at = threadIdx.x % 16 * 8;
  const int64_t block = static_cast<int64_t>(blockIdx.x) * across + group % across;
  const int64_t blocks = (K + kBlock - 1) / kBlock, column = block * kBlock + at;
  if (block >= blocks) return;                    // whole groups of sixteen lanes
  const int64_t rows = kThreads / 16 / across;    // of a workgroup at a time
  for (int64_t row0 = blockIdx.y * (rows * kRowsEach) + group / across; row0 < M; row0 += gridDim.y * (rows * kRowsEach)) {
    Eight<T> v[kRowsEach];
#pragma unroll
    for (int i = 0; i < kRowsEach; ++i) {
      const int64_t row = row0 + i * rows;
      v[i] = load_eight(x + min(row, M - 1) * row_stride + min(column, K - 1), K - column);
    }
#pragma unroll
    for (int i = 0; i < kRowsEach; ++i) {
      const int64_t row = row0 + i * rows;
      uint32_t largest = row_largest(largest_size(v[i], false));
      if (__any(largest >= 0x7F800000u)) largest = row_largest(largest_size(v[i], true));
      const BlockScale s = scale_of<kE8>(largest);
      if (row >= M) continue;
      put_eight(codes + row * codes_stride + column, K - column, v[i], s.inverse);
      if (at == 0) put_scale<kE8>(scales, row * blocks + block, s.stored);
    }
  }
}

// What a call writes in one orientation; codes is null where it is not asked for.
struct Quantized {
  uint8_t* codes;
  int64_t stride;
  void* scales;
};

// Tiles of 128 x 128: blocks of 128 rows, and the transposed orientation.  A lane holds eight neighbouring
// columns of four neighbouring rows, twice, so that four rows' codes of a column make a word of LDS.  Bound by memory where one
// orientation is asked for (50257 x 2048 fp32 transposed 94 us, 5.5 TB/s), by its instructions where both are (32000 x 4096 bf16 in blocks of
// 128 rows 94 us, 5.6 TB/s; with magnitudes as floats and rows loaded one after another 190).
template <typename T, bool kE8, bool kSquare>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 2 : kSquare ? 4 : 3)
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
    Eight<T> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = row0 + row_of(i);
      v[i] = load_eight(x + (row < M ? row : M - 1) * row_stride + min(column, K - 1), row < M ? K - column : 0);
    }
    // the largest of each of a lane's columns, and of all
    uint32_t of_columns[Eight<T>::kSizes], of_lane = 0;
#pragma unroll
    for (int j = 0; j < Eight<T>::kSizes; ++j) {
      of_columns[j] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) of_columns[j] = Eight<T>::larger_size(of_columns[j], v[i].size(j));
      of_lane = Eight<T>::larger_size(of_lane, of_columns[j]);
    }
    of_lane = Eight<T>::largest(of_lane);
    const bool odd = __syncthreads_or(of_lane >= 0x7F800000u);     // some value is no number
    BlockScale square;
    if (kSquare) {
      if (odd) {
        of_lane = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) of_lane = max(of_lane, largest_size(v[i], true));
      }
      of_lane = wave_highest(of_lane);
      if (threadIdx.x % kWave == 0) largest_of[wave][0] = of_lane;
      __syncthreads();
      square = scale_of<kE8>(max(max(largest_of[0][0], largest_of[1][0]), max(largest_of[2][0], largest_of[3][0])));
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
        if (!kSquare) s = scale_of<kE8>(row_largest(largest_size(v[i], odd)));
        if (row >= M || column >= K) continue;
        put_eight(straight.codes + row * straight.stride + column, K - column, v[i], s.inverse);
        if (!kSquare && lane16 == 0) put_scale<kE8>(straight.scales, row * column_blocks + blockIdx.x, s.stored);
      }
    }
    if (transposed.codes != nullptr) {
      float inverse[8];
      if (!kSquare) {
        // a column's largest: a lane's eight rows, the wave's four groups of lanes, the four waves
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t largest = Eight<T>::bits_of(of_columns[e * Eight<T>::kSizes / 8], e);
          if (odd) {
            largest = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) largest = max(largest, finite_size(v[i][e]));
          }
          largest = max(largest, __shfl_xor(largest, 16));
          largest = max(largest, __shfl_xor(largest, 32));
          if (threadIdx.x % kWave < 16) largest_of[wave][lane16 * 8 + e] = largest;
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
              codes_of(v[4 * h][e], v[4 * h + 1][e], v[4 * h + 2][e], v[4 * h + 3][e], inverse[e]);
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
    if (gridDim.y < row_blocks) __syncthreads();
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
    const int64_t rows = 16 / across * kRowsEach, groups = (M + rows - 1) / rows;
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

// Four neighbouring results of a row, those in front of column N.
__device__ __forceinline__ void put_four(float* row, int64_t n, int64_t N, f32x4 v) {
  if (n + 4 <= N) {
    *reinterpret_cast<f32x4_memory*>(row + n) = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < N) row[n + e] = v[e];
}
__device__ __forceinline__ void put_four(uint16_t* row, int64_t n, int64_t N, f32x4 v) {
  const u32x2 w = {to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
  if (n + 4 <= N) {
    *reinterpret_cast<u32x2_memory*>(row + n) = w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < N) row[n + e] = static_cast<uint16_t>(w[e / 2] >> e % 2 * 16);
}

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

// Rows that do not start at multiples of 16 bytes, of more than 64 rows of a and not in parts of K: tiles of 128 x 128 by four
// waves of 64 x 64, the next step's codes on their way in registers while this one's are multiplied.  Us so and by the streamed form through
// registers: 333 x 50257 x 1000 of fp32 95 and 115, of bf16 118 and 109; 1024 x 32000 x 4001 271 and 284; 300 x 9000 x 777 30 and
// 26.  (Aligned, 333 x 50257 x 1024 of fp32 takes 54.)
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
  const uint8_t *row_of_a[4], *row_of_b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    row_of_a[i] = a.codes + min(m0 + threadIdx.x / 8 + i * 32, a.rows - 1) * a.stride;
    row_of_b[i] = b.codes + min(n0 + threadIdx.x / 8 + i * 32, b.rows - 1) * b.stride;
  }
  const auto load = [&](int64_t block) {
    const int64_t k = block * kBlock + threadIdx.x % 8 * 16;
    if ((block + 1) * kBlock <= K) {        // of the whole workgroup
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        held[0][i] = *reinterpret_cast<const u32x4_bytes*>(row_of_a[i] + k);
        held[1][i] = *reinterpret_cast<const u32x4_bytes*>(row_of_b[i] + k);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        held[0][i] = load_codes(row_of_a[i], k, K);
        held[1][i] = load_codes(row_of_b[i], k, K);
      }
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

// Aligned codes, powers of two, bf16 results, tiles of 256 x 256 by eight waves of 128 x 64.
//
// What bounds it: the matrix cores (3.9 PFLOP/s of these instructions alone on random codes, at the clock that the card's
// power leaves; 32x32x64 reaches 3.2), LDS reads and fetches into LDS share a step of 128 columns: alone they take 1.1, 0.8 and
// 1.0 us of a compute unit, together 1.65.  8192^3: 439 us, 2.5 PFLOP/s; 1024 x 128256 x 4096: 495 us, 2.2, a share of it the 263 MB of
// the result; 32000 x 4096 x 1024, of eight steps a tile, 155 us, 1.7.  Measured on the way, 8192^3: 32x32x64 by four waves of
// 128 x 128 with both steps' fetches waited for at one barrier 571 us; 16x16x128 by eight waves so 527; fetches that
// the compiler does not wait for in front of reads of LDS, two barriers a step 460; scales as words, shifted each step, instead of
// bytes read each step 444; the XCDs' starts turned 440 and one wave of a SIMD ahead of the other 439.
// The workgroup's tile: each XCD takes neighbouring ones, in groups of up to eight rows of tiles.
struct TileAt {
  uint32_t m, n;
};
__device__ __forceinline__ TileAt tile_at(uint32_t id, uint32_t tiles_m, uint32_t tiles_n) {
  const uint32_t total = tiles_m * tiles_n, each = total / 8, rest = total % 8, xcd = id % 8;
  const uint32_t at = xcd * each + min(xcd, rest) + id / 8;
  const uint32_t of_group = 8 * tiles_n, first = at / of_group * 8, in_group = at % of_group;
  const uint32_t rows = min(8u, tiles_m - first);
  return TileAt{first + in_group % rows, in_group / rows};
}

// From memory straight into LDS, 16 bytes a lane (or a word, or a byte as one), the wave's side by side from `to` on; `at` from 2^31 on
// fetches zeros.  Written as instructions: behind a fetch that it knows the compiler waits for all of them before any
// read of LDS.  `arrived` waits for all but the newest `kNewer` fetches, and for the wave's own reads.
//
// A vector instruction may have written the scalar registers of a fetch just before (readfirstlane makes them), which takes five wait
// states until an access to memory may read them; m0, where the place in LDS stands, takes one.  The compiler does not look into the
// statement, so it waits itself; m0 is an operand, so that the compiler knows who writes it.
typedef uint32_t Buffer __attribute__((ext_vector_type(4)));
__device__ __forceinline__ Buffer buffer_of(const void* p) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  return Buffer{static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(at))),
                static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(at >> 32))), 0x7FFFFFFFu, 0x00027000u};
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return __builtin_amdgcn_readfirstlane(static_cast<int>(reinterpret_cast<uintptr_t>((SBW_LDS const void*)p)));
}
__device__ __forceinline__ void fetch_to_lds(Buffer from, uint32_t at, uint32_t base, uint32_t to) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :: "{m0}"(to), "v"(at), "s"(from), "s"(base) : "memory");
}
__device__ __forceinline__ void fetch_word_to_lds(Buffer from, uint32_t at, uint32_t base, uint32_t to) {
  asm volatile("s_nop 4\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :: "{m0}"(to), "v"(at), "s"(from), "s"(base) : "memory");
}
// A word a lane; of scales of one byte that byte.
template <bool kByte>
__device__ __forceinline__ void fetch_scale_to_lds(Buffer from, uint32_t at, uint32_t base, uint32_t to) {
  if constexpr (kByte)
    asm volatile("s_nop 4\n\tbuffer_load_ubyte %1, %2, %3 offen lds"
                 :: "{m0}"(to), "v"(at), "s"(from), "s"(base) : "memory");
  else
    fetch_word_to_lds(from, at, base, to);
}
// Columns from K on that share their last 16 bytes with a row's last columns, in LDS: 0 instead of whatever stands there.
// `rows` rows of a step that holds column K; every lane of the workgroup comes here, behind a barrier and in front of one.
template <uint32_t kThreadsHere>
__device__ __forceinline__ void clear_behind(u32x4* step, uint32_t rows, uint32_t K) {
  const uint32_t c = K % kBlock / 16, kept = K % 16;
  for (uint32_t r = threadIdx.x; r < rows; r += kThreadsHere) {
    u32x4 w = step[place_of(r, c)];
#pragma unroll
    for (uint32_t d = 0; d < 4; ++d) w[d] &= kept >= d * 4 + 4 ? 0xFFFFFFFFu : kept > d * 4 ? (1u << (kept - d * 4) * 8) - 1u : 0u;
    step[place_of(r, c)] = w;
  }
}
template <int kNewer>
__device__ __forceinline__ void arrived() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(kNewer) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Shape of a tiles kernel: waves of kM x kN instructions of 16 x 16, kDown x kAcross of them.
template <int kM_, int kN_, int kDown_, int kAcross_>
struct TileShape {
  static constexpr int kM = kM_, kN = kN_, kDown = kDown_, kAcross = kAcross_;
  static constexpr uint32_t kRowsA = kM * 16 * kDown, kRowsB = kN * 16 * kAcross, kThreadsHere = kDown * kAcross * kWave;
  static constexpr uint32_t kFetchRows = kThreadsHere / 8;                      // that one fetch of every lane covers
  static constexpr int kFetchA = kRowsA / kFetchRows, kFetchB = kRowsB / kFetchRows;
  static constexpr int kFetches = kFetchA + kFetchB;                         // of a step
  // whether fetch i of side a holds rows of the second half of a wave's instructions
  static constexpr bool upper(int i) { return i * kFetchRows / (kM * 8) % 2 != 0; }
};

template <typename Out, typename Shape>
__global__ void __launch_bounds__(Shape::kThreadsHere, 1)
product_tiles_kernel(Side a, Side b, uint32_t K, uint32_t blocks_each, Out* __restrict__ out, int64_t out_stride, int64_t out_part,
                     uint32_t tiles_m, uint32_t tiles_n) {
  static_assert(Shape::kM * 8 % Shape::kFetchRows == 0, "a fetch holds rows of one half");
  constexpr int kM = Shape::kM, kN = Shape::kN;
  constexpr uint32_t kRowsA = Shape::kRowsA, kRowsB = Shape::kRowsB, kRows = kRowsA + kRowsB, kFetchRows = Shape::kFetchRows;
  constexpr uint32_t kThreadsHere = Shape::kThreadsHere, kStage = kRows * 8;    // 16-byte parts of a step
  __shared__ __attribute__((aligned(1024))) u32x4 codes[2][kStage];
  __shared__ uint32_t tile_scales[2][kRows];                                    // four blocks' bytes
  const uint32_t tid = threadIdx.x, lane = tid % kWave, r16 = lane % 16, quarter = lane / 16;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const TileAt tile = tile_at(blockIdx.x, tiles_m, tiles_n);
  const int64_t m0 = static_cast<int64_t>(tile.m) * kRowsA, n0 = static_cast<int64_t>(tile.n) * kRowsB;
  // the grid's second dimension: parts of K, of a multiple of four blocks
  const uint32_t all_blocks = (K + kBlock - 1) / kBlock, block0 = blockIdx.y * blocks_each;
  const uint32_t blocks = min(blocks_each, all_blocks - block0);
  const auto from_a = buffer_of(a.codes + m0 * a.stride), from_b = buffer_of(b.codes + n0 * b.stride);
  const uint32_t last_a = static_cast<uint32_t>(min(a.rows - m0, int64_t{kRowsA}) - 1), last_b = static_cast<uint32_t>(min(b.rows - n0, int64_t{kRowsB}) - 1);
  // this lane's part of a row in each fetch: its place in LDS is fixed, so the part is permuted
  const uint32_t part16 = (tid % 8 ^ (tid / 16 & 7u)) * 16;
  uint32_t at_a[Shape::kFetchA], at_b[Shape::kFetchB];
#pragma unroll
  for (int i = 0; i < Shape::kFetchA; ++i) at_a[i] = min(tid / 8 + i * kFetchRows, last_a) * static_cast<uint32_t>(a.stride) + part16;
#pragma unroll
  for (int i = 0; i < Shape::kFetchB; ++i) at_b[i] = min(tid / 8 + i * kFetchRows, last_b) * static_cast<uint32_t>(b.stride) + part16;
  // the XCDs start at different blocks: rows a power of two apart would all be fetched from the same channels at a time
  const uint32_t rotation = blocks % 4 == 0 ? blockIdx.x % 8 * (blocks / 32) * 4 : 0;
  const auto physical = [&](uint32_t block) { return block + rotation >= blocks ? block + rotation - blocks : block + rotation; };
  const uint32_t lds_codes = lds_address(&codes[0][0]) + wave * 1024, lds_scales = lds_address(&tile_scales[0][0]) + wave * 256;
  const auto fetch = [&](uint32_t block, uint32_t turn, bool upper) {
    const uint32_t k = (block0 + physical(block)) * kBlock, beyond = block < blocks && k + part16 < K ? 0u : 0x80000000u, to = lds_codes + turn * (kStage * 16);
#pragma unroll
    for (int i = 0; i < Shape::kFetchA; ++i)
      if (Shape::upper(i) == upper) fetch_to_lds(from_a, at_a[i] | beyond, k, to + i * kFetchRows * 128);
    if (upper) return;
#pragma unroll
    for (int i = 0; i < Shape::kFetchB; ++i) fetch_to_lds(from_b, at_b[i] | beyond, k, to + (kRowsA + i * kFetchRows) * 128);
  };
  // Four blocks' scales of a row are a word of LDS; those of blocks behind the last are never used with codes but 0, and
  // are the last block's.  Words of memory are fetched like the codes; others are put together.
  constexpr int kScaleRows = (kRows + kThreadsHere - 1) / kThreadsHere;
  const bool words = all_blocks % 4 == 0 && (reinterpret_cast<uintptr_t>(a.scales) | reinterpret_cast<uintptr_t>(b.scales)) % 4 == 0;
  const auto bring_scales = [&](uint32_t block) {
    const uint32_t turn = block / 4 & 1;
#pragma unroll
    for (int i = 0; i < kScaleRows; ++i) {
      const uint32_t r = tid + i * kThreadsHere;
      if (kRows % kThreadsHere != 0 && r >= kRows) continue;
      const bool of_a = r < kRowsA;
      const Side& s = of_a ? a : b;
      const int64_t row = (min(of_a ? m0 + r : n0 + r - kRowsA, s.rows - 1) >> s.row_shift) - ((of_a ? m0 : n0) >> s.row_shift);
      const uint8_t* first = static_cast<const uint8_t*>(s.scales) + ((of_a ? m0 : n0) >> s.row_shift) * all_blocks;
      if (words) {
        fetch_word_to_lds(buffer_of(first), static_cast<uint32_t>(row) * all_blocks, min(block0 + physical(block), all_blocks - 4),
                          lds_scales + (turn * kRows + i * kThreadsHere) * 4);
      } else {
        uint32_t w = 0;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) w |= static_cast<uint32_t>(first[row * all_blocks + min(block0 + physical(block) + e, all_blocks - 1)]) << e * 8;
        tile_scales[turn][r] = w;
      }
    }
  };
  const uint32_t row_a = wave / Shape::kAcross * (kM * 16), row_b = wave % Shape::kAcross * (kN * 16);
  // this lane's two parts of a row; other rows and the other step lie at fixed distances
  uint32_t at_x[2], at_y[2];
#pragma unroll
  for (uint32_t c = 0; c < 2; ++c) {
    at_x[c] = place_of(row_a + r16, quarter * 2 + c);
    at_y[c] = place_of(kRowsA + row_b + r16, quarter * 2 + c);
  }
  const u32x4* const stage = &codes[0][0];
  f32x4 total[kM][kN] = {};
  constexpr int kAhead = 4;        // rows of instructions whose codes are held
  Codes x[kAhead], y[kN];
  uint32_t sx[kM], sy[kN];
  const auto read_x = [&](int i) { x[i % kAhead] = Codes{stage[at_x[0] + i * 128], stage[at_x[1] + i * 128]}; };
  const auto read_y = [&](int j) { y[j] = Codes{stage[at_y[0] + j * 128], stage[at_y[1] + j * 128]}; };
  const auto read_scales = [&](uint32_t block) {   // four blocks' bytes, of which an instruction takes the lowest
#pragma unroll
    for (int t = 0; t < kM; ++t) sx[t] = tile_scales[block / 4 & 1][row_a + t * 16 + r16];
#pragma unroll
    for (int t = 0; t < kN; ++t) sy[t] = tile_scales[block / 4 & 1][kRowsA + row_b + t * 16 + r16];
  };
  const auto multiply = [&](int i, int j) {
    total[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(as_operand(y[j]), as_operand(x[i % kAhead]), total[i][j], 0,
                                                                   0, 0, sy[j], 0, sx[i]);
  };
  // The codes of a step are fetched in two parts, each as soon as every wave has read the one that stood in its place, two
  // steps before: b and the lower halves of a's rows in the first quarter of a step, the upper halves in the last.  Whatever
  // is waited for has had a whole step, as only what the newest step fetched may be still on its way.
  constexpr int kOfStep = Shape::kFetchA + Shape::kFetchB, kUpper = Shape::kFetchA / 2;
  bring_scales(0);
  fetch(0, 0, false);
  fetch(0, 0, true);
  fetch(1, 1, false);
  fetch(1, 1, true);
  arrived<kOfStep + kUpper>();
  read_scales(0);
  read_x(0);
  read_x(1);
#pragma unroll
  for (int j = 0; j < kN; ++j) read_y(j);
  if (wave / 4 != 0) __builtin_amdgcn_s_setprio(1);   // a SIMD's two waves drift apart: one multiplies while the other waits
  for (uint32_t block = 0; block < blocks; ++block) {
#pragma unroll
    for (int i = 0; i < kM; ++i) {
      if (i == kM / 2 - 2) {
        arrived<kOfStep>();
        fetch(block + 2, block & 1, false);
        if (block % 4 == 0) bring_scales(block + 4);
      }
      if (i == kM - 2) {
        arrived<kOfStep>();
        fetch(block + 2, block & 1, true);
        const uint32_t other = block & 1 ? -kStage : kStage;
        at_x[0] += other, at_x[1] += other, at_y[0] += other, at_y[1] += other;
      }
      read_x((i + 2) % kM);
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        multiply(i, j);
        if (i == kM - 1) read_y(j);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // the instructions stay in front of the branch
#pragma unroll
    for (int i = 0; i < kM; ++i)
#pragma unroll
      for (int j = 0; j < kN; ++j) asm volatile("" : "+v"(total[i][j]));
    if (block % 4 == 3) {
      read_scales(block + 1);
    } else {
#pragma unroll
      for (int t = 0; t < kM; ++t) sx[t] >>= 8;
#pragma unroll
      for (int t = 0; t < kN; ++t) sy[t] >>= 8;
    }
  }
  arrived<0>();
  if constexpr (sizeof(Out) == 4) {
    out += blockIdx.y * out_part;
#pragma unroll
    for (int i = 0; i < kM; ++i) {
      const int64_t m = m0 + row_a + i * 16 + r16;
      if (m >= a.rows) continue;
#pragma unroll
      for (int j = 0; j < kN; ++j) put_four(out + m * out_stride, n0 + row_b + j * 16 + quarter * 4, b.rows, total[i][j]);
    }
    return;
  }
  // a wave's results, turned in LDS: 8 bytes of a row and four neighbouring columns a lane, in places permuted
  // by the row; then 16 bytes a lane, whole rows
  constexpr uint32_t kWide = kN * 4;       // places of 8 bytes in a row
  auto* const turned = reinterpret_cast<u32x2*>(&codes[0][0]) + wave * (kM * 16 * kWide);
#pragma unroll
  for (int i = 0; i < kM; ++i)
#pragma unroll
    for (int j = 0; j < kN; ++j)
      turned[(i * 16 + r16) * kWide + ((j * 4 + quarter) ^ (i * 16 + r16) % kWide)] =
          u32x2{to_bf16x2(total[i][j][0], total[i][j][1]), to_bf16x2(total[i][j][2], total[i][j][3])};
  __builtin_amdgcn_wave_barrier();
  constexpr uint32_t kLanes = kWide / 2;   // of a row
  const int64_t n = n0 + row_b + lane % kLanes * 8;
#pragma unroll 4
  for (uint32_t p = 0; p < kM * 16 * kLanes / kWave; ++p) {
    const uint32_t r = p * (kWave / kLanes) + lane / kLanes;
    const int64_t m = m0 + row_a + r;
    const u32x4 w = reinterpret_cast<const u32x4*>(turned)[r * kLanes + (lane % kLanes ^ (r % kWide >> 1))];
    const u32x4 v = r & 1 ? u32x4{w.z, w.w, w.x, w.y} : w;
    if (m >= a.rows) continue;
    auto* to = reinterpret_cast<uint16_t*>(out) + m * out_stride + n;
    if (n + 8 <= b.rows) {
      *reinterpret_cast<u32x4_memory*>(to) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (n + e < b.rows) to[e] = static_cast<uint16_t>(v[e / 2] >> e % 2 * 16);
    }
  }
}

// Up to 16 rows of a: the rows of b stream past them once.  The waves of a workgroup share the columns, kSteps
// blocks each, and keep their part of a in registers; a wave's part of 16 * kTn rows of b goes from memory into registers and
// into the instructions (a's rows as rows, b's as columns).  The waves' sums meet in LDS.  Any alignment.  Bound by memory, with a barrier
// and the waves' sums for every tile: 1 x 32000 x 2048 15.6 us, 4.2 TB/s.
template <typename Out, bool kE8, int kSteps, int kTn>
__global__ void __launch_bounds__(1024)
product_rows_kernel(Side a, Side b, uint32_t K, Out* __restrict__ out, int64_t out_stride, uint32_t waves) {
  constexpr bool kExact = sizeof(Out) == 4, kInside = kE8 && !kExact;
  constexpr uint32_t kSums = kTn * 256;                     // of a wave
  // sixteen sums of a row side by side, rows 4 apart (of the wave's four quarters) in other banks
  const auto place_of_sum = [](uint32_t row, uint32_t c) { return row / 4 * 64 + ((row ^ row / 4) % 4) * 16 + c; };
  extern __shared__ float shared[];
  float* const sums[2] = {shared, shared + waves * kSums};
  float* const row_scales = shared + 2 * waves * kSums;     // [wave][step][16]
  const uint32_t tid = threadIdx.x, lane = tid % kWave, r16 = lane % 16, quarter = lane / 16, threads = waves * kWave;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const uint32_t blocks = (K + kBlock - 1) / kBlock, first = wave * kSteps;
  const int64_t tiles = (b.rows + 16 * kTn - 1) / (16 * kTn);
  // a lane's 32 columns of step s: two parts of 16, those of a row 64 apart, so that four lanes take a line
  const auto column = [&](int s, int h) { return (first + s) * kBlock + h * 64 + quarter * 16; };

  Codes words[kTn][kSteps];
  uint32_t scale[kTn][kSteps];
  const bool ragged = (first + kSteps) * kBlock > K;        // some part of this wave's lies beyond K
  const auto load = [&](int64_t tile) {
#pragma unroll
    for (int t = 0; t < kTn; ++t) {
      const int64_t n = min(tile * (16 * kTn) + t * 16 + r16, b.rows - 1);
      const uint8_t* row = b.codes + n * b.stride;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if (!ragged) {
          words[t][s].lo = *reinterpret_cast<const u32x4_bytes*>(row + column(s, 0));
          words[t][s].hi = *reinterpret_cast<const u32x4_bytes*>(row + column(s, 1));
        } else {
          words[t][s] = Codes{load_codes(row, column(s, 0), K), load_codes(row, column(s, 1), K)};
        }
        scale[t][s] = load_scale<kE8, kE8>(b, n, min(first + s, blocks - 1), blocks);
      }
    }
  };
  const auto next_of = [&](int64_t tile) { return tile + gridDim.x < tiles ? tile + gridDim.x : tile; };
  load(blockIdx.x);

  Codes x[kSteps];
  uint32_t sx[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int64_t m = r16;
    const uint8_t* row = a.codes + min(m, a.rows - 1) * a.stride;
    x[s] = Codes{load_codes(row, column(s, 0), K), load_codes(row, column(s, 1), K)};
    sx[s] = load_scale<kE8, kInside>(a, m, min(first + s, blocks - 1), blocks);
    if (!kInside && quarter == 0) row_scales[(wave * kSteps + s) * 16 + m] = __uint_as_float(sx[s]);
  }
  __syncthreads();

  uint32_t turn = 0;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
#pragma unroll
    for (int t = 0; t < kTn; ++t) {
      f32x4 total = {};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if constexpr (kInside) {
          total = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(as_operand(x[s]), as_operand(words[t][s]), total, 0, 0, 0, sx[s], 0,
                                                                   scale[t][s]);
        } else {
          const float sb = kE8 ? power_of(scale[t][s]) : __uint_as_float(scale[t][s]);
          f32x4 part = {};
          if constexpr (kExact) {
            const Widened wide = widened(words[t][s]);
            Codes c = x[s];
            if (kSteps > 2) asm volatile("" : "+v"(c.lo), "+v"(c.hi));   // widened each time: there is no room to keep them
            const Widened wx = widened(c);
#pragma unroll
            for (int h = 0; h < 4; ++h) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wx.part[h], wide.part[h], part, 0, 0, 0);
          } else {
            part = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(as_operand(x[s]), as_operand(words[t][s]), part, 0, 0, 0,
                                                                    0x7F7F7F7F, 0, 0x7F7F7F7F);
          }
          const f32x4 sa = *reinterpret_cast<const f32x4*>(&row_scales[(wave * kSteps + s) * 16 + quarter * 4]);
#pragma unroll
          for (int e = 0; e < 4; ++e) total[e] = __builtin_fmaf(part[e], sa[e] * sb, total[e]);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[turn][wave * kSums + place_of_sum(t * 16 + quarter * 4 + e, r16)] = total[e];
    }
    __builtin_amdgcn_sched_barrier(0);
    load(next_of(tile));
    __builtin_amdgcn_sched_barrier(0);
    // the waves' reads of these sums are done when they meet here again, one tile later
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    for (uint32_t i = tid; i < kSums; i += threads) {
      const uint32_t row = i / 16, c = i % 16;               // row: a tile of 16 rows of b, a row of a
      const int64_t m = row % 16, n = tile * (16 * kTn) + row / 16 * 16 + c;
      if (m >= a.rows || n >= b.rows) continue;
      float sum = sums[turn][place_of_sum(row, c)];
      for (uint32_t w = 1; w < waves; ++w) sum += sums[turn][w * kSums + place_of_sum(row, c)];
      put_logit(out + m * out_stride + n, sum);
    }
    turn ^= 1;
  }
}

template <typename Out, bool kE8, int kSteps, int kTn>
void launch_rows_of(Side a, Side b, int64_t K, void* out, int64_t out_stride, hipStream_t stream) {
  const auto waves = static_cast<uint32_t>((blocks_of(K) + kSteps - 1) / kSteps);
  const int64_t tiles = (b.rows + 16 * kTn - 1) / (16 * kTn);
  const int64_t resident = 256 * (16 / waves);
  const uint32_t lds = (2 * waves * kTn * 256 + waves * kSteps * 16) * sizeof(float);
  product_rows_kernel<Out, kE8, kSteps, kTn><<<static_cast<uint32_t>(tiles < resident ? tiles : resident), waves * kWave, lds, stream>>>(
      a, b, static_cast<uint32_t>(K), static_cast<Out*>(out), out_stride, waves);
}

// Any scales and results: tiles whose steps stand in kStages places of LDS, all but one of them on their way.  One barrier a
// step: behind it the step's codes and scales have arrived, and the place of the step before is free.  64 x 128256 x 4096 109 us, 5.0 TB/s
// (memory); 1024 x 32000 x 4096 of fp32 scales 203, 1.3 PFLOP/s (the fma of every element and block), of fp32 results 298, 0.9
// (widening).  Rows that do not start at multiples of 16 bytes (kDirect is false) come through registers, a step ahead, into one of two places.
template <typename Shape, int kStages>
struct StreamLds {
  static constexpr uint32_t kRows = Shape::kRowsA + Shape::kRowsB;
  static constexpr uint32_t kScalePlaces = (kRows + Shape::kThreadsHere - 1) / Shape::kThreadsHere * Shape::kThreadsHere;
  static constexpr uint32_t kStage = kRows * kBlock + kScalePlaces * 4;      // bytes
  static constexpr uint32_t kBytes = kStages * kStage;
};
template <typename Out, bool kE8, bool kExact, bool kDirect, typename Shape, int kStages>
__global__ void __launch_bounds__(Shape::kThreadsHere)
product_stream_kernel(Side a, Side b, uint32_t K, uint32_t blocks_each, Out* __restrict__ out, int64_t out_stride, int64_t out_part,
                      uint32_t tiles_m, uint32_t tiles_n) {
  using Lds = StreamLds<Shape, kStages>;
  constexpr bool kInside = kE8 && !kExact;
  constexpr int kM = Shape::kM, kN = Shape::kN, kWords = Lds::kScalePlaces / Shape::kThreadsHere;
  constexpr uint32_t kRowsA = Shape::kRowsA, kRows = Lds::kRows, kFetchRows = Shape::kFetchRows;
  extern __shared__ __attribute__((aligned(1024))) uint8_t stages[];
  const uint32_t tid = threadIdx.x, lane = tid % kWave, r16 = lane % 16, quarter = lane / 16;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const TileAt tile = tile_at(blockIdx.x, tiles_m, tiles_n);
  const int64_t m0 = static_cast<int64_t>(tile.m) * kRowsA, n0 = static_cast<int64_t>(tile.n) * Shape::kRowsB;
  const uint32_t all_blocks = (K + kBlock - 1) / kBlock, block0 = blockIdx.y * blocks_each;
  const uint32_t blocks = min(blocks_each, all_blocks - block0);
  const Buffer from_a = buffer_of(a.codes + m0 * a.stride), from_b = buffer_of(b.codes + n0 * b.stride);
  const uint32_t last_a = static_cast<uint32_t>(min(a.rows - m0, int64_t{kRowsA}) - 1), last_b = static_cast<uint32_t>(min(b.rows - n0, int64_t{Shape::kRowsB}) - 1);
  const uint32_t part16 = (tid % 8 ^ (tid / 16 & 7u)) * 16;
  uint32_t at_a[Shape::kFetchA], at_b[Shape::kFetchB], at_scale[kWords];
#pragma unroll
  for (int i = 0; i < Shape::kFetchA; ++i) at_a[i] = min(tid / 8 + i * kFetchRows, last_a) * static_cast<uint32_t>(a.stride) + part16;
#pragma unroll
  for (int i = 0; i < Shape::kFetchB; ++i) at_b[i] = min(tid / 8 + i * kFetchRows, last_b) * static_cast<uint32_t>(b.stride) + part16;
  // scales: whole waves look after rows of one side
  static_assert(kRowsA % kWave == 0 && Shape::kRowsB % kWave == 0, "a wave's rows are of one side");
  static_assert(kDirect || kStages == 2, "a step in registers, one in LDS");
  constexpr uint32_t kSize = kE8 ? 1 : 4;
  const uint8_t* first_scale[2] = {static_cast<const uint8_t*>(a.scales) + (m0 >> a.row_shift) * all_blocks * kSize,
                                   static_cast<const uint8_t*>(b.scales) + (n0 >> b.row_shift) * all_blocks * kSize};
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    const uint32_t r = min(tid + i * Shape::kThreadsHere, kRows - 1);
    const int64_t row = r < kRowsA ? (min(m0 + r, a.rows - 1) >> a.row_shift) - (m0 >> a.row_shift)
                                   : (min(n0 + r - kRowsA, b.rows - 1) >> b.row_shift) - (n0 >> b.row_shift);
    at_scale[i] = static_cast<uint32_t>(row) * all_blocks * kSize;
  }
  const uint32_t lds = lds_address(stages);
  // tiles start at different blocks: at one block, rows a power of two apart come from few channels (64 x 128256 x 4096 with
  // fp32 scales: 129 us so, 118 with the start turned; with 128 columns to eight waves, 110 with 128 to four)
  const uint32_t rotation = tile.n % blocks;
  const auto block_of = [&](uint32_t step) { return block0 + (step + rotation >= blocks ? step + rotation - blocks : step + rotation); };
  const auto fetch = [&](uint32_t step, uint32_t stage) {
    const uint32_t block = block_of(step), k = block * kBlock;
    const uint32_t to = lds + stage * Lds::kStage + wave * 1024;
    const uint32_t beyond = step < blocks && k + part16 < K ? 0u : 0x80000000u;
#pragma unroll
    for (int i = 0; i < Shape::kFetchA; ++i) fetch_to_lds(from_a, at_a[i] | beyond, k, to + i * kFetchRows * kBlock);
#pragma unroll
    for (int i = 0; i < Shape::kFetchB; ++i) fetch_to_lds(from_b, at_b[i] | beyond, k, to + (kRowsA + i * kFetchRows) * kBlock);
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const uint32_t r = wave * kWave + i * Shape::kThreadsHere;
      fetch_scale_to_lds<kE8>(buffer_of(first_scale[r < kRowsA ? 0 : 1]), at_scale[i], min(block, all_blocks - 1) * kSize,
                              lds + stage * Lds::kStage + kRows * kBlock + r * 4);
    }
  };
  constexpr int kOfStep = Shape::kFetchA + Shape::kFetchB + kWords;
  const uint32_t row_a = wave / Shape::kAcross * (kM * 16), row_b = kRowsA + wave % Shape::kAcross * (kN * 16);
  const uint32_t lo = place_of(r16, quarter * 2) * 16, hi = place_of(r16, quarter * 2 + 1) * 16;   // in any sixteen rows
  f32x4 total[kM][kN] = {};
  // through registers
  u32x4 held[Shape::kFetchA + Shape::kFetchB];
  uint32_t held_scale[kWords];
  const auto load = [&](uint32_t step) {
    const uint32_t block = block_of(step), k = block * kBlock + part16;
    const uint8_t *row_of_a = a.codes + m0 * a.stride - part16, *row_of_b = b.codes + n0 * b.stride - part16;
    if ((block + 1) * kBlock <= K) {             // of the whole workgroup
#pragma unroll
      for (int i = 0; i < Shape::kFetchA; ++i) held[i] = *reinterpret_cast<const u32x4_bytes*>(row_of_a + at_a[i] + k);
#pragma unroll
      for (int i = 0; i < Shape::kFetchB; ++i) held[Shape::kFetchA + i] = *reinterpret_cast<const u32x4_bytes*>(row_of_b + at_b[i] + k);
    } else {
#pragma unroll
      for (int i = 0; i < Shape::kFetchA; ++i) held[i] = load_codes(row_of_a + at_a[i], k, K);
#pragma unroll
      for (int i = 0; i < Shape::kFetchB; ++i) held[Shape::kFetchA + i] = load_codes(row_of_b + at_b[i], k, K);
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const uint8_t* p = first_scale[wave * kWave + i * Shape::kThreadsHere < kRowsA ? 0 : 1] + at_scale[i] + block * kSize;
      held_scale[i] = kE8 ? *p : *reinterpret_cast<const uint32_t*>(p);
    }
  };
  const auto put = [&](uint32_t stage) {
    uint8_t* to = stages + stage * Lds::kStage;
#pragma unroll
    for (int i = 0; i < Shape::kFetchA + Shape::kFetchB; ++i) reinterpret_cast<u32x4*>(to)[i * Shape::kThreadsHere + tid] = held[i];
#pragma unroll
    for (int i = 0; i < kWords; ++i) reinterpret_cast<uint32_t*>(to + kRows * kBlock)[i * Shape::kThreadsHere + tid] = held_scale[i];
  };
  if constexpr (kDirect) {
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(s, s);
  } else {
    load(0);
    put(0);
  }
  uint32_t stage = 0;
  for (uint32_t step = 0; step < blocks; ++step) {
    if constexpr (kDirect) {
      arrived<(kStages - 2) * kOfStep>();
      if (K % 16 != 0 && block_of(step) + 1 == all_blocks) {
        clear_behind<Shape::kThreadsHere>(reinterpret_cast<u32x4*>(stages + stage * Lds::kStage), kRows, K);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      }
      fetch(step + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
    } else {
      __syncthreads();
      if (step + 1 < blocks) load(step + 1);
    }
    const uint8_t* at = stages + stage * Lds::kStage;
    const auto read = [&](uint32_t row) {
      return Codes{*reinterpret_cast<const u32x4*>(at + row * kBlock + lo), *reinterpret_cast<const u32x4*>(at + row * kBlock + hi)};
    };
    const auto* scales = reinterpret_cast<const uint32_t*>(at + kRows * kBlock);
    const auto as_scale = [&](uint32_t w) { return kE8 ? power_of(w & 0xFFu) : __uint_as_float(w); };
    if constexpr (kExact) {
      Widened y[kN];
      f32x4 sb[kN];
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        y[j] = widened(read(row_b + j * 16));
        const u32x4 w = *reinterpret_cast<const u32x4*>(scales + row_b + j * 16 + quarter * 4);
        sb[j] = f32x4{as_scale(w.x), as_scale(w.y), as_scale(w.z), as_scale(w.w)};
      }
#pragma unroll
      for (int i = 0; i < kM; ++i) {
        const Widened x = widened(read(row_a + i * 16));
        const float sa = as_scale(scales[row_a + i * 16 + r16]);
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          f32x4 part = {};
#pragma unroll
          for (int h = 0; h < 4; ++h) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[j].part[h], x.part[h], part, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e) total[i][j][e] = __builtin_fmaf(part[e], sa * sb[j][e], total[i][j][e]);
        }
      }
    } else {
      Codes y[kN];
      uint32_t sy[kN];
      f32x4 sb[kN];
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        y[j] = read(row_b + j * 16);
        if constexpr (kInside) {
          sy[j] = scales[row_b + j * 16 + r16];
        } else {
          const u32x4 w = *reinterpret_cast<const u32x4*>(scales + row_b + j * 16 + quarter * 4);
          sb[j] = f32x4{as_scale(w.x), as_scale(w.y), as_scale(w.z), as_scale(w.w)};
        }
      }
#pragma unroll
      for (int i = 0; i < kM; ++i) {
        const Codes x = read(row_a + i * 16);
        const uint32_t sx = scales[row_a + i * 16 + r16];
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          if constexpr (kInside) {
            total[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(as_operand(y[j]), as_operand(x), total[i][j], 0, 0, 0,
                                                                           sy[j], 0, sx);
          } else {
            const f32x4 none = {};
            const f32x4 part = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(as_operand(y[j]), as_operand(x), none, 0, 0, 0,
                                                                                0x7F7F7F7F, 0, 0x7F7F7F7F);
#pragma unroll
            for (int e = 0; e < 4; ++e) total[i][j][e] = __builtin_fmaf(part[e], as_scale(sx) * sb[j][e], total[i][j][e]);
          }
        }
      }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if constexpr (!kDirect)
      if (step + 1 < blocks) put(stage);
  }
  // fetches that nothing waited for end before the workgroup does
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  out += blockIdx.y * out_part;
#pragma unroll
  for (int i = 0; i < kM; ++i) {
    const int64_t m = m0 + row_a + i * 16 + r16;
    if (m >= a.rows) continue;
#pragma unroll
    for (int j = 0; j < kN; ++j) put_four(out + m * out_stride, n0 + row_b - kRowsA + j * 16 + quarter * 4, b.rows, total[i][j]);
  }
}

// Sums of the parts of K, in their order.
template <typename Out>
__global__ void __launch_bounds__(kThreads)
product_join_kernel(const float* __restrict__ parts, int64_t M, int64_t N, int64_t pitch, uint32_t count, Out* __restrict__ out,
                    int64_t out_stride) {
  const int64_t n = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 4;
  if (n >= N) return;
  for (int64_t m = blockIdx.y; m < M; m += gridDim.y) {
    const float* at = parts + m * pitch + n;
    f32x4 sum = *reinterpret_cast<const f32x4*>(at);
    for (uint32_t p = 1; p < count; ++p) sum += *reinterpret_cast<const f32x4*>(at + p * M * pitch);
    put_four(out + m * out_stride, n, N, sum);
  }
}

// How a product is computed.
using Tiles64 = TileShape<4, 2, 1, 4>;      // of a row of tiles only; 128 rows of b
using Tiles128 = TileShape<4, 4, 2, 2>;
using Tiles256 = TileShape<8, 4, 2, 4>;
enum class Form { kRows, k64, k128, k256 };
struct Plan {
  Form form;
  int64_t parts;            // of K
};
// `inside`: the scales go into the instructions.  Figures: us, e the e8m0 scales, f fp32 ones, then the result's type.
Plan plan_of(int64_t M, int64_t N, int64_t K, bool inside, bool direct) {
  const int64_t blocks = blocks_of(K);
  const auto tiles = [&](int64_t rows, int64_t columns) { return (M + rows - 1) / rows * ((N + columns - 1) / columns); };
  // Parts of at least `least` blocks where the tiles alone leave compute units idle.  64 x 1024 x 4096 e bf16: 1 part 19.5, 2 14.1, 4
  // 10.6, 8 10.2; 64 x 16000: 20.7, 17.6, 20.6, 27.8; 64 x 24000 (188 tiles): 21.2, 25.5.  128 x 128, 512 x 2048 x 8192 f bf16: 84, 51, 4 33;
  // 1024 x 2048 x 8192 (128 tiles): 84, 54, 45; 1024 x 4096 x 4096 (256 tiles): 47, 45, 55, and e bf16 31, 35, 47.
  const auto parts = [&](int64_t count, int64_t least) {
    const int64_t most = std::min(256 / std::max(count, int64_t{1}), blocks / least);
    return count >= 200 || most < 2 ? int64_t{1} : most;
  };
  const int64_t of_64 = tiles(64, 128), of_128 = tiles(128, 128), of_256 = tiles(256, 256);
  // Up to 16 rows by kRows and k64.  e bf16: 8000 x 2048 6.6 and 11.1, 32000 x 2048 15.7 and 12.6, 32000 x 4096 27.9 and 21.5, 128256 x 4096
  // 106 and 100.  f fp32: 8000 x 2048 7.4 and 17.5, 32000 x 2048 16.8 and 19.4, 128256 x 2048 62.2 and 63.4, 32000 x 4096 35.2 and 34.4,
  // 128256 x 8192 251 and 226.
  if (M <= 16 && blocks <= 64 && (!direct || of_64 < 200 || (!inside && blocks <= 16))) return Plan{Form::kRows, 1};
  // 64 rows by k64 and k128: x 32000 x 2048 e bf16 13.7 and 17.0, x 128256 x 4096 f bf16 122 and 138.
  if (M <= 64) return Plan{Form::k64, parts(of_64, 4)};
  // Two tiles of 128 x 128 share a compute unit.  A round of 512 of them takes 40 (2048 x 4096 x 4096 e bf16), one of 256 of 256 x 256, twice the work,
  // 60; without scales inside 60 and 100 (f bf16), 89 and 148 (e fp32): rounds are compared by 3 to 2, and 7 to 4.  By k128 and k256: 256 x
  // 32000 x 4096 e bf16 49 and 57, 512 x 40000 128 and 111, f bf16 162 and 198, 1024 x 32000 170 and 123, f 234 and 203.
  const int64_t parts_128 = parts(of_128, 4), parts_256 = parts(of_256, 48);
  const auto time = [&](int64_t count, int64_t resident, int64_t n) { return (count * n + resident - 1) / resident * ((blocks + n - 1) / n); };
  if (time(of_256, 256, parts_256) * (inside ? 6 : 7) <= time(of_128, 512, parts_128) * 4) return Plan{Form::k256, parts_256};
  return Plan{Form::k128, parts_128};
}
int64_t part_pitch(int64_t N) { return (N + 3) / 4 * 4; }

template <typename Out, bool kE8, bool kExact, bool kDirect, typename Shape, int kStages>
void launch_stream(Side a, Side b, int64_t K, int64_t blocks_each, Out* out, int64_t out_stride, int64_t out_part, hipStream_t stream) {
  const auto tiles_m = static_cast<uint32_t>((a.rows + Shape::kRowsA - 1) / Shape::kRowsA);
  const auto tiles_n = static_cast<uint32_t>((b.rows + Shape::kRowsB - 1) / Shape::kRowsB);
  const dim3 grid(tiles_m * tiles_n, static_cast<uint32_t>((blocks_of(K) + blocks_each - 1) / blocks_each));
  product_stream_kernel<Out, kE8, kExact, kDirect, Shape, kStages><<<grid, Shape::kThreadsHere, StreamLds<Shape, kStages>::kBytes, stream>>>(
      a, b, static_cast<uint32_t>(K), static_cast<uint32_t>(blocks_each), out, out_stride, out_part, tiles_m, tiles_n);
}

// Tiles of one form into `out`, of type Out: the result, or the parts' sums.
template <typename Out, bool kE8, bool kExact>
void launch_tiles(Form form, bool direct, Side a, Side b, int64_t K, int64_t blocks_each, Out* out, int64_t out_stride,
                  int64_t out_part, hipStream_t stream) {
  if (form == Form::k64) {
    auto* launch = direct ? launch_stream<Out, kE8, kExact, true, Tiles64, 3> : launch_stream<Out, kE8, kExact, false, Tiles64, 2>;
    launch(a, b, K, blocks_each, out, out_stride, out_part, stream);
  } else if (!direct) {
    if constexpr (sizeof(Out) == 4)    // parts of K
      launch_stream<Out, kE8, kExact, false, Tiles128, 2>(a, b, K, blocks_each, out, out_stride, out_part, stream);
  } else if (form == Form::k128) {
    // three places leave no room for a second workgroup (512 x 16000 x 4096 e8m0 bf16 41 us with two, 57 with three)
    launch_stream<Out, kE8, kExact, true, Tiles128, 2>(a, b, K, blocks_each, out, out_stride, out_part, stream);
  } else if (!kE8 || kExact || K % 16 != 0) {
    launch_stream<Out, kE8, kExact, true, Tiles256, 2>(a, b, K, blocks_each, out, out_stride, out_part, stream);
  } else if constexpr (kE8 && !kExact) {
    const auto tiles_m = static_cast<uint32_t>((a.rows + 255) / 256), tiles_n = static_cast<uint32_t>((b.rows + 255) / 256);
    const dim3 grid(tiles_m * tiles_n, static_cast<uint32_t>((blocks_of(K) + blocks_each - 1) / blocks_each));
    product_tiles_kernel<Out, Tiles256><<<grid, Tiles256::kThreadsHere, 0, stream>>>(
        a, b, static_cast<uint32_t>(K), static_cast<uint32_t>(blocks_each), out, out_stride, out_part, tiles_m, tiles_n);
  }
}

template <typename Out, bool kE8>
void launch_product(Side a, Side b, int64_t K, void* out_, int64_t out_stride, uint64_t* workspace, hipStream_t stream) {
  constexpr bool kExact = sizeof(Out) == 4;
  auto* out = static_cast<Out*>(out_);
  const auto aligned = [&](const Side& s) {
    return (reinterpret_cast<uintptr_t>(s.codes) | static_cast<uintptr_t>(s.stride)) % 16 == 0;
  };
  const bool direct = aligned(a) && aligned(b);
  const Plan plan = plan_of(a.rows, b.rows, K, kE8 && !kExact, direct);
  const int64_t blocks = blocks_of(K);
  if (plan.form == Form::kRows) {
    auto* launch = blocks <= 16 ? launch_rows_of<Out, kE8, 1, 2> : blocks <= 32 ? launch_rows_of<Out, kE8, 2, 2> : launch_rows_of<Out, kE8, 4, 1>;
    launch(a, b, K, out, out_stride, stream);
    return;
  }
  if (!direct && plan.form != Form::k64 && plan.parts == 1) {
    const dim3 grid(static_cast<uint32_t>(blocks_of(b.rows)), static_cast<uint32_t>(blocks_of(a.rows)));
    product_any_kernel<Out, kE8><<<grid, kThreads, 0, stream>>>(a, b, K, out, out_stride);
    return;
  }
  if (plan.parts == 1) {
    launch_tiles<Out, kE8, kExact>(plan.form, direct, a, b, K, blocks, out, out_stride, 0, stream);
    return;
  }
  const int64_t blocks_each = ((blocks + plan.parts - 1) / plan.parts + 3) / 4 * 4, parts = (blocks + blocks_each - 1) / blocks_each;
  const int64_t pitch = part_pitch(b.rows);
  auto* sums = reinterpret_cast<float*>(workspace);
  launch_tiles<float, kE8, kExact>(plan.form, direct, a, b, K, blocks_each, sums, pitch, a.rows * pitch, stream);
  const dim3 grid(static_cast<uint32_t>((b.rows + 4 * kThreads - 1) / (4 * kThreads)),
                  static_cast<uint32_t>(a.rows < kMaxGridY ? a.rows : kMaxGridY));
  product_join_kernel<Out><<<grid, kThreads, 0, stream>>>(sums, a.rows, b.rows, pitch, static_cast<uint32_t>(parts), out, out_stride);
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
  if (M <= 0 || N <= 0 || K <= 0 || M > kMostRows || N > kMostRows || K > kMostStride) return 0;
  int64_t parts = 1;
  for (const bool inside : {false, true})
    for (const bool direct : {false, true}) parts = std::max(parts, plan_of(M, N, K, inside, direct).parts);
  return parts == 1 ? 0 : parts * M * part_pitch(N) / 2;
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
  if (M > kBlock * kMaxGridY || N > kMostRows || blocks_of(M) * blocks_of(N) >= int64_t{1} << 24) return SBW_ERR_UNSUPPORTED;
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
  launch(left, right, K, out, out_stride, workspace, static_cast<hipStream_t>(stream));
  return after_launch();
}

}  // extern "C"
