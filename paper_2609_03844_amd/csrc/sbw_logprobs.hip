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

constexpr int kMostTokens = SBW_STEP_MAX_TOKENS;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.693147180559945309417f;
// A score's floor inside the weighted sums: its exponential is 0, and 0 times it is 0 where 0 times -inf
// would be NaN.  No lower than it has to be, as the gradient multiplies it by an upstream one.
constexpr float kScoreFloor = -1000.0f;
// c; finite for every inv_t, as the largest logit's score is 0 times it.
__host__ __device__ inline float score_factor(float inv_t) { return fminf(inv_t * kLog2e, 3.402823466e38f); }

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
constexpr uint32_t kLowestKey = 0x007FFFFFu;   // of -inf

// (x - m) * inv_t - ln_s; halved on the way, so that only a result beyond fp32 is infinite.
__device__ __forceinline__ float logprob_of(float x, float m, float inv_t, float ln_s) {
  return __builtin_fmaf((0.5f * x - 0.5f * m) * inv_t, 2.0f, -ln_s);
}

// Wave reductions by DPP moves: within rows of 16 lanes, then row broadcasts that carry the
// result to lane 63, from where every lane gets it.  Lanes a move does not reach see the identity.
template <int kCtrl, int kRowMask>
__device__ __forceinline__ float dpp_moved(float v, float identity) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(identity), __float_as_int(v), kCtrl, kRowMask,
                                                    0xF, false));
}
template <typename F>
__device__ __forceinline__ float wave_reduce(float v, float identity, F f) {
  v = f(v, dpp_moved<0xB1, 0xF>(v, identity));    // quad_perm [1,0,3,2]
  v = f(v, dpp_moved<0x4E, 0xF>(v, identity));    // quad_perm [2,3,0,1]
  v = f(v, dpp_moved<0x141, 0xF>(v, identity));   // row_half_mirror
  v = f(v, dpp_moved<0x140, 0xF>(v, identity));   // row_mirror
  v = f(v, dpp_moved<0x142, 0xA>(v, identity));   // row_bcast:15 into rows 1 and 3
  v = f(v, dpp_moved<0x143, 0xC>(v, identity));   // row_bcast:31 into rows 2 and 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
// The larger of two, NaN if either is.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_largest(float v) {
  return wave_reduce(v, -INFINITY, [](float a, float b) { return larger(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_reduce(v, 0.0f, [](float a, float b) { return a + b; });
}

// ---------------------------------------------------------------------------
// Vectors of a row.  Vector j holds columns j * kPer .. j * kPer + kPer - 1; the row's last
// one may be partial (its other places read as -inf and are not written).
// ---------------------------------------------------------------------------
template <typename T>
constexpr uint32_t kPerOf = 16 / sizeof(T);

__device__ __forceinline__ void set_elem(f32x4& v, int e, float x) { v[e] = x; }
__device__ __forceinline__ void set_elem(u32x4& v, int e, uint16_t x) {
  const uint32_t shift = (e & 1) * 16;
  v[e >> 1] = (v[e >> 1] & ~(0xFFFFu << shift)) | static_cast<uint32_t>(x) << shift;
}


template <typename T>
__device__ __forceinline__ typename VecOf<T>::Value load_whole(const T* row, uint32_t j) {
  return *reinterpret_cast<const typename VecOf<T>::Memory*>(row + j * kPerOf<T>);
}
// The same past the caches, for logits that are read once.
template <typename T>
__device__ __forceinline__ typename VecOf<T>::Value load_once(const T* row, uint32_t j) {
  return stream_load(reinterpret_cast<const typename VecOf<T>::Memory*>(row + j * kPerOf<T>));
}
template <typename T>
__device__ __forceinline__ typename VecOf<T>::Value load_any(const T* row, uint32_t V, uint32_t j) {
  const uint32_t at = j * kPerOf<T>;
  if (at + kPerOf<T> <= V) return load_whole(row, j);
  typename VecOf<T>::Value v = lowest_vec(typename VecOf<T>::Value{});
#pragma unroll
  for (uint32_t e = 0; e < kPerOf<T>; ++e)
    if (at + e < V) set_elem(v, e, row[at + e]);
  return v;
}

// ---------------------------------------------------------------------------
// Row statistics: the largest logit m, S and A of a part of a row (0 of each where m is
// -inf), and their join.
// ---------------------------------------------------------------------------
struct Stats {
  float m, S, A;
};
__device__ __forceinline__ Stats join(Stats a, Stats b, float c) {
  const float m = larger(a.m, b.m);
  if (m == -INFINITY) return Stats{m, 0.0f, 0.0f};
  const float da = (a.m - m) * c, db = (b.m - m) * c;
  const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
  return Stats{m, fa * a.S + fb * b.S,
               fa * __builtin_fmaf(a.S, fmaxf(da, kScoreFloor), a.A) +
                   fb * __builtin_fmaf(b.S, fmaxf(db, kScoreFloor), b.A)};
}

// Of a wave's lanes, the same in every lane.
__device__ __forceinline__ Stats join_lanes(Stats s, float c) {
  const float m = wave_largest(s.m);
  const float d = s.m == -INFINITY ? kScoreFloor : (s.m - m) * c;
  const float f = __builtin_amdgcn_exp2f(d);
  s.A = wave_sum(f * __builtin_fmaf(s.S, fmaxf(d, kScoreFloor), s.A));
  s.S = wave_sum(f * s.S);
  s.m = m;
  return s;
}

// The row's statistics from its parts, the same in every lane of the wave.
__device__ __forceinline__ Stats join_parts(const Stats* parts, uint32_t count, float c) {
  Stats s{-INFINITY, 0.0f, 0.0f};
  for (uint32_t i = threadIdx.x % kWave; i < count; i += kWave) s = join(s, parts[i], c);
  return join_lanes(s, c);
}

// Keys of the largest logits of a row's groups, what one lane reads in the pass, and blocks of 16 groups.
constexpr int kBlockLanes = 16;
constexpr int kBlocksOf = kThreads / kBlockLanes;   // blocks of a segment
struct Maxima {
  uint32_t *groups, *blocks;
};
__device__ __forceinline__ Maxima row_maxima(Maxima of_launch, int64_t b, uint32_t segments) {
  return Maxima{of_launch.groups + b * segments * kThreads, of_launch.blocks + b * segments * kBlocksOf};
}
// The largest of a row of 16 lanes, in each of them.
__device__ __forceinline__ uint32_t row_largest(uint32_t k) {
  const auto step = [](uint32_t a, int b) { return max(a, static_cast<uint32_t>(b)); };
  k = step(k, __builtin_amdgcn_update_dpp(0, static_cast<int>(k), 0xB1, 0xF, 0xF, false));    // quad_perm [1,0,3,2]
  k = step(k, __builtin_amdgcn_update_dpp(0, static_cast<int>(k), 0x4E, 0xF, 0xF, false));    // quad_perm [2,3,0,1]
  k = step(k, __builtin_amdgcn_update_dpp(0, static_cast<int>(k), 0x141, 0xF, 0xF, false));   // row_half_mirror
  return step(k, __builtin_amdgcn_update_dpp(0, static_cast<int>(k), 0x140, 0xF, 0xF, false)); // row_mirror
}

__device__ __forceinline__ uint32_t wave_highest(uint32_t k) {
  k = row_largest(k);
  k = max(k, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(k), 0x142, 0xA, 0xF, false)));
  k = max(k, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(k), 0x143, 0xC, 0xF, false)));
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(k), 63));
}

// Sums over logits x relative to a base m.  (Scores by one fma, x c - m c, would save an instruction of ten,
// but the rounding of m c is past any range for rows masked with the type's lowest value.)
struct Sums {
  float base, c, S = 0.0f, A = 0.0f;
  __device__ __forceinline__ Sums(float m, float c_) : base(m == -INFINITY ? 0.0f : m), c(c_) {}
  __device__ __forceinline__ void add(float x) {
    const float y = (x - base) * c;
    const float p = __builtin_amdgcn_exp2f(y);
    S += p;
    A = __builtin_fmaf(p, fmaxf(y, kScoreFloor), A);   // 0 * -inf is no part of the sum
  }
};

// The streaming pass: one read of every logit, bound by HBM (bf16 statistics: as much by the ten
// instructions a logit, four of them its exponential: with the second launch 1024 x 128256 take 49.9 us, 5.3 TB/s,
// where 512 x 152064 fp32 move 5.8 to 6.1).  512 x 152064 fp32: 46.7-47.3 us, 6.6 TB/s; 256 x 152064 bf16, maxima
// only: 13.7 us, 5.7 TB/s; one row of 32000: 2.6 us, a launch and a memory round trip.
// A workgroup takes a segment of kThreads * kVecs
// vectors of a row, a lane kVecs of them, kThreads vectors apart.  A wave writes the statistics
// of its part; with kTop a lane also writes the key of its largest logit (its group's maximum),
// from which the selection finds the few groups that can hold one of the k largest.
//
// Sixteen lanes' maxima give the maximum of a larger group, a block, which a small k needs to look at first.
// A selection reads some of the logits again, so only a pass without one goes past the caches (512 x 152064
// fp32 without one: 53.0 us, 59.4 through them; 256 x 152064 bf16 and 20 alternatives: 23.5 and 22.0 us).
template <typename T, int kVecs, bool kStats, bool kTop>
__global__ void __launch_bounds__(kThreads)
row_pass_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, float c,
                Stats* __restrict__ parts, Maxima maxima) {
  constexpr uint32_t kPer = kPerOf<T>;
  const uint32_t j0 = blockIdx.x * (kThreads * kVecs) + threadIdx.x;
  const bool whole = (blockIdx.x + 1) * (kThreads * kVecs) <= V / kPer;
  for (int64_t b = blockIdx.y; b < B; b += gridDim.y) {
    const T* row = logits + b * row_stride;
    typename VecOf<T>::Value x[kVecs];
    if (whole) {
#pragma unroll
      for (int u = 0; u < kVecs; ++u)
        x[u] = kTop ? load_whole(row, j0 + u * kThreads) : load_once(row, j0 + u * kThreads);
    } else {
#pragma unroll
      for (int u = 0; u < kVecs; ++u) x[u] = load_any(row, V, j0 + u * kThreads);
    }
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < kVecs; ++u)
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e) m = larger(m, elem(x[u], e));
    const int64_t segment = b * gridDim.x + blockIdx.x;
    if (kTop) {
      const uint32_t key = order_key(m);
      maxima.groups[segment * kThreads + threadIdx.x] = key;
      const uint32_t of_block = row_largest(key);
      if (threadIdx.x % kBlockLanes == 0)
        maxima.blocks[segment * kBlocksOf + threadIdx.x / kBlockLanes] = of_block;
    }
    if (kStats) {
      m = wave_largest(m);
      Sums sums(m, c);
#pragma unroll
      for (int u = 0; u < kVecs; ++u)
#pragma unroll
        for (uint32_t e = 0; e < kPer; ++e) sums.add(elem(x[u], e));
      sums.S = wave_sum(sums.S);
      sums.A = wave_sum(sums.A);
      if (threadIdx.x % kWave == 0)
        parts[segment * (kThreads / kWave) + threadIdx.x / kWave] = Stats{m, sums.S, sums.A};
    }
  }
}

// ---------------------------------------------------------------------------
// The k first logits of a row in order, by one workgroup, from the maxima of its groups.
//
// A chain of short dependent steps: threshold, groups, logits and order take 11-14 thousand cycles (the kernel
// 5-8 us) for 5 to 50 of a row, 19 for 100; 1024 of 151936 take the kernel 18 us.
// A threshold t with at least k group maxima at or above it has at least k logits there, all in
// those groups; bisection stops at a t that leaves not many more than k groups.  Their logits
// from t on are gathered as (key << 32 | ~column), which no two logits share, and sorted.
// For a small k the blocks' maxima serve as well, a sixteenth as many: the first wave bisects them by itself,
// without a barrier.
// Where too many groups tie at t (a mask, equal logits), only what lies above t is gathered,
// fewer than k groups, and the rest are the first columns that equal t.  Those are looked for from column 0 on,
// 256 vectors at a time, each time a memory round trip and a barrier: where a tenth of a row's last quarter ties for
// its largest logit, 40 of 1 x 32000 fp32 take 24 us (7.6 without ties), of 1 x 152064 87 (9.5), of 256 x 152064 bf16 82
// (21.9); logits clipped or rounded so that ties stand everywhere take no longer than others.
// ---------------------------------------------------------------------------
// Two sizes: a few hundred logits by 4 waves, up to 1024 by 16.
template <bool kSmall_>
struct SelectionSize {
  static constexpr bool kSmall = kSmall_;
  static constexpr int kT = kSmall ? 256 : 1024;
  static constexpr uint32_t kList = kSmall ? 1024 : 4096;     // gathered logits
  static constexpr uint32_t kGroups = kSmall ? 512 : 2048;    // listed groups
  static constexpr int kHeld = 8;                             // groups' keys of a lane of the small size
};
// k of the small size.  Us small and large: 16 x 151936 fp32 100 13.4 and 14.9, 256 17.0 and 16.6; 64 x 128256 bf16 100
// 15.6 and 16.2, 256 20.3 and 17.6.  (Where the blocks do not suffice the large one is ahead sooner: 150 of 1 x 32000,
// 256 blocks, 17-19 and 12.)
constexpr uint32_t kSmallMost = 256;
// Gathered logits, about 1.3 k, that are ordered by counting all of them.  Us by counting and by buckets, 16 x 151936
// fp32: 40 11.0 and 11.7, 100 13.4 and 13.4, 160 15.5 and 14.7.
constexpr uint32_t kRankMost = 128;
constexpr uint32_t kBuckets = 256;       // the others are counted in their bucket of keys

template <typename Size>
struct Selection {
  uint64_t list[Size::kList], other[Size::kList];
  uint32_t starts[kBuckets];
  uint32_t groups[Size::kGroups], slots[2][Size::kT / kWave];
  uint32_t taken, listed, blocks, key, from;
};

// The sum over the workgroup of one number a wave, the same in every lane; `turn` alternates.
template <typename Size>
__device__ __forceinline__ uint32_t group_sum(uint32_t of_wave, Selection<Size>& s, uint32_t turn) {
  constexpr uint32_t kWaves = Size::kT / kWave;
  static_assert(kWaves == 4 || kWaves == 16, "the sums of a quad, or of a row of lanes");
  if (threadIdx.x % kWave == 0) s.slots[turn & 1][threadIdx.x / kWave] = of_wave;
  __syncthreads();
  int n = static_cast<int>(s.slots[turn & 1][threadIdx.x % kWaves]);
  n += __builtin_amdgcn_update_dpp(0, n, 0xB1, 0xF, 0xF, false);    // quad_perm [1,0,3,2]
  n += __builtin_amdgcn_update_dpp(0, n, 0x4E, 0xF, 0xF, false);    // quad_perm [2,3,0,1]
  if (kWaves == 16) {
    n += __builtin_amdgcn_update_dpp(0, n, 0x141, 0xF, 0xF, false);   // row_half_mirror
    n += __builtin_amdgcn_update_dpp(0, n, 0x140, 0xF, 0xF, false);   // row_mirror
  }
  return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(n));
}

// Bisection between two keys: lo has at least k at or above it, hi fewer.  The first steps go down from the
// largest logit by a half of it and more; then between the keys, which is near enough to between the
// logits where both have one sign.
struct Bisection {
  uint32_t lo, hi, step = 0;
  float reach = 1.0f;
  __device__ __forceinline__ uint32_t middle() {
    uint32_t mid = lo + (hi - lo) / 2;
    const bool first = lo == kLowestKey;
    if (step < 16 && (first || ((lo ^ hi) & 0x80000000u) != 0)) {
      const float z = logit_of_key(hi);
      const float t = first ? z - __builtin_fmaf(0.5f, fabsf(z), 1.0f) * reach : 0.5f * logit_of_key(lo) + 0.5f * z;
      const uint32_t key = __builtin_amdgcn_readfirstlane(order_key(t));
      reach *= 4.0f;
      if (key > lo && key < hi) mid = key;
    }
    ++step;
    return mid;
  }
};

// One more in a counter of LDS, lane by lane: few lanes of a wave count at a time, and the code that joins
// them is longer than they take (the kernels here run once through, and their instructions come from L2).
__device__ __forceinline__ uint32_t count_one(uint32_t& counter) {
  uint32_t one = 1;
  asm volatile("" : "+v"(one));
  return atomicAdd(&counter, one);
}

// Appends the wanted logits of the listed groups to the list (counting on beyond its end).  The row has at
// least one whole vector: a partial one is read as the last kPer columns, without those before it.
template <typename T, int kVecs, typename Size, typename F>
__device__ __forceinline__ void gather_listed(const T* row, uint32_t V, Selection<Size>& s, F wanted) {
  constexpr uint32_t kPer = kPerOf<T>;
  constexpr int kT = Size::kT;
  const uint32_t items = s.listed * kVecs;
  const auto column_of = [&](uint32_t item) {
    const uint32_t g = s.groups[item / kVecs];
    return (g / kThreads * (kThreads * kVecs) + item % kVecs * kThreads + g % kThreads) * kPer;
  };
  const auto load_at = [&](uint32_t column) {
    return *reinterpret_cast<const typename VecOf<T>::Memory*>(row + min(column, V - kPer));
  };
  if (threadIdx.x >= items) return;
  uint32_t column = column_of(threadIdx.x);
  auto x = load_at(column);
  for (uint32_t i = threadIdx.x; i < items; i += kT) {
    const uint32_t next_column = column_of(min(i + kT, items - 1));   // on its way while this one is looked at
    const auto next = load_at(next_column);
    const uint32_t first = min(column, V - kPer);
#pragma unroll
    for (uint32_t e = 0; e < kPer; ++e) {
      const uint32_t key = order_key(elem(x, e));
      if (wanted(key) && first + e >= column) {
        const uint32_t at = count_one(s.taken);
        if (at < Size::kList) s.list[at] = static_cast<uint64_t>(key) << 32 | ~(first + e);
      }
    }
    x = next;
    column = next_column;
  }
}

// What s.list holds: `taken` logits, the k first among them; where `above` is set the fewer than k above
// `key` only, and logits that equal it make up the rest.
struct Gathered {
  uint32_t taken, key;
  bool above;
};

// Whatever the row holds.  A lane holds kHeld groups' keys, and reads any others each time.
template <typename T, int kVecs, int kHeld, typename Size>
__device__ __forceinline__ Gathered gather_any(const T* row, uint32_t V, const uint32_t* maxima,
                                            uint32_t groups, uint32_t k, Selection<Size>& s) {
  constexpr uint32_t kPer = kPerOf<T>;
  constexpr int kT = Size::kT;
  constexpr uint32_t kListMost = Size::kList, kGroupsMost = Size::kGroups;
  const uint32_t tid = threadIdx.x;
  uint32_t turn = 0;
  uint32_t held[kHeld];
  uint32_t highest = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    held[i] = tid + i * kT < groups ? maxima[tid + i * kT] : 0u;   // 0 is below every key
    highest = max(highest, held[i]);
  }
  for (uint32_t g = tid + kHeld * kT; g < groups; g += kT) highest = max(highest, maxima[g]);
  highest = wave_highest(highest);
  if (tid % kWave == 0) s.slots[turn & 1][tid / kWave] = highest;
  if (tid == 0) s.taken = s.listed = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kT / kWave; ++w) highest = max(highest, s.slots[turn & 1][w]);
  ++turn;

  const auto groups_from = [&](uint32_t t) {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) n += __popcll(__ballot(held[i] >= t));
    for (uint32_t g0 = kHeld * kT; g0 < groups; g0 += kT)
      n += __popcll(__ballot(g0 + tid < groups && maxima[g0 + tid] >= t));
    return group_sum(n, s, turn++);
  };
  Bisection at{kLowestKey, highest};
  uint32_t from = groups;                       // group maxima at or above at.lo
  if (from > k) {
    const uint32_t most = k + k / 4 + 16;
    const uint32_t at_highest = groups_from(highest);
    if (at_highest >= k) {
      at.lo = highest;
      from = at_highest;
    }
    while (from > most && at.hi - at.lo > 1) {
      const uint32_t mid = at.middle();
      const uint32_t n = groups_from(mid);
      if (n >= k) {
        at.lo = mid;
        from = n;
      } else {
        at.hi = mid;
      }
    }
  }
  // `above`: what lies above at.lo only
  bool above = from > kGroupsMost;
  const auto wanted = [&](uint32_t key) { return above ? key > at.lo : key >= at.lo; };
  const auto list_group = [&](uint32_t g, uint32_t key) {
    if (!wanted(key)) return;
    const uint32_t n = count_one(s.listed);
    if (n < kGroupsMost) s.groups[n] = g;
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (tid + i * kT < groups) list_group(tid + i * kT, held[i]);
  for (uint32_t g = tid + kHeld * kT; g < groups; g += kT) list_group(g, maxima[g]);
  __syncthreads();

  // every logit of the listed groups
  const uint32_t items = s.listed * kVecs;
  const auto each_listed = [&](auto&& f) {
    for (uint32_t i = tid; i < items; i += kT) {
      const uint32_t g = s.groups[i / kVecs];
      const uint32_t j = g / kThreads * (kThreads * kVecs) + i % kVecs * kThreads + g % kThreads;
      const auto x = load_any(row, V, j);
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e)
        if (j * kPer + e < V) f(order_key(elem(x, e)), j * kPer + e);
    }
  };
  const auto gather = [&] {
    if (V >= kPer) {
      gather_listed<T, kVecs>(row, V, s, wanted);
    } else if (tid < V) {
      const uint32_t key = order_key(logit_of(row[tid]));
      if (wanted(key)) s.list[count_one(s.taken)] = static_cast<uint64_t>(key) << 32 | ~tid;
    }
    __syncthreads();
  };
  gather();
  uint32_t taken = s.taken;
  if (taken > kListMost) {
    // the largest stand together in few groups: bisection over their logits
    if (above) ++at.lo;
    above = false;
    at.hi = highest;
    at.step = 0;
    const auto logits_from = [&](uint32_t t) {
      uint32_t n = 0;
      each_listed([&](uint32_t key, uint32_t) { n += key >= t; });
#pragma unroll
      for (int d = kWave / 2; d > 0; d /= 2) n += __shfl_xor(n, d);
      return group_sum(n, s, turn++);
    };
    const uint32_t at_highest = logits_from(highest);
    if (at_highest >= k) {
      at.lo = highest;
      taken = at_highest;
    }
    while (taken > kListMost && at.hi - at.lo > 1) {
      const uint32_t mid = at.middle();
      const uint32_t n = logits_from(mid);
      if (n >= k) {
        at.lo = mid;
        taken = n;
      } else {
        at.hi = mid;
      }
    }
    above = taken > kListMost;
    __syncthreads();
    if (tid == 0) s.taken = 0;
    __syncthreads();
    gather();
    taken = s.taken;
  }
  return Gathered{taken, at.lo, above};
}

// The list filled up to k by the first columns that equal `key`.
template <typename T, typename Size>
__device__ __forceinline__ void fill_equal(const T* row, uint32_t V, uint32_t k, uint32_t taken, uint32_t key,
                                        Selection<Size>& s) {
  constexpr uint32_t kPer = kPerOf<T>;
  constexpr int kT = Size::kT;
  const uint32_t tid = threadIdx.x;
  uint32_t turn = 0;
  __syncthreads();
  for (uint32_t j0 = 0; taken < k && j0 * kPer < V; j0 += kT) {
    const uint32_t j = j0 + tid;
    uint32_t equal = 0;
    if (j * kPer < V) {
      const auto x = load_any(row, V, j);
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e)
        equal |= static_cast<uint32_t>(j * kPer + e < V && order_key(elem(x, e)) == key) << e;
    }
    uint32_t before = __popc(equal);
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const uint32_t n = __shfl_up(before, d);
      if (tid % kWave >= static_cast<uint32_t>(d)) before += n;
    }
    const uint32_t of_wave = __shfl(before, kWave - 1);
    if (tid % kWave == 0) s.slots[turn & 1][tid / kWave] = of_wave;
    __syncthreads();
    before += taken - __popc(equal);
    for (uint32_t w = 0; w < kT / kWave; ++w) {
      if (w < tid / kWave) before += s.slots[turn & 1][w];
      taken += s.slots[turn & 1][w];
    }
    ++turn;
    for (uint32_t e = 0; e < kPer; ++e)
      if (equal >> e & 1u) {
        if (before < k) s.list[before] = static_cast<uint64_t>(key) << 32 | ~(j * kPer + e);
        ++before;
      }
  }
  __syncthreads();
}

// The same for k that the blocks' maxima suffice for; `taken` is more than the list holds where they do not
// (the row's largest logits stand together).  A wave holds kHeld * 64 blocks.
template <typename T, int kVecs, int kHeld, typename Size>
__device__ __forceinline__ Gathered gather_from_blocks(const T* row, uint32_t V, Maxima maxima, uint32_t blocks,
                                                       uint32_t k, Selection<Size>& s) {
  constexpr int kT = Size::kT;
  constexpr uint32_t kListMost = Size::kList, kGroupsMost = Size::kGroups;
  const uint32_t tid = threadIdx.x;
  uint32_t* const listed_blocks = reinterpret_cast<uint32_t*>(s.list);   // until the logits are gathered
  if (tid < kWave) {
    uint32_t held[kHeld];
    uint32_t highest = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = tid + i * kWave < blocks ? maxima.blocks[tid + i * kWave] : 0u;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) highest = max(highest, held[i]);
    highest = wave_highest(highest);
    const auto blocks_from = [&](uint32_t t) {
      uint32_t n = 0;
#pragma unroll
      for (int i = 0; i < kHeld; ++i) n += __popcll(__ballot(held[i] >= t));
      return n;
    };
    const uint32_t most = k + k / 4 + 16;
    Bisection at{kLowestKey, highest};
    uint32_t from = blocks;
    const uint32_t at_highest = blocks_from(highest);
    if (at_highest >= k) {
      at.lo = highest;
      from = at_highest;
    }
    while (from > most && at.hi - at.lo > 1) {
      const uint32_t mid = at.middle();
      const uint32_t n = blocks_from(mid);
      if (n >= k) {
        at.lo = mid;
        from = n;
      } else {
        at.hi = mid;
      }
    }
    // too many blocks tie at at.lo: those above it, fewer than k
    const bool above = from > most;
    uint32_t listed = 0;
    if (!above || at.lo != 0xFFFFFFFFu) {
      const uint32_t least = at.lo + (above ? 1u : 0u);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        const uint64_t mask = __ballot(held[i] >= least);
        if (held[i] >= least)
          listed_blocks[listed + __popcll(mask & ((uint64_t{1} << tid) - 1u))] = tid + i * kWave;
        listed += __popcll(mask);
      }
    }
    if (tid == 0) {
      s.taken = s.listed = 0;
      s.blocks = listed;
      s.key = at.lo;
      s.from = above;
    }
  }
  __syncthreads();
  const bool above = s.from != 0;
  const uint32_t key_at = s.key, least = key_at + (above ? 1u : 0u);
  // the blocks' groups that reach the threshold, and their logits; several loads of a lane on their way together
  const uint32_t candidates = s.blocks * kBlockLanes;
  for (uint32_t i = tid; i < candidates; i += 4 * kT) {
    uint32_t g[4], key[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t n = min(i + j * kT, candidates - 1);
      g[j] = listed_blocks[n / kBlockLanes] * kBlockLanes + n % kBlockLanes;
      key[j] = maxima.groups[g[j]];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j * kT < candidates && key[j] >= least) {
        const uint32_t n = count_one(s.listed);
        if (n < kGroupsMost) s.groups[n] = g[j];
      }
  }
  __syncthreads();
  if (s.listed > kGroupsMost) return Gathered{kListMost + 1, key_at, above};
  gather_listed<T, kVecs>(row, V, s, [&](uint32_t key) { return key >= least; });
  __syncthreads();
  return Gathered{s.taken, key_at, above};
}

// The gathered logits in order: each to the place that counting the larger ones gives it.  Many are first put
// into buckets of neighbouring keys, in order of the buckets, so that only those of its bucket are counted.
template <typename Size>
__device__ __forceinline__ const uint64_t* sorted(uint32_t taken, Selection<Size>& s) {
  constexpr int kT = Size::kT;
  const uint32_t tid = threadIdx.x;
  // how many of list[first .. end) are larger; four reads on their way together
  const auto larger_of = [](const uint64_t* list, uint32_t first, uint32_t end, uint64_t mine) {
    uint32_t rank = 0;
    for (uint32_t n = first; n < end; n += 4) {
      uint64_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = list[min(n + i, end - 1)];
#pragma unroll
      for (int i = 0; i < 4; ++i) rank += n + i < end && x[i] > mine;
    }
    return rank;
  };
  if (taken <= kRankMost) {
    // 0 is below every logit; the list has room for a whole number of eights
    if (tid < 8) s.list[taken + tid] = 0;
    __syncthreads();
    if (tid < taken) {
      const uint64_t mine = s.list[tid];
      uint32_t rank = 0;
      for (uint32_t n = 0; n < taken; n += 8)
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) rank += s.list[n + i] > mine;
      s.other[rank] = mine;
    }
    __syncthreads();
    return s.other;
  }
  // the range of keys
  uint32_t low = 0xFFFFFFFFu, high = 0;
  for (uint32_t i = tid; i < taken; i += kT) {
    const uint32_t key = static_cast<uint32_t>(s.list[i] >> 32);
    low = min(low, key);
    high = max(high, key);
  }
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) {
    low = min(low, __shfl_xor(low, d));
    high = max(high, __shfl_xor(high, d));
  }
  for (uint32_t i = tid; i < kBuckets; i += kT) s.starts[i] = 0;
  if (tid % kWave == 0) {
    s.slots[0][tid / kWave] = low;
    s.slots[1][tid / kWave] = high;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kT / kWave; ++w) {
    low = min(low, s.slots[0][w]);
    high = max(high, s.slots[1][w]);
  }
  const int bits = 32 - __clz(high - low);            // 0 where all are equal
  const uint32_t shift = bits > 8 ? bits - 8 : 0;     // keys of a bucket: 2^shift
  const auto bucket_of = [&](uint64_t x) { return (high - static_cast<uint32_t>(x >> 32)) >> shift; };
  for (uint32_t i = tid; i < taken; i += kT) atomicAdd(&s.starts[bucket_of(s.list[i])], 1u);
  __syncthreads();
  // counts into ends: a wave sums four buckets a lane
  if (tid < kWave) {
    uint32_t n[kBuckets / kWave], total = 0;
#pragma unroll
    for (int i = 0; i < static_cast<int>(kBuckets / kWave); ++i) total += n[i] = s.starts[tid * (kBuckets / kWave) + i];
    uint32_t before = total;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const uint32_t x = __shfl_up(before, d);
      if (tid >= static_cast<uint32_t>(d)) before += x;
    }
    before -= total;
#pragma unroll
    for (int i = 0; i < static_cast<int>(kBuckets / kWave); ++i) {
      before += n[i];
      s.starts[tid * (kBuckets / kWave) + i] = before;
    }
  }
  __syncthreads();
  // from its end down, a bucket fills to its start: afterwards starts holds the starts
  for (uint32_t i = tid; i < taken; i += kT) s.other[atomicSub(&s.starts[bucket_of(s.list[i])], 1u) - 1u] = s.list[i];
  __syncthreads();
  for (uint32_t i = tid; i < taken; i += kT) {
    const uint64_t mine = s.other[i];
    const uint32_t bucket = bucket_of(mine);
    const uint32_t first = s.starts[bucket], end = bucket + 1 < kBuckets ? s.starts[bucket + 1] : taken;
    s.list[first + larger_of(s.other, first, end, mine)] = mine;
  }
  __syncthreads();
  return s.list;
}

// A function of its own, not part of its kernels: within them it has too few scalar registers and takes a third
// longer (1024 of 16 x 151936 in one run: 33 us, 24 so; later steps took it to 20).  Its pointers carry their address
// spaces, or every access of LDS and memory would be a flat one.
//
// The blocks' maxima are taken for k up to half of the blocks.  Us by blocks and by groups: 40 of 1 x 32000 fp32 7.4
// and 17.0, of 1 x 152064 9.0 and 88, of 256 x 152064 bf16 21.9 and 35.6; beyond half of 256 blocks 140 11.2 and 19.5, 180 15.2
// and 18.8, 200 23.2 and 18.5.  A form holds as few keys a lane as the row allows: 40 of 1 x 32000 7.4 us, 9.0
// with room for 20; 1000 17.1 and 18.6.
#define SBW_LDS __attribute__((address_space(3)))
#define SBW_GLOBAL __attribute__((address_space(1)))
template <typename T, int kVecs, typename Size>
__device__ __noinline__ const uint64_t* select_row(const SBW_GLOBAL T* row_, uint32_t V,
                                                   const SBW_GLOBAL uint32_t* groups,
                                                   const SBW_GLOBAL uint32_t* block_maxima, uint32_t segments,
                                                   uint32_t k, SBW_LDS Selection<Size>* selection) {
  const T* row = (const T*)row_;
  Selection<Size>& s = *(Selection<Size>*)selection;
  const Maxima maxima{(uint32_t*)groups, (uint32_t*)block_maxima};
  k = min(k, V);
  const uint32_t blocks = segments * kBlocksOf;
  Gathered r{Size::kList + 1, 0u, false};
  if constexpr (Size::kSmall) {
    if (V >= kPerOf<T> && 2 * k <= blocks) {
      if (blocks <= 5 * kWave) r = gather_from_blocks<T, kVecs, 5, Size>(row, V, maxima, blocks, k, s);
      else if (blocks <= 20 * kWave) r = gather_from_blocks<T, kVecs, 20, Size>(row, V, maxima, blocks, k, s);
    }
    __syncthreads();
  }
  if (r.taken > Size::kList) {
    const uint32_t count = segments * kThreads;
    if constexpr (Size::kSmall) r = gather_any<T, kVecs, Size::kHeld, Size>(row, V, maxima.groups, count, k, s);
    else if (count <= 5 * Size::kT) r = gather_any<T, kVecs, 5, Size>(row, V, maxima.groups, count, k, s);
    else r = gather_any<T, kVecs, 20, Size>(row, V, maxima.groups, count, k, s);
  }
  if (r.above && r.taken < k) {
    fill_equal(row, V, k, r.taken, r.key, s);
    r.taken = k;
  }
  return sorted(r.taken, s);
}

// ---------------------------------------------------------------------------
// What a call writes for each row.
// ---------------------------------------------------------------------------
struct Outputs {
  const int32_t* tokens;
  uint32_t n, top;
  float inv_t;
  uint32_t vbase;          // of the candidates' ids
  float *logprobs, *lse, *entropy, *stats;
  int32_t* top_ids;
  float* top_values;       // log probabilities, or logits of candidates
};

// A lane's given token, read before its row's statistics are known.
template <typename T>
struct Given {
  int32_t token = -1;
  float logit = 0.0f;
  __device__ __forceinline__ Given(const Outputs& o, int64_t b, const T* row, uint32_t V, uint32_t j) {
    if (j < o.n) token = o.tokens[b * o.n + j];
    if (token >= 0 && static_cast<uint32_t>(token) < V) logit = logit_of(row[token]);
    else token = -1;
  }
};

// Log sum, entropy and the given tokens' log probabilities, by `lanes` lanes; ln S.
template <typename T>
__device__ __forceinline__ float write_statistics(const Outputs& o, int64_t b, const T* row, uint32_t V, Stats r,
                                                  Given<T> given, uint32_t lane, uint32_t lanes) {
  const float ln_s = logf(r.S);
  const bool empty = r.m == -INFINITY;
  if (lane == 0) {
    if (o.lse != nullptr) o.lse[b] = empty ? -INFINITY : __builtin_fmaf(r.m, o.inv_t, ln_s);
    if (o.entropy != nullptr) o.entropy[b] = empty ? 0.0f : ln_s - kLn2 * (r.A / r.S);
    if (o.stats != nullptr) o.stats[2 * b] = r.m, o.stats[2 * b + 1] = ln_s;
  }
  for (uint32_t j = lane; j < o.n; j += lanes) {
    if (j != lane) given = Given<T>(o, b, row, V, j);
    o.logprobs[b * o.n + j] =
        given.token < 0 ? 0.0f : empty ? -INFINITY : logprob_of(given.logit, r.m, o.inv_t, ln_s);
  }
  return ln_s;
}

// The selected columns with their log probabilities (kStats) or logits.
template <bool kStats>
__device__ __forceinline__ void write_selected(const Outputs& o, int64_t b, uint32_t V, const uint64_t* best, float m,
                                               float ln_s, uint32_t lanes) {
  for (uint32_t j = threadIdx.x; j < o.top; j += lanes) {
    const bool some = j < V;
    const uint64_t x = best[some ? j : 0u];
    const float logit = logit_of_key(static_cast<uint32_t>(x >> 32));
    o.top_ids[b * o.top + j] = some ? static_cast<int32_t>(o.vbase + ~static_cast<uint32_t>(x)) : -1;
    if (o.top_values == nullptr) continue;
    o.top_values[b * o.top + j] = !some                              ? -INFINITY
                                  : !kStats                         ? logit
                                  : m == -INFINITY                   ? -INFINITY
                                                                     : logprob_of(logit, m, o.inv_t, ln_s);
  }
}

// After the pass.  Without a selection one wave a row joins the statistics and writes (a launch and the two loads of
// token and logit: 4.9 us for 512 rows); with one a workgroup.
template <typename T>
__global__ void __launch_bounds__(kThreads)
join_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, uint32_t segments,
            const Stats* __restrict__ parts, Outputs o) {
  for (int64_t b = static_cast<int64_t>(blockIdx.x) * (kThreads / kWave) + threadIdx.x / kWave; b < B;
       b += static_cast<int64_t>(gridDim.x) * (kThreads / kWave)) {
    const uint32_t count = segments * (kThreads / kWave), lane = threadIdx.x % kWave;
    const T* row = logits + b * row_stride;
    const Given<T> given(o, b, row, V, lane);
    const Stats r = join_parts(parts + b * count, count, score_factor(o.inv_t));
    write_statistics(o, b, row, V, r, given, lane, kWave);
  }
}

template <typename T, int kVecs, typename Size, bool kStats>
__global__ void __launch_bounds__(Size::kT)
select_kernel(const T* __restrict__ logits, int64_t B, uint32_t V, int64_t row_stride, uint32_t segments,
              const Stats* __restrict__ parts, Maxima maxima, Outputs o) {
  __shared__ Selection<Size> s;
  __shared__ float of_row[2];
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const T* row = logits + b * row_stride;
    // the statistics are the other waves' while the first one looks for the threshold
    if (kStats && threadIdx.x >= kWave) {
      const uint32_t lane = threadIdx.x - kWave, count = segments * (kThreads / kWave);
      const Given<T> given(o, b, row, V, lane);
      const Stats r = join_parts(parts + b * count, count, score_factor(o.inv_t));
      const float ln_s = write_statistics(o, b, row, V, r, given, lane, Size::kT - kWave);
      if (lane == 0) of_row[0] = r.m, of_row[1] = ln_s;
    }
    const Maxima m = row_maxima(maxima, b, segments);
    const uint64_t* best = select_row<T, kVecs, Size>(
        (const SBW_GLOBAL T*)row, V, (const SBW_GLOBAL uint32_t*)m.groups, (const SBW_GLOBAL uint32_t*)m.blocks,
        segments, o.top, (SBW_LDS Selection<Size>*)&s);
    write_selected<kStats>(o, b, V, best, of_row[0], of_row[1], Size::kT);
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Gradient: one read and one write of every logit, bound by HBM.  From a graph, into two gradients in turn: 256 x
// 152064 fp32 50.6 us (6.2 TB/s), 1024 x 128256 bf16 with the entropy's 84-88 us (6.0-6.3).
// ---------------------------------------------------------------------------
__device__ __forceinline__ void put_logit(float* p, float x) { *p = x; }
__device__ __forceinline__ void put_logit(uint16_t* p, float x) {
  *p = static_cast<uint16_t>(to_bf16x2(x, 0.0f));
}
__device__ __forceinline__ f32x4 packed(const float (&d)[4]) { return f32x4{d[0], d[1], d[2], d[3]}; }
__device__ __forceinline__ u32x4 packed(const float (&d)[8]) {
  return u32x4{to_bf16x2(d[0], d[1]), to_bf16x2(d[2], d[3]), to_bf16x2(d[4], d[5]), to_bf16x2(d[6], d[7])};
}
template <typename T>
__device__ __forceinline__ void store_any(T* row, uint32_t V, uint32_t j, typename VecOf<T>::Value v) {
  const uint32_t at = j * kPerOf<T>;
  if (at + kPerOf<T> <= V) {
    stream_store(reinterpret_cast<typename VecOf<T>::Memory*>(row + at), v);
    return;
  }
#pragma unroll
  for (uint32_t e = 0; e < kPerOf<T>; ++e)
    if (at + e < V) put_logit(row + at + e, elem(v, e));
}

// What a row's gradient is made of.  For column v with score y = (x_v - m) inv_t and
// log p = y - ln S:  d_v = inv_t * (p (share - g_H log p) + the gradients of the tokens v),
// share = g_lse - sum_j g_j - g_H H.  This is all but the last product, by inv_t, which comes after the sum: only
// a gradient beyond the type's range is infinite then, and a column of probability 0 has 0 for any inv_t.
struct RowGradient {
  float m, ln_s, inv_t, share, g_entropy;
  __device__ __forceinline__ float operator()(float x, float of_tokens) const {
    const float y = __builtin_fmaf(x - m, inv_t, -ln_s);
    const float p = __builtin_amdgcn_exp2f(y * kLog2e);
    return __builtin_fmaf(p, __builtin_fmaf(-g_entropy, fmaxf(y, kScoreFloor), share), of_tokens);
  }
};

// Several tokens a row (kOne is false): the first wave lists those of the segment in their order and marks their
// columns; a lane that meets a marked column adds up its gradients from the list.  One token is compared with every
// column instead: 256 x 152064 fp32 50.4 us (55.4 by the list), 1024 x 128256 bf16 84.7 (94.4).
template <typename T, int kVecs, bool kOne>
__global__ void __launch_bounds__(kThreads)
token_logprobs_grad_kernel(const T* logits, int64_t B, uint32_t V, int64_t row_stride,
                           const int32_t* __restrict__ tokens, uint32_t n,
                           const float* __restrict__ stats, const float* __restrict__ entropy,
                           const float* __restrict__ grad_logprobs,
                           const float* __restrict__ grad_lse,
                           const float* __restrict__ grad_entropy, float inv_t, T* grad,
                           int64_t grad_stride) {
  constexpr uint32_t kPer = kPerOf<T>;
  constexpr uint32_t kSegment = kThreads * kVecs * kPer;
  __shared__ uint32_t ids[kOne ? 1 : kMostTokens], marked[kOne ? 1 : kSegment / 32];
  __shared__ float gs[kOne ? 1 : kMostTokens], total_of_row;
  __shared__ uint32_t listed;
  const uint32_t j0 = blockIdx.x * (kThreads * kVecs) + threadIdx.x;
  const bool whole = (blockIdx.x + 1) * (kThreads * kVecs) <= V / kPer;
  const uint32_t first = blockIdx.x * kSegment;   // the segment's columns
  const uint32_t ids_end = min(V, 0x80000000u);   // of tokens, from where on they are negative ids
  for (int64_t b = blockIdx.y; b < B; b += gridDim.y) {
    const T* row = logits + b * row_stride;
    T* out = grad + b * grad_stride;
    typename VecOf<T>::Value x[kVecs];
    if (whole) {
#pragma unroll
      for (int u = 0; u < kVecs; ++u) x[u] = load_once(row, j0 + u * kThreads);
    } else {
#pragma unroll
      for (int u = 0; u < kVecs; ++u) x[u] = load_any(row, V, j0 + u * kThreads);
    }
    RowGradient r{stats[2 * b], stats[2 * b + 1], inv_t, 0.0f, 0.0f};
    if (grad_lse != nullptr) r.share = grad_lse[b];
    if (grad_entropy != nullptr) {
      r.g_entropy = grad_entropy[b];
      r.share = __builtin_fmaf(-r.g_entropy, entropy[b], r.share);
    }
    uint32_t token = 0xFFFFFFFFu;
    float g = 0.0f;
    if (kOne) {
      token = static_cast<uint32_t>(tokens[b]);
      if (token >= ids_end) token = 0xFFFFFFFFu;
      g = token < ids_end ? grad_logprobs[b] : 0.0f;
    } else {
      if (b != blockIdx.y) __syncthreads();   // the last row's list is done with
      if (threadIdx.x < kWave) {
        for (uint32_t i = threadIdx.x; i < kSegment / 32; i += kWave) marked[i] = 0;
        uint32_t before = 0;
        for (uint32_t i0 = 0; i0 < n; i0 += kWave) {
          const uint32_t i = i0 + threadIdx.x;
          const uint32_t t = i < n ? static_cast<uint32_t>(tokens[b * n + i]) : 0xFFFFFFFFu;
          const float of_token = t < ids_end ? grad_logprobs[b * n + i] : 0.0f;
          g += of_token;
          const bool here = t < ids_end && t - first < kSegment;
          const uint64_t mask = __ballot(here);
          if (here) {
            const uint32_t at = before + __popcll(mask & ((uint64_t{1} << threadIdx.x) - 1u));
            ids[at] = t;
            gs[at] = of_token;
            atomicOr(&marked[(t - first) / 32], 1u << (t - first) % 32);
          }
          before += __popcll(mask);
        }
        g = wave_sum(g);
        if (threadIdx.x == 0) {
          total_of_row = g;
          listed = before;
        }
      }
      __syncthreads();
      g = total_of_row;
    }
    r.share -= g;
    const bool empty = r.m == -INFINITY;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      const uint32_t j = j0 + u * kThreads;
      float d[kPer];
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e) d[e] = r(elem(x[u], e), kOne && j * kPer + e == token ? g : 0.0f);
      if (!kOne) {
        const uint32_t at = j * kPer - first;
        const uint32_t marks = marked[at / 32] >> at % 32 & ((1u << kPer) - 1u);
        if (marks != 0) {
#pragma unroll
          for (uint32_t e = 0; e < kPer; ++e) {
            if ((marks >> e & 1u) == 0) continue;
            float of_column = 0.0f;
            for (uint32_t i = 0; i < listed; ++i) of_column += ids[i] == j * kPer + e ? gs[i] : 0.0f;
            d[e] += of_column;
          }
        }
      }
#pragma unroll
      for (uint32_t e = 0; e < kPer; ++e) d[e] *= inv_t;
      if (empty) {
#pragma unroll
        for (uint32_t e = 0; e < kPer; ++e) d[e] = 0.0f;
      }
      store_any(out, V, j, packed(d));
    }
  }
}

// ---------------------------------------------------------------------------
// Launch shapes.
// ---------------------------------------------------------------------------
// Vectors of a lane in the pass: the long form reads 32 logits, the short one 8.
template <typename T>
constexpr int kLongVecs = sizeof(T) == 4 ? 8 : 4;
template <typename T>
constexpr int kShortVecs = sizeof(T) == 4 ? 2 : 1;
constexpr int64_t kLongSegment = kThreads * 32, kShortSegment = kThreads * 8;

// Whether the pass takes the long form: rows that make enough workgroups of it, and so many blocks that the
// selection is left with few.  Us of a call, long and short: 128256 columns, no alternatives, fp32 8 rows 6.2 and 6.6, 32
// (512 workgroups) 8.4 and 8.8, 512 43.7 and 46.4, bf16 512 26.1 and 34.4; with 20 alternatives bf16 16 rows 9.9 and
// 11.2, 64 12.8 and 15.0, 512 30.2 and 43.5.  32000 columns, fp32 16 rows 5.5 and 4.8, 128 (512 workgroups) 8.6 and 7.9, 1024
// 24.9 and 26.2; with 20 alternatives 9.0 and 8.0, 12.4 and 11.7, 37.8 and 34.9.  So the length of a row would tell the
// better form more often than the number of workgroups does, which is off by up to 1.3 us below 512 of them and 3
// above.  For a large k only with eight groups for each, as every vector of a listed group
// is another line to fetch, or where the lanes could not hold the short form's (1024 of 16 x 151936
// fp32: 20.9 us short, 23.6 long; 500 of 100 x 150000 bf16, 24.7 and 22.3).
bool long_segments(int64_t B, int64_t V, int64_t top) {
  const int64_t segments = (V + kLongSegment - 1) / kLongSegment;
  if (top > kSmallMost) return V / 32 >= 8 * top || V / 8 > 20 * SelectionSize<false>::kT;
  return B * segments >= 512 && segments * kBlocksOf >= 2 * top;
}
int64_t segments_of(int64_t B, int64_t V, int64_t top) {
  const int64_t size = long_segments(B, V, top) ? kLongSegment : kShortSegment;
  return (V + size - 1) / size;
}
// uint64 elements of the workspace a segment takes: the statistics of its waves, a key a lane and a block
constexpr int64_t kPartElems = sizeof(Stats) * (kThreads / kWave) / 8;
constexpr int64_t kMaximaElems = (kThreads + kBlocksOf) / 2;

Maxima maxima_at(uint64_t* p, int64_t B, int64_t segments) {
  auto* groups = reinterpret_cast<uint32_t*>(p);
  return Maxima{groups, groups + B * segments * kThreads};
}

template <typename T, bool kStats, bool kTop>
void launch_pass(const T* logits, int64_t B, uint32_t V, int64_t row_stride, float c, int64_t top, uint64_t* parts,
                 Maxima maxima, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(segments_of(B, V, top)),
                  static_cast<uint32_t>(B < kMaxGridY ? B : kMaxGridY));
  auto* kernel = long_segments(B, V, top) ? row_pass_kernel<T, kLongVecs<T>, kStats, kTop>
                                          : row_pass_kernel<T, kShortVecs<T>, kStats, kTop>;
  kernel<<<grid, kThreads, 0, stream>>>(logits, B, V, row_stride, c, reinterpret_cast<Stats*>(parts), maxima);
}

template <typename T, bool kStats>
void launch_rows(const void* logits_, int64_t B, uint32_t V, int64_t row_stride, const Outputs& o,
                 uint64_t* workspace, hipStream_t stream) {
  const T* logits = static_cast<const T*>(logits_);
  const uint32_t rows = static_cast<uint32_t>(grid_for(B));
  const bool small = o.top <= kSmallMost;
  const auto segments = static_cast<uint32_t>(segments_of(B, V, o.top));
  const auto* parts = reinterpret_cast<const Stats*>(workspace);
  const float c = score_factor(o.inv_t);
  if (o.top == 0) {
    if constexpr (kStats) {
      launch_pass<T, true, false>(logits, B, V, row_stride, c, 0, workspace, Maxima{}, stream);
      join_kernel<T><<<static_cast<uint32_t>(grid_for((B + 3) / 4)), kThreads, 0, stream>>>(
          logits, B, V, row_stride, segments, parts, o);
    }
    return;
  }
  const Maxima maxima = maxima_at(workspace + (kStats ? B * segments * kPartElems : 0), B, segments);
  launch_pass<T, kStats, true>(logits, B, V, row_stride, c, o.top, workspace, maxima, stream);
  using Small = SelectionSize<true>;
  using Large = SelectionSize<false>;
  auto* kernel = long_segments(B, V, o.top) ? (small ? select_kernel<T, kLongVecs<T>, Small, kStats>
                                                     : select_kernel<T, kLongVecs<T>, Large, kStats>)
                                            : (small ? select_kernel<T, kShortVecs<T>, Small, kStats>
                                                     : select_kernel<T, kShortVecs<T>, Large, kStats>);
  kernel<<<rows, small ? Small::kT : Large::kT, 0, stream>>>(logits, B, V, row_stride, segments, parts, maxima, o);
}

template <typename T>
void launch_grad(const void* logits, int64_t B, uint32_t V, int64_t row_stride, const int32_t* tokens, uint32_t n,
                 const float* stats, const float* entropy, const float* grad_logprobs, const float* grad_lse,
                 const float* grad_entropy, float inv_t, void* grad, int64_t grad_stride, hipStream_t stream) {
  // Two vectors a lane, past the caches both ways, into a buffer that the last call did not write.  In one run, fp32
  // 256 x 152064: 50.8 us (four vectors 53.5, stores through the caches 56.6); bf16 1024 x 128256: 84.1 (one vector
  // 89.9, through the caches 91.2).
  constexpr int kVecs = 2;
  constexpr int64_t kSegment = kThreads * kVecs * kPerOf<T>;
  const dim3 grid(static_cast<uint32_t>((V + kSegment - 1) / kSegment),
                  static_cast<uint32_t>(B < kMaxGridY ? B : kMaxGridY));
  if (grad_logprobs == nullptr) n = 0;
  const auto launch = [&](auto* kernel) {
    kernel<<<grid, kThreads, 0, stream>>>(static_cast<const T*>(logits), B, V, row_stride, tokens, n, stats, entropy,
                                           grad_logprobs, grad_lse, grad_entropy, inv_t, static_cast<T*>(grad),
                                           grad_stride);
  };
  if (n == 1) launch(token_logprobs_grad_kernel<T, kVecs, true>);
  else launch(token_logprobs_grad_kernel<T, kVecs, false>);
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
  if (B <= 0 || V <= 0 || V > kMostColumns || top < 0 || top > kMostTokens) return 0;
  return B * segments_of(B, V, top) * (kPartElems + (top > 0 ? kMaximaElems : 0));
}

int64_t sbw_top_candidates_workspace(int64_t B, int64_t V, int64_t k) {
  if (B <= 0 || V <= 0 || V > kMostColumns || k < 1 || k > kMostTokens) return 0;
  return B * segments_of(B, V, k) * kMaximaElems;
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
  const Outputs o{tokens, static_cast<uint32_t>(n), static_cast<uint32_t>(top), inv_temperature, 0u, logprobs, lse,
                  entropy, stats, top_ids, top_logprobs};
  auto* launch = dtype == SBW_F32 ? launch_rows<float, true> : launch_rows<uint16_t, true>;
  launch(logits, B, static_cast<uint32_t>(V), row_stride, o, workspace, st);
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
  auto* launch = dtype == SBW_F32 ? launch_grad<float> : launch_grad<uint16_t>;
  launch(logits, B, static_cast<uint32_t>(V), row_stride, tokens, static_cast<uint32_t>(n), stats, entropy,
         grad_logprobs, grad_lse, grad_entropy, inv_temperature, grad, grad_stride, st);
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
  const Outputs o{nullptr, 0u, static_cast<uint32_t>(k), 1.0f, static_cast<uint32_t>(v_offset), nullptr, nullptr,
                  nullptr, nullptr, ids, values};
  auto* launch = dtype == SBW_F32 ? launch_rows<float, false> : launch_rows<uint16_t, false>;
  launch(logits, B, static_cast<uint32_t>(V), row_stride, o, workspace, st);
  return after_launch();
}

}  // extern "C"
