// Bounds of the keys in each page of a paged cache, and for each unit (sequence, layer, KV head) the pages that its queries can score highest in.
//
// A page's bounds are the lowest and the largest key of every column.  No key within them has a dot product with q above sum_c max(q_c low_c,
// q_c high_c), so that the sum over the G query heads of a unit, sum_c high_c up_c + low_c down_c with up_c = sum_g max(q_gc, 0) and
// down_c = sum_g min(q_gc, 0), ranks pages without reading their keys.  It is summed in 64 bits and rounded to 32 once: another
// order of summation changes a sum by some 2^-53 of its terms, and the score only where that crosses the middle between two values of 32 bits.
//
// A few bytes and operations a page: bound by chains of loads and by the search for the smallest key that is taken.  From 64 units on a workgroup has a
// unit, scores and choice: 112 units of 512 pages 15 us (scores 9.7), 896 of 102 pages 16 (12.2); as two kernels 9.0 + 5.2 and 15.6 + 6.5.  Fewer units'
// scores are shared out over more workgroups: 4 units of 512 pages 4.3 + 5.1, unless a unit's bounds are at most half of what sixteen
// waves have under way at once (64 KB): 1 to 63 units of 64 pages of 128 bf16 columns one after another 4.2 to 5.0 in place of 5.7 to 6.5.  64-bit arithmetic is not what takes the time (products left out: the same).
#include <algorithm>
#include <type_traits>

#include "fc_common.h"
#include "paged.h"

namespace fc {

namespace {

constexpr int kBoundThreads = 256, kBoundWaves = kBoundThreads / 64;
constexpr int kRowsAtOnce = 8;         // of a lane
constexpr int kScoreThreads = 256, kScoreWaves = kScoreThreads / 64;
constexpr int kPagesAtOnce = 4, kQueriesAtOnce = 8;
constexpr int kMostKeys = 4096;        // that a workgroup has in LDS, or in registers
constexpr int kFewBounds = 65536;      // bytes of a unit's bounds

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of a row as fp32
template <typename T> struct Columns;
template <> struct Columns<uint16_t> {
  static constexpr int kCount = 8;
  static __device__ __forceinline__ void get(const u32x4& v, float (&o)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __uint_as_float(v[i] << 16);
      o[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ u32x4 put(const float (&x)[8]) {      // (values that are bf16 already)
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xFFFF0000u);
    return v;
  }
};
template <> struct Columns<float> {
  static constexpr int kCount = 4;
  static __device__ __forceinline__ void get(const u32x4& v, float (&o)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(v[i]);
  }
  static __device__ __forceinline__ u32x4 put(const float (&x)[4]) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};

// A wave looks 64 entries of the tables up at a time, a lane each, and then works on the pages that there are, one after another.  Entries are
// dealt out in the order of place in the table, then unit: what lies behind the last row is last for all units.  Bound by memory: 11 500 pages of 64 rows of
// 256 bytes (0.19 GB) 36 us, 5.3 TB/s, past the last-level cache; 42 with a claim on it, however many rows or waves are under way.
template <typename T>
__global__ __launch_bounds__(kBoundThreads) void page_bounds_kernel(PagedArgs a, int row_bytes, char* __restrict__ bounds) {
  typedef Columns<T> C;
  constexpr int N = C::kCount;
  const int lane = threadIdx.x & 63, lanes = row_bytes / 16, abreast = 64 / lanes, mine = lane / lanes, part = lane - mine * lanes;
  const int64_t waves = (int64_t)gridDim.x * kBoundWaves, wave = (int64_t)blockIdx.x * kBoundWaves + (threadIdx.x >> 6);
  const int64_t units = (int64_t)a.B * a.L * a.H, items = units * a.max_pages;
  for (int64_t base = wave; base < items; base += 64 * waves) {
    const int64_t item = base + lane * waves;
    int page = -1, rows = 0;
    if (item < items) {
      const int at = (int)(item / units), u = (int)(item - at * units), b = u / (a.L * a.H), in = u - b * a.L * a.H;
      rows = (int)max((int64_t)0, min((int64_t)a.page_size, rows_of(a, b, in / a.H) - (int64_t)at * a.page_size));
      if (rows > 0) page = a.table[b * a.table_b + (int64_t)in * a.max_pages + at];
    }
    uint64_t there = __ballot(rows > 0 && page >= 0 && page < a.num_pages);
    while (there) {
      const int from = __builtin_ctzll(there);
      there &= there - 1;
      const int64_t pg = __builtin_amdgcn_readlane(page, from);
      const int n = __builtin_amdgcn_readlane(rows, from);
      const char* const k = static_cast<const char*>(a.K) + pg * a.page_size * row_bytes + part * 16;
      float low[N], high[N];
#pragma unroll
      for (int i = 0; i < N; ++i) { low[i] = INFINITY; high[i] = -INFINITY; }
      if (mine < abreast)
        for (int r = mine; r < n; r += abreast * kRowsAtOnce) {
          u32x4 v[kRowsAtOnce];
#pragma unroll
          for (int j = 0; j < kRowsAtOnce; ++j) v[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(k + (int64_t)min(r + j * abreast, n - 1) * row_bytes));
#pragma unroll
          for (int j = 0; j < kRowsAtOnce; ++j) {
            float x[N];
            C::get(v[j], x);
#pragma unroll
            for (int i = 0; i < N; ++i) { low[i] = fminf(low[i], x[i]); high[i] = fmaxf(high[i], x[i]); }
          }
        }
      for (int r = 1; r < abreast; ++r)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float l = __shfl(low[i], (lane + r * lanes) & 63, 64), g = __shfl(high[i], (lane + r * lanes) & 63, 64);
          if (mine == 0) { low[i] = fminf(low[i], l); high[i] = fmaxf(high[i], g); }
        }
      if (mine == 0) {
        char* const to = bounds + 2 * pg * row_bytes + part * 16;
        *reinterpret_cast<u32x4*>(to) = C::put(low);
        *reinterpret_cast<u32x4*>(to + row_bytes) = C::put(high);
      }
    }
  }
}

// What is compared in place of a score: 0 for a page that is not there, 1 for a score that is not a number, all ones for one that is taken whatever its score.
__device__ __forceinline__ uint32_t key_of(float score) {
  if (score != score) return 1u;
  const uint32_t u = __float_as_uint(score == 0.f ? 0.f : score);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ double add_lanes_16(double v) { // the sum over each 16 lanes, in all of them
  auto moved = [](double x, auto ctrl) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, decltype(ctrl)::value, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), decltype(ctrl)::value, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  v += moved(v, std::integral_constant<int, 0xB1>{});      // quad_perm: the neighbour, then the other pair
  v += moved(v, std::integral_constant<int, 0x4E>{});
  v += moved(v, std::integral_constant<int, 0x141>{});     // row_half_mirror, row_mirror
  return v + moved(v, std::integral_constant<int, 0x140>{});
}

__device__ __forceinline__ float as_float(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float as_float(float x) { return x; }

// What a unit's queries make of each column, up and down.  A thread sums up a column, all find theirs in LDS; the caller has a barrier between both.
// (Each query to its own sum: differences of sums over all would lose a small one of the other sign.  One that is not a number goes to both.)
template <typename T, int D> __device__ __forceinline__ void sum_queries(const T* q, int G, double (*sums)[D], int thread) {
  if (thread >= D) return;
  double up = 0.0, down = 0.0;
  for (int g0 = 0; g0 < G; g0 += kQueriesAtOnce) {
    T v[kQueriesAtOnce];
#pragma unroll
    for (int j = 0; j < kQueriesAtOnce; ++j) v[j] = q[(int64_t)min(g0 + j, G - 1) * D + thread];
#pragma unroll
    for (int j = 0; j < kQueriesAtOnce; ++j) {
      const float x = as_float(v[j]);
      if (g0 + j < G) {
        up += (double)(x < 0.f ? 0.f : x);
        down += (double)(x > 0.f ? 0.f : x);
      }
    }
  }
  sums[0][thread] = up;
  sums[1][thread] = down;
}

// Keys of pages first, first + stride, ... (a wave's; kAbreast side by side, kPagesAtOnce of a lane group under way together), of a unit's `blocks`.
// The queries (at q) are summed up behind the first requests.
template <typename T, int D, typename Put>
__device__ __forceinline__ int score_pages(const PagedArgs& a, int b, int in, const T* bounds, const T* q, int G, double (*sums)[D], int begin, int stride,
                                           int first, int last, int lane, const Put& put) {
  typedef Columns<T> C;
  constexpr int N = C::kCount, kLanes = D / N, kAbreast = 64 / kLanes;
  const int mine = lane / kLanes, part = lane % kLanes;
  const int32_t* const table = a.table + b * a.table_b + (int64_t)in * a.max_pages;
  int page[kPagesAtOnce];
  auto look_up = [&](int p0) {
#pragma unroll
    for (int j = 0; j < kPagesAtOnce; ++j) page[j] = table[min(p0 + j * kAbreast + mine, a.max_pages - 1)];
  };
  look_up(begin);
  const int blocks = pages_of(a, b, in / a.H);
  u32x4 low[kPagesAtOnce], high[kPagesAtOnce];
  bool there[kPagesAtOnce];
  auto request = [&](int p0) {
#pragma unroll
    for (int j = 0; j < kPagesAtOnce; ++j) {
      there[j] = p0 + j * kAbreast + mine < blocks && page[j] >= 0 && page[j] < a.num_pages;
      const T* const from = bounds + (int64_t)(there[j] ? page[j] : 0) * 2 * D + part * N;
      low[j] = *reinterpret_cast<const u32x4*>(from);
      high[j] = *reinterpret_cast<const u32x4*>(from + D);
    }
  };
  if (begin < blocks) request(begin);
  sum_queries<T, D>(q, G, sums, threadIdx.x);
  __syncthreads();
  auto over_lanes = [](double s) {
    if constexpr (kLanes == 8) {
#pragma unroll
      for (int d = 4; d; d >>= 1) s += __shfl_xor(s, d, 64);
    } else {
      s = add_lanes_16(s);
      if (kLanes == 32) s += __shfl_xor(s, 16, 64);
    }
    return s;
  };
  float largest = 0.f;                                     // of all scores, infinity if one is not a number
  double up[N], down[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    up[i] = sums[0][part * N + i];
    down[i] = sums[1][part * N + i];
  }
  for (int p0 = begin; p0 < blocks; p0 += stride) {
    const bool more = p0 + stride < blocks;
    if (more) look_up(p0 + stride);
    double s[kPagesAtOnce];
    bool had[kPagesAtOnce];
#pragma unroll
    for (int j = 0; j < kPagesAtOnce; ++j) {
      float x[N], y[N];
      C::get(low[j], x);
      C::get(high[j], y);
      had[j] = there[j];
      s[j] = 0.0;
#pragma unroll
      for (int i = 0; i < N; ++i) s[j] = fma((double)x[i], down[i], fma((double)y[i], up[i], s[j]));
    }
    if (more) request(p0 + stride);
#pragma unroll
    for (int j = 0; j < kPagesAtOnce; ++j) {
      s[j] = over_lanes(s[j]);
      largest = fmaxf(largest, s[j] == s[j] ? fabsf((float)s[j]) : INFINITY);
      const int p = p0 + j * kAbreast + mine;
      if (part == 0 && p < blocks) put(p, !had[j] ? 0u : (p < first || p >= blocks - last) ? 0xFFFFFFFFu : key_of((float)s[j]));
    }
  }
  if (!__any(largest == INFINITY)) return blocks;
  // Pages with an infinite bound, or queries that are infinite (or no numbers), once more: 0 times infinity is 0 there, and a column whose keys are all NaNs,
  // +infinity and -infinity its bounds, counts as one that reaches from -infinity to +infinity.  (A loop by itself: in the one above its registers
  // leave fewer waves, 17.5 us in place of 16.2.)
  auto product = [](float bound, double query) {
    const double p = (double)bound * query;
    return p != p && bound == bound && query == query ? 0.0 : p;
  };
#pragma unroll 1
  for (int p0 = begin; p0 < blocks; p0 += stride)
#pragma unroll 1
    for (int j = 0; j < kPagesAtOnce; ++j) {
      const int p = p0 + j * kAbreast + mine, at = p < blocks ? table[p] : -1;
      const bool is = at >= 0 && at < a.num_pages;
      const T* const from = bounds + (int64_t)(is ? at : 0) * 2 * D + part * N;
      double s = 0.0;
      bool odd = false;
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        const float x = as_float(from[i]), y = as_float(from[D + i]);
        const double u = sums[0][part * N + i], d = sums[1][part * N + i];
        const bool none = x == INFINITY && y == -INFINITY;
        odd = odd || !(fabs((double)x) + fabs((double)y) + fabs(u) + fabs(d) < (double)INFINITY);
        s += product(none ? INFINITY : y, u) + product(none ? -INFINITY : x, d);
      }
      s = over_lanes(s);
      const uint64_t odd_lanes = __ballot(odd) >> (mine * kLanes) & (~0ull >> (64 - kLanes));
      if (part == 0 && is && odd_lanes && p >= first && p < blocks - last) put(p, key_of((float)s));
    }
  return blocks;
}

// grid = (parts of a unit's pages, units): few units of more than a few pages, or more pages than choose_whole_kernel has room for
template <typename T, int D>
__global__ __launch_bounds__(kScoreThreads) void page_score_kernel(PagedArgs a, const T* __restrict__ Q, int G, const T* __restrict__ bounds, int first, int last,
                                                                   uint32_t* __restrict__ keys) {
  constexpr int kAtATime = 64 / (D / Columns<T>::kCount) * kPagesAtOnce;
  __shared__ double sums[2][D];
  const int u = blockIdx.y, b = u / (a.L * a.H), in = u - b * a.L * a.H;
  const int waves = gridDim.x * kScoreWaves, wave = blockIdx.x * kScoreWaves + (threadIdx.x >> 6);
  score_pages<T, D>(a, b, in, bounds, Q + (int64_t)u * G * D, G, sums, wave * kAtATime, waves * kAtATime, first, last, threadIdx.x & 63, [&](int p, uint32_t key) { keys[(int64_t)u * a.max_pages + p] = key; });
}

// The `count` largest keys of a unit, of equal ones the first, in the order of the table, by WAVES waves (thread `tid` of them).  The smallest key that
// is taken is found bit by bit, by ballots.  A lane has up to K keys in registers, and where there are more reads all of them again for each bit.
template <int K, int WAVES, typename Get>
__device__ __forceinline__ void choose_largest(int blocks, int count, int tid, const Get& get, int32_t* __restrict__ out) {
  constexpr int kThreads = 64 * WAVES, kHeld = K * kThreads;
  __shared__ int counts[2][WAVES], both[2][WAVES];
  const int lane = tid & 63, wave = tid >> 6;
  uint32_t held[K];
  auto load = [&](int base) {
#pragma unroll
    for (int j = 0; j < K; ++j) held[j] = get(min(base + j * kThreads + tid, max(blocks - 1, 0)));
#pragma unroll
    for (int j = 0; j < K; ++j) held[j] = base + j * kThreads + tid < blocks ? held[j] : 0u;
  };
  load(0);
  const bool whole = blocks <= kHeld;
  int turn = 0;
  auto over_waves = [&](int n) {
    if constexpr (WAVES == 1) return n;
    if (lane == 0) counts[turn][wave] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) n += counts[turn][w];
    turn ^= 1;
    return n;
  };
  auto at_least = [&](uint32_t least) {                    // (least > 0)
    int n = 0;
    for (int base = 0; base < blocks; base += kHeld) {
      if (!whole) load(base);
#pragma unroll
      for (int j = 0; j < K; ++j) n += __popcll(__ballot(held[j] >= least));
    }
    return over_waves(n);
  };
  const int want = min(count, at_least(1u));
  uint32_t least = 0u;
  int with_least = 0;                                      // how many of those that are equal to it
  if (want > 0) {
    bool exact = false;                                    // as many keys as are wanted are not smaller: they are the ones
    for (int bit = 31; bit >= 0 && !exact; --bit) {
      const int n = at_least(least | 1u << bit);
      if (n >= want) least |= 1u << bit;
      exact = n == want;
    }
    with_least = exact ? want : want - (least == 0xFFFFFFFFu ? 0 : at_least(least + 1u));
  }
  int above = 0, equal = 0;                                // before this place
  if constexpr (WAVES > 1) __syncthreads();                // (all have read the last count)
  if (want > 0)
    for (int base = 0; base < blocks; base += kHeld) {
      if (!whole) load(base);
#pragma unroll
      for (int j = 0; j < K; ++j) {
        const uint64_t gt = __ballot(held[j] > least), eq = __ballot(held[j] == least), before = (1ull << lane) - 1ull;
        int gt_before = above + __popcll(gt & before), eq_before = equal + __popcll(eq & before);
        if constexpr (WAVES == 1) {
          above += __popcll(gt);
          equal += __popcll(eq);
        } else {
          if (lane == 0) { counts[j & 1][wave] = __popcll(gt); both[j & 1][wave] = __popcll(eq); }
          __syncthreads();
#pragma unroll
          for (int w = 0; w < WAVES; ++w) {
            const int g = counts[j & 1][w], e = both[j & 1][w];
            if (w < wave) { gt_before += g; eq_before += e; }
            above += g;
            equal += e;
          }
        }
        if (held[j] > least || (held[j] == least && eq_before < with_least)) out[gt_before + min(eq_before, with_least)] = base + j * kThreads + tid;
      }
    }
  for (int i = want + tid; i < count; i += kThreads) out[i] = -1;
}

// ... by a wave alone where it has registers for all keys: a barrier for each bit costs more than the others' help.
template <int WAVES, typename Get>
__device__ __forceinline__ void choose_by(int blocks, int count, const Get& get, int32_t* out) {
  if (blocks <= 8 * 64) {
    if (threadIdx.x >= 64) return;
    if (blocks <= 2 * 64) choose_largest<2, 1>(blocks, count, threadIdx.x, get, out);
    else if (blocks <= 4 * 64) choose_largest<4, 1>(blocks, count, threadIdx.x, get, out);
    else choose_largest<8, 1>(blocks, count, threadIdx.x, get, out);
  } else {
    choose_largest<kMostKeys / (64 * WAVES), WAVES>(blocks, count, threadIdx.x, get, out);
  }
}

__global__ __launch_bounds__(1024) void choose_kernel(PagedArgs a, const uint32_t* __restrict__ keys, int count, int32_t* __restrict__ chosen) {
  const int u = blockIdx.x, b = u / (a.L * a.H), in = u - b * a.L * a.H;
  const uint32_t* const key = keys + (int64_t)u * a.max_pages;
  choose_by<16>(pages_of(a, b, in / a.H), count, [&](int p) { return key[p]; }, chosen + (int64_t)u * count);
}

// Both in one: a workgroup a unit, keys in LDS.
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 4) void choose_whole_kernel(PagedArgs a, const T* __restrict__ Q, int G, const T* __restrict__ bounds, int count, int first,
                                                                  int last, int32_t* __restrict__ chosen) {
  constexpr int kAtATime = 64 / (D / Columns<T>::kCount) * kPagesAtOnce;
  __shared__ double sums[2][D];
  extern __shared__ uint32_t keys[];
  const int u = blockIdx.x, b = u / (a.L * a.H), in = u - b * a.L * a.H, wave = threadIdx.x >> 6;
  const int blocks = score_pages<T, D>(a, b, in, bounds, Q + (int64_t)u * G * D, G, sums, wave * kAtATime, WAVES * kAtATime, first, last, threadIdx.x & 63,
                                       [&](int p, uint32_t key) { keys[p] = key; });
  __syncthreads();
  choose_by<WAVES>(blocks, count, [&](int p) { return keys[p]; }, chosen + (int64_t)u * count);
}

}  // namespace

hipError_t page_bounds_launch(const fc_paged_kv& kv, void* bounds, hipStream_t s) {
  const PagedArgs a = paged_args(kv);
  const int64_t items = (int64_t)a.B * a.L * a.H * a.max_pages;
  const unsigned groups = (unsigned)std::min<int64_t>(2048, (items + kBoundWaves - 1) / kBoundWaves);
  const int e = kv.dtype == FC_BF16 ? 2 : 4;
  ProfileScope ps("page_bounds_kernel", s);
  auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(groups), dim3(kBoundThreads), 0, s, a, kv.head_dim * e, static_cast<char*>(bounds)); };
  kv.dtype == FC_BF16 ? launch(page_bounds_kernel<uint16_t>) : launch(page_bounds_kernel<float>);
  return hipGetLastError();
}

size_t choose_workspace_bytes(int64_t units, int max_pages) { return (size_t)units * max_pages * sizeof(uint32_t); }

hipError_t choose_launch(const void* Q, int group, const fc_paged_kv& kv, const void* bounds, int count, int first, int last, int32_t* chosen, void* ws,
                         hipStream_t s) {
  const PagedArgs a = paged_args(kv);
  const int units = a.B * a.L * a.H;
  uint32_t* const keys = static_cast<uint32_t*>(ws);
  auto by_type = [&](auto launch) {
    if (kv.dtype == FC_BF16) kv.head_dim == 128 ? launch(uint16_t{}, std::integral_constant<int, 128>{}) : launch(uint16_t{}, std::integral_constant<int, 64>{});
    else kv.head_dim == 128 ? launch(float{}, std::integral_constant<int, 128>{}) : launch(float{}, std::integral_constant<int, 64>{});
  };
  // many units, or few pages (one launch in place of two, at 1 to 63 units one after another: 128 pages of 128 bf16 columns 5.3 to 5.8 us, 6.4 to 7.1;
  // 256, or 64 KB more, 6.8 to 7.5 and 6.3 to 7.5, 512 10.9 to 11.9 and 7.7 to 9.7)
  const bool few = (int64_t)a.max_pages * 2 * kv.head_dim * (kv.dtype == FC_BF16 ? 2 : 4) <= kFewBounds;
  if (a.max_pages <= kMostKeys && (units >= 64 || few)) {
    ProfileScope ps("choose_whole_kernel", s);
    by_type([&](auto type, auto dim) {
      typedef decltype(type) T;
      constexpr int D = decltype(dim)::value;
      auto launch = [&](auto kern, int waves) {
        hipLaunchKernelGGL(kern, dim3(units), dim3(64 * waves), a.max_pages * sizeof(uint32_t), s, a, static_cast<const T*>(Q), group, static_cast<const T*>(bounds),
                           count, first, last, chosen);
      };
      // (112 units of 512 pages: sixteen waves each 14 us, four 19; of more units four, so that several are on a compute unit)
      units <= 256 ? launch(choose_whole_kernel<T, D, 16>, 16) : launch(choose_whole_kernel<T, D, 4>, 4);
    });
    return hipGetLastError();
  }
  {
    ProfileScope ps("page_score_kernel", s);
    const int at_a_time = 64 / (kv.head_dim / (kv.dtype == FC_BF16 ? 8 : 4)) * kPagesAtOnce * kScoreWaves;
    const unsigned parts = (unsigned)std::max(1, std::min((a.max_pages + at_a_time - 1) / at_a_time, (4096 + units - 1) / units));
    by_type([&](auto type, auto dim) {
      typedef decltype(type) T;
      hipLaunchKernelGGL((page_score_kernel<T, decltype(dim)::value>), dim3(parts, units), dim3(kScoreThreads), 0, s, a, static_cast<const T*>(Q), group,
                         static_cast<const T*>(bounds), first, last, keys);
    });
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ProfileScope ps("choose_kernel", s);
  hipLaunchKernelGGL(choose_kernel, dim3(units), dim3(1024), 0, s, a, static_cast<const uint32_t*>(keys), count, chosen);
  return hipGetLastError();
}

}  // namespace fc
