// Bounds of the keys in each page of a paged cache, and for each unit (sequence, layer, KV head) the pages that its queries can score highest in.
//
// A page's bounds are the lowest and the largest key of every column.  No key within them has a dot product with q above sum_c max(q_c low_c,
// q_c high_c), so that the sum over the G query heads of a unit, sum_c high_c up_c + low_c down_c with up_c = sum_g max(q_gc, 0) and
// down_c = sum_g min(q_gc, 0), ranks pages without reading their keys.  It is summed in 64 bits and rounded to 32 once: the order of the
// pages then does not depend on the order of the sum.
#include <algorithm>

#include "fc_common.h"
#include "paged.h"

namespace fc {

namespace {

constexpr int kBoundThreads = 256, kBoundWaves = kBoundThreads / 64;
constexpr int kRowsAtOnce = 4;         // of a lane
constexpr int kScoreThreads = 256, kScoreWaves = kScoreThreads / 64;
constexpr int kChooseThreads = 256;

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
// dealt out in the order of place in the table, then unit: what lies behind the last row is last for all units.
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
      rows = rows_of(a, b, in / a.H) - at * a.page_size;
      rows = min(rows, a.page_size);
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
          for (int j = 0; j < kRowsAtOnce; ++j) v[j] = *reinterpret_cast<const u32x4*>(k + (int64_t)min(r + j * abreast, n - 1) * row_bytes);
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

// grid = (parts of a unit's pages, units)
template <typename T, int D>
__global__ __launch_bounds__(kScoreThreads) void page_score_kernel(PagedArgs a, const T* __restrict__ Q, int G, const T* __restrict__ bounds, int first, int last,
                                                                   uint32_t* __restrict__ keys) {
  typedef Columns<T> C;
  constexpr int N = C::kCount, kLanes = D / N, kAbreast = 64 / kLanes;
  const int u = blockIdx.y, b = u / (a.L * a.H), in = u - b * a.L * a.H;
  const int lane = threadIdx.x & 63, mine = lane / kLanes, part = lane % kLanes;
  const int blocks = pages_of(a, b, in / a.H);
  double up[N], down[N];
#pragma unroll
  for (int i = 0; i < N; ++i) up[i] = down[i] = 0.0;
  for (int g = 0; g < G; ++g) {
    float x[N];
    C::get(*reinterpret_cast<const u32x4*>(Q + ((int64_t)u * G + g) * D + part * N), x);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      up[i] += x[i] > 0.f ? (double)x[i] : x[i] < 0.f ? 0.0 : (double)x[i];       // (what is not a number is in both)
      down[i] += x[i] < 0.f ? (double)x[i] : x[i] > 0.f ? 0.0 : (double)x[i];
    }
  }
  const int waves = gridDim.x * kScoreWaves, wave = blockIdx.x * kScoreWaves + (threadIdx.x >> 6);
  const int32_t* const table = a.table + b * a.table_b + (int64_t)in * a.max_pages;
  for (int p0 = wave * kAbreast; p0 < blocks; p0 += waves * kAbreast) {
    const int p = p0 + mine;
    const int page = p < blocks ? table[p] : -1;
    const bool there = page >= 0 && page < a.num_pages;
    const T* const from = bounds + (int64_t)(there ? page : 0) * 2 * D + part * N;
    float low[N], high[N];
    C::get(*reinterpret_cast<const u32x4*>(from), low);
    C::get(*reinterpret_cast<const u32x4*>(from + D), high);
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fma((double)low[i], down[i], fma((double)high[i], up[i], s));
#pragma unroll
    for (int d = kLanes / 2; d; d >>= 1) s += __shfl_xor(s, d, 64);
    if (part == 0 && p < blocks)
      keys[(int64_t)u * a.max_pages + p] = !there ? 0u : (p < first || p >= blocks - last) ? 0xFFFFFFFFu : key_of((float)s);
  }
}

// The `count` largest keys of a unit, of equal ones the first, in the order of the table.  A workgroup per unit: the smallest key that is
// taken is found bit by bit.
__global__ __launch_bounds__(kChooseThreads) void choose_kernel(PagedArgs a, const uint32_t* __restrict__ keys, int count, int32_t* __restrict__ chosen) {
  constexpr int kWaves = kChooseThreads / 64;
  __shared__ int counts[2][kWaves], above_of[kWaves], equal_of[kWaves];
  const int u = blockIdx.x, b = u / (a.L * a.H), in = u - b * a.L * a.H, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int blocks = pages_of(a, b, in / a.H);
  const uint32_t* const key = keys + (int64_t)u * a.max_pages;
  int turn = 0;
  auto at_least = [&](uint32_t least) {
    int n = 0;
    for (int p = tid; p < blocks; p += kChooseThreads) n += key[p] >= least ? 1 : 0;
#pragma unroll
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d, 64);
    if (lane == 0) counts[turn][wave] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) n += counts[turn][w];
    turn ^= 1;
    return n;
  };
  const int want = min(count, at_least(1u));
  uint32_t least = 1u;
  int with_least = 0;
  if (want > 0) {
    uint32_t found = 0;
    for (int bit = 31; bit >= 0; --bit)
      if (at_least(found | 1u << bit) >= want) found |= 1u << bit;
    least = found;
    with_least = want - (found == 0xFFFFFFFFu ? 0 : at_least(found + 1u));       // of those that are equal to it
  }
  int32_t* const out = chosen + (int64_t)u * count;
  int taken = 0, equal = 0;
  for (int p0 = 0; p0 < blocks && want > 0; p0 += kChooseThreads) {
    const int p = p0 + tid;
    const uint32_t k = p < blocks ? key[p] : 0u;
    const uint64_t eq = __ballot(k == least && p < blocks), gt = __ballot(k > least);
    if (lane == 0) { equal_of[wave] = __popcll(eq); above_of[wave] = __popcll(gt); }
    __syncthreads();
    const uint64_t before = (1ull << lane) - 1ull;
    int eq_before = equal + __popcll(eq & before), gt_before = taken - min(equal, with_least) + __popcll(gt & before);
    int eq_all = 0, gt_all = 0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) { eq_before += equal_of[w]; gt_before += above_of[w]; }
      eq_all += equal_of[w];
      gt_all += above_of[w];
    }
    const bool mine = k > least || (k == least && p < blocks && eq_before < with_least);
    if (mine) out[gt_before + min(eq_before, with_least)] = p;
    taken += gt_all + min(equal + eq_all, with_least) - min(equal, with_least);
    equal += eq_all;
    __syncthreads();
  }
  for (int i = want + tid; i < count; i += kChooseThreads) out[i] = -1;
}

}  // namespace

hipError_t page_bounds_launch(const fc_paged_kv& kv, void* bounds, hipStream_t s) {
  const PagedArgs a = paged_args(kv);
  const int64_t items = (int64_t)a.B * a.L * a.H * a.max_pages;
  const unsigned groups = (unsigned)std::min<int64_t>(1024, (items + kBoundWaves - 1) / kBoundWaves);
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
  {
    ProfileScope ps("page_score_kernel", s);
    const int abreast = 64 / (kv.head_dim / (kv.dtype == FC_BF16 ? 8 : 4)) * kScoreWaves;
    const unsigned parts = (unsigned)std::max(1, std::min((a.max_pages + abreast - 1) / abreast, (2048 + units - 1) / units));
    auto launch = [&](auto kern, auto type) {
      typedef decltype(type) T;
      hipLaunchKernelGGL(kern, dim3(parts, units), dim3(kScoreThreads), 0, s, a, static_cast<const T*>(Q), group, static_cast<const T*>(bounds), first, last, keys);
    };
    if (kv.dtype == FC_BF16) kv.head_dim == 128 ? launch(page_score_kernel<uint16_t, 128>, uint16_t{}) : launch(page_score_kernel<uint16_t, 64>, uint16_t{});
    else kv.head_dim == 128 ? launch(page_score_kernel<float, 128>, float{}) : launch(page_score_kernel<float, 64>, float{});
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ProfileScope ps("choose_kernel", s);
  hipLaunchKernelGGL(choose_kernel, dim3(units), dim3(kChooseThreads), 0, s, a, static_cast<const uint32_t*>(keys), count, chosen);
  return hipGetLastError();
}

}  // namespace fc
