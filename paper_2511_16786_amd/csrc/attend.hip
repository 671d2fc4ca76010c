// Decode-step attention over a paged cache where sequences share rows, or read chosen pages alone:  out = softmax(q K^T * scale) V, one new token a
// sequence, query head g reads KV head g / G.
//
//   shared   the rows of the prompt that a run of sequences has in common, then the rows of each one's own.  A prompt's rows are read for
//            all of these sequences together: their m * G queries are the rows of one product.
//   chosen   the rows of the pages that a list names for each unit (sequence, layer, KV head).
//
// Both products are on the matrix cores.  bf16 rows: 16x16x32, products exact in fp32; probabilities are two bf16 terms, each rounded to nearest
// (17 bits, off by 7e-7 in the mean; one term would be off by 1e-3).  fp32 rows: 16x16x4 in fp32.  Sums and softmax are in fp32.
// With c16 = lane % 16 and g4 = lane / 16, and 16 rows of K and V a tile:
//   scores:  A = K rows (row c16), B = queries (query c16), the same columns of both for each g4; a lane has the scores of rows 4 g4 + i, query c16
//   output:  A = probabilities (query c16, rows 4 g4 + i, as the scores come out), B = V (the same rows, a column for each c16 and output tile)
#include <algorithm>
#include <type_traits>

#include "fc_common.h"
#include "paged.h"

namespace fc {

namespace {

constexpr int kAttThreads = 256, kAttWaves = kAttThreads / 64;
constexpr int kTileQueries = 16;       // of a workgroup
constexpr int kLeastSteps = 4;         // of a piece
constexpr int kGroups = 1024;          // pieces that a launch over shared rows aims at

typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kNoRow = 0xFFFFFFFFu;

// A piece of work's result for `rows` queries: largest scores (in log2) [rows], sums [rows], weighted V [rows][d].
__host__ __device__ inline int64_t record_floats(int rows, int d) { return ((int64_t)rows * (d + 2) + 3) / 4 * 4; }

__device__ __forceinline__ bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8, (u32x4{a, b, c, d}));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {        // to nearest
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{a, b}), bf16x2));
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <typename V> __device__ __forceinline__ V load_past(const void* p) { return __builtin_nontemporal_load(static_cast<const V*>(p)); }

// The 16 queries of a tile as the score product takes them, and 16 or 32 rows (a step) of K and V as both products take them.
template <typename T, int D> struct Form;
template <int D> struct Form<uint16_t, D> {
  static constexpr int kTiles = 2, kRows = 32, KW = D / 8, VT = D / 16, VW = VT / 2;
  struct Queries { uint32_t w[KW]; };
  struct Rows { uint32_t k[2][KW], v[2][4][VW]; };
  static __device__ __forceinline__ int column(int c16, int t) { return VT * c16 + t; }   // of output tile t
  static __device__ __forceinline__ void queries(const uint16_t* q, bool has, int g4, Queries& o) {
#pragma unroll
    for (int i = 0; i < KW; ++i) o.w[i] = 0u;
    if (has)
#pragma unroll
      for (int i = 0; i < KW / 4; ++i) {
        const u32x4 u = *reinterpret_cast<const u32x4*>(q + 8 * g4 + 32 * i);
        o.w[4 * i] = u.x; o.w[4 * i + 1] = u.y; o.w[4 * i + 2] = u.z; o.w[4 * i + 3] = u.w;
      }
  }
  static __device__ __forceinline__ void load_k(const uint16_t* base, int64_t row, int g4, int tile, Rows& x) {
    const uint16_t* const p = base + row * D + 8 * g4;
#pragma unroll
    for (int i = 0; i < KW / 4; ++i) {
      const u32x4 u = load_past<u32x4>(p + 32 * i);
      x.k[tile][4 * i] = u.x; x.k[tile][4 * i + 1] = u.y; x.k[tile][4 * i + 2] = u.z; x.k[tile][4 * i + 3] = u.w;
    }
  }
  static __device__ __forceinline__ void load_v(const uint16_t* base, int64_t row, int c16, int tile, int i, Rows& x) {
    const uint16_t* const p = base + row * D + VT * c16;
    if constexpr (VW == 4) {
      const u32x4 u = load_past<u32x4>(p);
      x.v[tile][i][0] = u.x; x.v[tile][i][1] = u.y; x.v[tile][i][2] = u.z; x.v[tile][i][3] = u.w;
    } else {
      const u32x2 u = load_past<u32x2>(p);
      x.v[tile][i][0] = u.x; x.v[tile][i][1] = u.y;
    }
  }
  static __device__ __forceinline__ float4v scores(const Queries& q, const Rows& x, int tile) {
    float4v acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KW / 4; ++s)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x.k[tile][4 * s], x.k[tile][4 * s + 1], x.k[tile][4 * s + 2], x.k[tile][4 * s + 3]),
                                                    as_bf16x8(q.w[4 * s], q.w[4 * s + 1], q.w[4 * s + 2], q.w[4 * s + 3]), acc, 0, 0, 0);
    return acc;
  }
  static __device__ __forceinline__ void add(const float (&p)[kTiles][4], const Rows& x, float4v (&out)[VT]) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = p[j / 2][j % 2 * 2], b = p[j / 2][j % 2 * 2 + 1];
      hi[j] = pack_bf16(a, b);
      lo[j] = pack_bf16(a - __uint_as_float(hi[j] << 16), b - __uint_as_float(hi[j] & 0xFFFF0000u));
    }
    const bf16x8 phi = as_bf16x8(hi[0], hi[1], hi[2], hi[3]), plo = as_bf16x8(lo[0], lo[1], lo[2], lo[3]);
#pragma unroll
    for (int t = 0; t < VT; ++t) {
      const uint32_t sel = (t & 1) ? 0x07060302u : 0x05040100u;
      const int w = t >> 1;
      auto two = [&](int tile, int i) { return __builtin_amdgcn_perm(x.v[tile][i + 1][w], x.v[tile][i][w], sel); };
      const bf16x8 v = as_bf16x8(two(0, 0), two(0, 2), two(1, 0), two(1, 2));
      out[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(phi, v, out[t], 0, 0, 0);
      out[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(plo, v, out[t], 0, 0, 0);
    }
  }
};
template <int D> struct Form<float, D> {
  static constexpr int kTiles = 1, kRows = 16, KW = D / 4, VT = D / 16;
  struct Queries { float w[KW]; };
  struct Rows { float k[1][KW], v[1][4][VT]; };
  // (a load takes 16 bytes a lane: four neighbouring columns of each half of a row)
  static __device__ __forceinline__ int column(int c16, int t) { return t / 4 * 64 + 4 * c16 + t % 4; }
  static __device__ __forceinline__ void queries(const float* q, bool has, int g4, Queries& o) {
#pragma unroll
    for (int i = 0; i < KW; ++i) o.w[i] = 0.f;
    if (has)
#pragma unroll
      for (int j = 0; j < KW / 4; ++j) {
        const float4v u = *reinterpret_cast<const float4v*>(q + 16 * j + 4 * g4);
        o.w[4 * j] = u.x; o.w[4 * j + 1] = u.y; o.w[4 * j + 2] = u.z; o.w[4 * j + 3] = u.w;
      }
  }
  static __device__ __forceinline__ void load_k(const float* base, int64_t row, int g4, int tile, Rows& x) {
    const float* const p = base + row * D + 4 * g4;
#pragma unroll
    for (int j = 0; j < KW / 4; ++j) {
      const float4v u = load_past<float4v>(p + 16 * j);
      x.k[tile][4 * j] = u.x; x.k[tile][4 * j + 1] = u.y; x.k[tile][4 * j + 2] = u.z; x.k[tile][4 * j + 3] = u.w;
    }
  }
  static __device__ __forceinline__ void load_v(const float* base, int64_t row, int c16, int tile, int i, Rows& x) {
    const float* const p = base + row * D + 4 * c16;
#pragma unroll
    for (int j = 0; j < VT / 4; ++j) {
      const float4v u = load_past<float4v>(p + 64 * j);
      x.v[tile][i][4 * j] = u.x; x.v[tile][i][4 * j + 1] = u.y; x.v[tile][i][4 * j + 2] = u.z; x.v[tile][i][4 * j + 3] = u.w;
    }
  }
  static __device__ __forceinline__ float4v scores(const Queries& q, const Rows& x, int tile) {
    float4v acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KW; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.k[tile][i], q.w[i], acc, 0, 0, 0);
    return acc;
  }
  static __device__ __forceinline__ void add(const float (&p)[kTiles][4], const Rows& x, float4v (&out)[VT]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < VT; ++t) out[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[0][i], x.v[0][i][t], out[t], 0, 0, 0);
  }
};

// A wave's online softmax: running maximum (in log2 units, common to the four lanes of a query), this lane's sum, weighted V of queries 4 g4 + i.
template <typename T, int D> struct State {
  typedef Form<T, D> F;
  float m = -INFINITY, sum = 0.f;
  float4v out[F::VT];
  __device__ __forceinline__ State() {
#pragma unroll
    for (int t = 0; t < F::VT; ++t) out[t] = float4v{0.f, 0.f, 0.f, 0.f};
  }
  // `where`: lane r has the cache row of row r of the step, or kNoRow
  __device__ __forceinline__ void step(const typename F::Queries& q, const typename F::Rows& x, uint32_t where, float scale_log2e, int g4) {
    float p[F::kTiles][4];
    float mx = -INFINITY;
#pragma unroll
    for (int tt = 0; tt < F::kTiles; ++tt) {
      const float4v acc = F::scores(q, x, tt);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool valid = (uint32_t)__shfl((int)where, 16 * tt + 4 * g4 + i, 64) != kNoRow;
        p[tt][i] = valid ? acc[i] * scale_log2e : -INFINITY;
        mx = fmaxf(mx, p[tt][i]);
      }
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m, mx);
    const bool none = m_new == -INFINITY;                  // (scores of a query with infinities, too)
    const float alpha = none ? 1.f : exp2f(m - m_new);
    m = m_new;
    float more = 0.f;
#pragma unroll
    for (int tt = 0; tt < F::kTiles; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[tt][i] = none ? 0.f : exp2f(p[tt][i] - m_new);
        more += p[tt][i];
      }
    sum = fmaf(sum, alpha, more);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = __shfl(alpha, 4 * g4 + i, 64);
#pragma unroll
      for (int t = 0; t < F::VT; ++t) out[t][i] *= a;
    }
    F::add(p, x, out);
  }
};

// Requests a step's rows.  Rows that are not there are read as the step's first one that is: what a cache holds in other places may be anything.
// False, and nothing requested, if there is none.
template <typename T, int D>
__device__ __forceinline__ bool request(const T* K, const T* V, uint32_t where, int lane, int c16, int g4, typename Form<T, D>::Rows& x) {
  typedef Form<T, D> F;
  const uint64_t there = __ballot(where != kNoRow);
  if (there == 0) return false;
  const uint32_t stand_in = (uint32_t)__builtin_amdgcn_readlane((int)where, __builtin_ctzll(there));
  const uint32_t row = where == kNoRow ? stand_in : where;
#pragma unroll
  for (int tt = 0; tt < F::kTiles; ++tt) {
    F::load_k(K, (uint32_t)__shfl((int)row, 16 * tt + c16, 64), g4, tt, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) F::load_v(V, (uint32_t)__shfl((int)row, 16 * tt + 4 * g4 + i, 64), c16, tt, i, x);
  }
  return true;
}

// Steps first, first + stride, ... below end of what `lookup` names (the cache row of row lane % kRows of a step), two under way.
template <typename T, int D, typename Lookup>
__device__ __forceinline__ void walk(State<T, D>& state, const typename Form<T, D>::Queries& q, const T* K, const T* V, int first, int end, int stride,
                                     float scale_log2e, int lane, const Lookup& lookup) {
  const int c16 = lane & 15, g4 = lane >> 4;
  typename Form<T, D>::Rows xa, xb;
  uint32_t wa = kNoRow, wb = kNoRow, next = kNoRow;
  bool has_a = false, has_b = false;
  if (first < end) {
    wa = lookup(first);
    if (first + stride < end) wb = lookup(first + stride);
    has_a = request<T, D>(K, V, wa, lane, c16, g4, xa);
    has_b = first + stride < end && request<T, D>(K, V, wb, lane, c16, g4, xb);
    if (first + 2 * stride < end) next = lookup(first + 2 * stride);
  }
  auto turn = [&](int st, typename Form<T, D>::Rows& x, uint32_t& w, bool& has) {
    if (has) state.step(q, x, w, scale_log2e, g4);
    has = false;
    if (st + 2 * stride < end) {
      w = next;
      has = request<T, D>(K, V, w, lane, c16, g4, x);
      if (st + 3 * stride < end) next = lookup(st + 3 * stride);
    }
  };
  for (int st = first; st < end; st += 2 * stride) {
    turn(st, xa, wa, has_a);
    if (st + stride < end) turn(st + stride, xb, wb, has_b);
  }
}

// The waves' states as one, through LDS in a fixed order: into a record of `rows` queries, or (whole) the result itself.
template <typename T, int D>
__device__ __forceinline__ void merge_waves(State<T, D>& state, int rows, float* record, float* whole) {
  typedef Form<T, D> F;
  __shared__ float sm_m[kAttWaves][16], sm_l[kAttWaves][16];
  __shared__ float sm_o[kAttWaves][16][D];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c16 = lane & 15, g4 = lane >> 4;
  state.sum += __shfl_xor(state.sum, 16, 64);
  state.sum += __shfl_xor(state.sum, 32, 64);
  if (g4 == 0) { sm_m[wave][c16] = state.m; sm_l[wave][c16] = state.sum; }
#pragma unroll
  for (int t = 0; t < F::VT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) sm_o[wave][4 * g4 + i][F::column(c16, t)] = state.out[t][i];
  __syncthreads();
  for (int item = tid; item < rows * D; item += kAttThreads) {
    const int g = item / D, dim = item % D;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w) M = fmaxf(M, sm_m[w][g]);
    float acc = 0.f, lt = 0.f;
    if (M > -INFINITY)
#pragma unroll
      for (int w = 0; w < kAttWaves; ++w) {
        const float f = exp2f(sm_m[w][g] - M);
        acc = fmaf(sm_o[w][g][dim], f, acc);
        lt = fmaf(sm_l[w][g], f, lt);
      }
    if (whole) {
      whole[(int64_t)g * D + dim] = lt > 0.f ? acc / lt : 0.f;
    } else {
      record[2 * rows + item] = acc;
      if (dim == 0) { record[g] = M; record[rows + g] = lt; }
    }
  }
}

// ---- pages that a list names -------------------------------------------------------------------
// grid = (parts, units): the waves of a unit's parts take its steps in turn, so that a list that ends early leaves none idle before the others.
template <typename T, int D>
__global__ __launch_bounds__(kAttThreads, 2) void attend_chosen_kernel(PagedArgs a, const T* __restrict__ Q, int G, const int32_t* __restrict__ chosen, int count,
                                                                       float scale_log2e, float* __restrict__ records, float* __restrict__ whole) {
  typedef Form<T, D> F;
  const int u = blockIdx.y, b = u / (a.L * a.H), in = u - b * a.L * a.H;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g4 = lane >> 4;
  const int rows = rows_of(a, b, in / a.H);
  const int32_t* const table = a.table + b * a.table_b + (int64_t)in * a.max_pages;
  const int32_t* const list = chosen + (int64_t)u * count;
  typename F::Queries q;
  F::queries(Q + ((int64_t)u * G + min(c16, G - 1)) * D, c16 < G, g4, q);
  auto lookup = [&](int st) -> uint32_t {
    const int at = st * F::kRows + (lane & (F::kRows - 1)), entry = at / a.page_size, off = at - entry * a.page_size;
    if (entry >= count) return kNoRow;
    const int p = list[entry];
    if (p < 0 || p >= a.max_pages || (int64_t)p * a.page_size + off >= rows) return kNoRow;
    const int page = table[p];
    return page >= 0 && page < a.num_pages ? (uint32_t)page * (uint32_t)a.page_size + (uint32_t)off : kNoRow;
  };
  const int waves = gridDim.x * kAttWaves, wave = blockIdx.x * kAttWaves + uniform(threadIdx.x >> 6);
  const int steps = (count * a.page_size + F::kRows - 1) / F::kRows;
  State<T, D> state;
  walk<T, D>(state, q, static_cast<const T*>(a.K), static_cast<const T*>(a.V), wave, steps, waves, scale_log2e, lane, lookup);
  merge_waves<T, D>(state, G, records + ((int64_t)u * gridDim.x + blockIdx.x) * record_floats(G, D), whole ? whole + (int64_t)u * G * D : nullptr);
}

// grid = (G, units), a thread per column
__global__ void chosen_merge_kernel(const float* __restrict__ records, int parts, int G, int D, float* __restrict__ out) {
  const int g = blockIdx.x, u = blockIdx.y, dim = threadIdx.x;
  const int64_t size = record_floats(G, D);
  const float* const base = records + (int64_t)u * parts * size;
  float M = -INFINITY, acc = 0.f, lt = 0.f;
  for (int k = 0; k < parts; ++k) M = fmaxf(M, base[k * size + g]);
  if (M > -INFINITY)
    for (int k = 0; k < parts; ++k) {
      const float* const rec = base + k * size;
      const float w = exp2f(rec[g] - M);
      acc = fmaf(rec[2 * G + g * D + dim], w, acc);
      lt = fmaf(rec[G + g], w, lt);
    }
  out[((int64_t)u * G + g) * D + dim] = lt > 0.f ? acc / lt : 0.f;
}

// ---- rows of a shared prompt, and of each sequence ---------------------------------------------
struct SharedArgs {
  PagedArgs common, own;         // of P prompts and of B sequences
  const int32_t* starts;         // [P + 1]
  int G, groups;
  int64_t most_common, most_own; // records of either kind that the workspace has
  float scale_log2e;
  float* common_records;
  float* own_records;
  int2* span;                    // of each prompt's layers, then of each sequence's: first record, pieces of a unit
  float* out;
};

// Sequences of prompt p: [first, first + n)
struct Run { int first, n; };
__device__ __forceinline__ Run run_of(const SharedArgs& a, int p) {
  const int s0 = min(max(a.starts[p], 0), a.own.B), s1 = min(max(a.starts[p + 1], 0), a.own.B);
  return {s0, max(0, s1 - s0)};
}
__device__ __forceinline__ int tiles_of(const SharedArgs& a, int n) { return (n * a.G + kTileQueries - 1) / kTileQueries; }

// Entry e: a layer of a prompt, or, behind all of these, of a sequence.  Its rows, and how many units and query tiles have them to read.
struct Entry { int rows, times; };
__device__ __forceinline__ Entry entry_at(const SharedArgs& a, int e) {
  const int L = a.own.L, shared = a.common.B * L;
  if (e < shared) {
    const int p = e / L;
    return {rows_of(a.common, p, e - p * L), a.own.H * tiles_of(a, run_of(a, p).n)};
  }
  const int b = (e - shared) / L;
  return {rows_of(a.own, b, e - shared - b * L), a.own.H};
}
template <int ROWS> __device__ __forceinline__ int steps_in(int rows) { return (rows + ROWS - 1) / ROWS; }

__device__ __forceinline__ int64_t wave_sum(int64_t v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}
__device__ __forceinline__ int64_t wave_scan(int64_t v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up(v, d, 64);
    if (lane >= d) v += o;
  }
  return v;
}

template <typename T, int D>
__global__ __launch_bounds__(kAttThreads, 2) void attend_shared_kernel(SharedArgs a, const T* __restrict__ Q) {
  typedef Form<T, D> F;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g4 = lane >> 4, wave = uniform(threadIdx.x >> 6);
  const int L = a.own.L, H = a.own.H, G = a.G, shared = a.common.B * L, entries = shared + a.own.B * L;
  // every wave finds out which piece is its workgroup's
  int64_t total = 0;
  for (int e0 = 0; e0 < entries; e0 += 64) {
    if (e0 + lane < entries) {
      const Entry x = entry_at(a, e0 + lane);
      total += (int64_t)steps_in<F::kRows>(x.rows) * x.times;
    }
  }
  total = wave_sum(total);
  const int each = (int)max((int64_t)kLeastSteps, (total + a.groups - 1) / a.groups);
  const int64_t w = blockIdx.x;
  int64_t before = 0, before_own = 0;
  int entry = -1, rows = 0, pieces = 0;
  int64_t place = 0;
  for (int e0 = 0; e0 < entries && entry < 0; e0 += 64) {
    Entry x{0, 0};
    if (e0 + lane < entries) x = entry_at(a, e0 + lane);
    const int mine = (steps_in<F::kRows>(x.rows) + each - 1) / each;
    const int64_t upto = before + wave_scan((int64_t)mine * x.times, lane);
    // (records of sequences are counted from the first of them on)
    const uint64_t first_own = __ballot(e0 + lane >= shared);
    if (e0 < shared && first_own) before_own = __shfl(upto - (int64_t)mine * x.times, __builtin_ctzll(first_own), 64);
    if (e0 == shared) before_own = before;
    const uint64_t past = __ballot(upto > w);
    if (past) {
      const int from = __builtin_ctzll(past);
      entry = e0 + from;
      rows = __builtin_amdgcn_readlane(x.rows, from);
      pieces = __builtin_amdgcn_readlane(mine, from);
      place = w - __shfl(upto - (int64_t)mine * x.times, from, 64);
    }
    before = __shfl(upto, 63, 64);
  }
  if (entry < 0) return;
  const bool is_own = entry >= shared;
  const int64_t index = is_own ? w - before_own : w;
  if (index >= (is_own ? a.most_own : a.most_common)) return;
  if (place == 0 && threadIdx.x == 0) a.span[entry] = int2{(int)index, pieces};
  const int unit = uniform((int)(place / pieces)), piece = uniform((int)(place - (int64_t)unit * pieces));
  // the unit's head, and the tile's queries
  const int seq = is_own ? (entry - shared) / L : entry / L, l = (is_own ? entry - shared : entry) - seq * L;
  int h = unit, first = seq, queries = G, tile = 0;
  if (!is_own) {
    const Run run = run_of(a, seq);
    const int tiles = tiles_of(a, run.n);
    h = unit / tiles;
    tile = unit - h * tiles;
    first = run.first;
    queries = min(kTileQueries, run.n * G - tile * kTileQueries);
  }
  const int r = tile * kTileQueries + c16, b = first + r / G, g = r % G;
  typename F::Queries q;
  F::queries(Q + (((int64_t)(c16 < queries ? b : first) * L + l) * H * G + (int64_t)h * G + (c16 < queries ? g : 0)) * D, c16 < queries, g4, q);
  const PagedArgs& kv = is_own ? a.own : a.common;
  const int32_t* const table = kv.table + seq * kv.table_b + ((int64_t)l * H + h) * kv.max_pages;
  const int page_size = kv.page_size;
  const int64_t num_pages = kv.num_pages;
  auto lookup = [&](int st) -> uint32_t {
    const int row = st * F::kRows + (lane & (F::kRows - 1));
    if (row >= rows) return kNoRow;
    const int p = row / page_size, page = table[p];
    return page >= 0 && page < num_pages ? (uint32_t)page * (uint32_t)page_size + (uint32_t)(row - p * page_size) : kNoRow;
  };
  const int steps = steps_in<F::kRows>(rows), share = pieces * kAttWaves, id = piece * kAttWaves + wave;
  State<T, D> state;
  walk<T, D>(state, q, static_cast<const T*>(kv.K), static_cast<const T*>(kv.V), (int)((int64_t)steps * id / share), (int)((int64_t)steps * (id + 1) / share),
             1, a.scale_log2e, lane, lookup);
  merge_waves<T, D>(state, queries, is_own ? a.own_records + index * record_floats(G, D) : a.common_records + index * record_floats(kTileQueries, D), nullptr);
}

// grid = (G, B * L * H), a thread per column: the records of the prompt's pieces and of the sequence's own, in order
template <int D>
__global__ void shared_merge_kernel(SharedArgs a) {
  const int L = a.own.L, H = a.own.H, G = a.G, g = blockIdx.x, u = blockIdx.y, dim = threadIdx.x, lane = dim & 63;
  const int b = u / (L * H), l = u / H % L, h = u % H, P = a.common.B;
  int p = -1;
  for (int p0 = 0; p0 < P && p < 0; p0 += 64) {
    bool mine = false;
    if (p0 + lane < P) {
      const Run run = run_of(a, p0 + lane);
      mine = b >= run.first && b < run.first + run.n;
    }
    const uint64_t found = __ballot(mine);
    if (found) p = p0 + __builtin_ctzll(found);
  }
  const float* from[2] = {nullptr, nullptr};
  int count[2] = {0, 0}, queries[2] = {G, G}, row[2] = {g, g};
  int64_t size[2] = {record_floats(kTileQueries, D), record_floats(G, D)};
  if (p >= 0 && rows_of(a.common, p, l) > 0) {
    const Run run = run_of(a, p);
    const int tiles = tiles_of(a, run.n), at = (b - run.first) * G + g, tile = at / kTileQueries;
    const int2 span = a.span[p * L + l];
    const int64_t index = span.x + (int64_t)(h * tiles + tile) * span.y;
    if (span.x >= 0 && span.y > 0 && index + span.y <= a.most_common) {
      from[0] = a.common_records + index * size[0];
      count[0] = span.y;
      queries[0] = min(kTileQueries, run.n * G - tile * kTileQueries);
      row[0] = at - tile * kTileQueries;
    }
  }
  if (rows_of(a.own, b, l) > 0) {
    const int2 span = a.span[(P + b) * L + l];
    const int64_t index = span.x + (int64_t)h * span.y;
    if (span.x >= 0 && span.y > 0 && index + span.y <= a.most_own) {
      from[1] = a.own_records + index * size[1];
      count[1] = span.y;
    }
  }
  float M = -INFINITY, acc = 0.f, lt = 0.f;
  for (int k = 0; k < 2; ++k)
    for (int i = 0; i < count[k]; ++i) M = fmaxf(M, from[k][i * size[k] + row[k]]);
  if (M > -INFINITY)
    for (int k = 0; k < 2; ++k)
      for (int i = 0; i < count[k]; ++i) {
        const float* const rec = from[k] + i * size[k];
        const float w = exp2f(rec[row[k]] - M);
        acc = fmaf(rec[2 * queries[k] + row[k] * D + dim], w, acc);
        lt = fmaf(rec[queries[k] + row[k]], w, lt);
      }
  a.out[((int64_t)u * G + g) * D + dim] = lt > 0.f ? acc / lt : 0.f;
}

// Query tiles of all prompts at most
int64_t most_tiles(int P, int B, int G) {
  const int runs = std::min(P, B);
  return runs + ((int64_t)B * G - runs) / kTileQueries;
}

struct SharedSizes {
  int64_t common, own, span, total;    // records, entries, bytes
};
SharedSizes shared_sizes(int P, int B, int L, int H, int G, int d) {
  SharedSizes z;
  z.common = kGroups + (int64_t)L * H * most_tiles(P, B, G);
  z.own = kGroups + (int64_t)L * H * B;
  z.span = (int64_t)(P + B) * L;
  z.total = (z.common * record_floats(kTileQueries, d) + z.own * record_floats(G, d)) * (int64_t)sizeof(float) + z.span * (int64_t)sizeof(int2);
  return z;
}

// Parts of a unit: enough waves for the chip, two steps each at least.
int chosen_parts(int units, int count, int page_size, int step_rows) {
  const int64_t steps = ((int64_t)count * page_size + step_rows - 1) / step_rows;
  return (int)std::max<int64_t>(1, std::min<int64_t>((1024 + units - 1) / units, steps / (2 * kAttWaves)));
}

}  // namespace

bool attend_supported(int group, int d) { return group >= 1 && group <= 16 && (d == 64 || d == 128); }

size_t attend_chosen_workspace_bytes(int units, int group, int d, int dtype, int page_size, int count) {
  const int parts = chosen_parts(units, count, page_size, dtype == FC_BF16 ? 32 : 16);
  return parts == 1 ? 0 : (size_t)units * parts * record_floats(group, d) * sizeof(float);
}

hipError_t attend_chosen_launch(const void* Q, int group, const fc_paged_kv& kv, const int32_t* chosen, int count, float scale, float* out, void* ws, hipStream_t s) {
  const PagedArgs a = paged_args(kv);
  const int units = a.B * a.L * a.H, d = kv.head_dim, parts = chosen_parts(units, count, a.page_size, kv.dtype == FC_BF16 ? 32 : 16);
  float* const records = static_cast<float*>(ws);
  {
    ProfileScope ps("attend_chosen_kernel", s);
    auto launch = [&](auto kern, auto type) {
      typedef decltype(type) T;
      hipLaunchKernelGGL(kern, dim3(parts, units), dim3(kAttThreads), 0, s, a, static_cast<const T*>(Q), group, chosen, count, scale * 1.4426950408889634f, records,
                         parts == 1 ? out : nullptr);
    };
    if (kv.dtype == FC_BF16) d == 128 ? launch(attend_chosen_kernel<uint16_t, 128>, uint16_t{}) : launch(attend_chosen_kernel<uint16_t, 64>, uint16_t{});
    else d == 128 ? launch(attend_chosen_kernel<float, 128>, float{}) : launch(attend_chosen_kernel<float, 64>, float{});
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  ProfileScope ps("chosen_merge_kernel", s);
  hipLaunchKernelGGL(chosen_merge_kernel, dim3(group, units), dim3(d), 0, s, records, parts, group, d, out);
  return hipGetLastError();
}

size_t attend_shared_workspace_bytes(int P, int B, int L, int H, int group, int d, int dtype) {
  (void)dtype;
  return (size_t)shared_sizes(P, B, L, H, group, d).total; }

hipError_t attend_shared_launch(const void* Q, int group, const fc_paged_kv& common, const int32_t* starts, const fc_paged_kv& own, float scale, float* out, void* ws,
                                hipStream_t s) {
  const int P = common.batch, B = own.batch, L = own.layers, H = own.kv_heads, d = own.head_dim;
  const SharedSizes z = shared_sizes(P, B, L, H, group, d);
  float* const records = static_cast<float*>(ws);
  float* const own_records = records + z.common * record_floats(kTileQueries, d);
  SharedArgs a{paged_args(common), paged_args(own), starts, group, kGroups, z.common, z.own, scale * 1.4426950408889634f, records, own_records,
               reinterpret_cast<int2*>(own_records + z.own * record_floats(group, d)), out};
  {
    ProfileScope ps("attend_shared_kernel", s);
    const int64_t groups = kGroups + (int64_t)L * H * (most_tiles(P, B, group) + B);
    auto launch = [&](auto kern, auto type) {
      typedef decltype(type) T;
      hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kAttThreads), 0, s, a, static_cast<const T*>(Q));
    };
    if (own.dtype == FC_BF16) d == 128 ? launch(attend_shared_kernel<uint16_t, 128>, uint16_t{}) : launch(attend_shared_kernel<uint16_t, 64>, uint16_t{});
    else d == 128 ? launch(attend_shared_kernel<float, 128>, float{}) : launch(attend_shared_kernel<float, 64>, float{});
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ProfileScope ps("shared_merge_kernel", s);
  auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(group, B * L * H), dim3(d), 0, s, a); };
  d == 128 ? launch(shared_merge_kernel<128>) : launch(shared_merge_kernel<64>);
  return hipGetLastError();
}

}  // namespace fc
