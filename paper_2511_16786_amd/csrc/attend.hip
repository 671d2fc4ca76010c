// Decode-step attention over a paged cache where sequences share rows, or read chosen pages alone:  out = softmax(q K^T * scale) V, one new token a
// sequence, query head g reads KV head g / G.
//
//   shared   the rows of the prompt that a run of sequences has in common, then the rows of each one's own.  A prompt's rows are read for
//            all of these sequences together: their m * G queries are the rows of one product.
//   chosen   the rows of the pages that a list names for each unit (sequence, layer, KV head).
//
// Both products are on the matrix cores.  bf16 rows: 16x16x32, products exact in fp32, probabilities as three bf16 terms that are exact together (24 bits;
// two are off by up to 2^-17).  fp32 rows: 16x16x4 in fp32.  Sums and softmax are in fp32.
// With c16 = lane % 16 and g4 = lane / 16, and 16 rows of K and V a tile:
//   scores:  A = K rows (row c16), B = queries (query c16), the same columns of both for each g4; a lane has the scores of rows 4 g4 + i, query c16
//   output:  A = probabilities (query c16, rows 4 g4 + i, as the scores come out), B = V (the same rows, a column for each c16 and output tile)
//
// Where 16 queries or fewer read the same rows, each of a workgroup's waves has rows of its own, straight into registers, and the waves' results are
// merged.  Bound by memory: 64 pages of 64 bf16 rows of 112 units (0.24 GB) 43 us, and as long without the arithmetic; some 8 us of it are the chain of
// list, table and first rows and the end, the rest is read at 6.7 TB/s.
// Where more do, the workgroup has up to 128 queries, two tiles of 16 a wave, and reads the rows once for all of them, through LDS.  16 answers of 7 heads to
// 28 layers of 4 heads, 6554 rows, and 128 rows of their own in the mean (0.50 GB, 43 GFLOP): 137 us (each 16 queries reading the rows for themselves 482), in the
// long run, when the clock has risen, 118.
// The prompts' rows by themselves take 76 us without the arithmetic, the arithmetic some 100 without them: matrix instructions keep a SIMD busy for a third
// of the time, others for two fifths, and two waves a SIMD, as many as 256 registers allow, overlap them in part only.  With two terms of probabilities 126.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "fc_common.h"
#include "paged.h"

namespace fc {

namespace {

constexpr int kAttThreads = 256, kAttWaves = kAttThreads / 64;
constexpr int kTileQueries = 128;      // of a workgroup
constexpr int kLeastSteps = 4;         // of a piece
constexpr int kGroups = 512;           // workgroups that are resident together
constexpr int kStepsLooked = 64;       // steps whose rows' places are looked up together
constexpr float kSlack = 16.f;         // how far scores (in log2) may exceed the running reference before it is moved

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
// x less the lower or the upper of two bf16 values: exact where that value is x cut off.  (One operation; the constants are kept from the
// compiler, which would take 0xBF800000 for an inline constant of another value in this instruction.)
__device__ __forceinline__ float less_low(float x, uint32_t two) {
  uint32_t c;
  asm("s_mov_b32 %0, 0xbf80" : "=s"(c));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, c), x, false);
}
__device__ __forceinline__ float less_high(float x, uint32_t two) {
  uint32_t c;
  asm("s_mov_b32 %0, 0xbf800000" : "=s"(c));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, c), x, false);
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// Past the last-level cache: for V's rows, whole lines at a time.  A load of K takes half a line of each of 16 rows, and the other half is to be there for
// the next one (64 pages of 28 layers: both past it 46.9 us, V alone 44.9, neither 50.0; 26 small pages of 8 x 28 39.3 / 36.4 / 42.2).
template <typename V> __device__ __forceinline__ V load_past(const void* p) { return __builtin_nontemporal_load(static_cast<const V*>(p)); }

// The 16 queries of a tile as the score product takes them, and 16 or 32 rows (a step) of K and V as both products take them.
template <typename T, int D> struct Form;
template <int D> struct Form<uint16_t, D> {
  static constexpr int kTiles = 2, kRows = 32, KW = D / 8, VT = D / 16, VW = VT / 2;
  struct Queries { uint32_t w[KW]; };
  struct Keys { uint32_t w[2][KW]; };
  struct Values { uint32_t w[2][4][VW]; };
  struct Weights { uint32_t term[3][4]; };
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
  static __device__ __forceinline__ void load_k(const uint16_t* base, int64_t row, int g4, int tile, Keys& x) {
    const uint16_t* const p = base + row * D + 8 * g4;
#pragma unroll
    for (int i = 0; i < KW / 4; ++i) {
      const u32x4 u = *reinterpret_cast<const u32x4*>(p + 32 * i);
      x.w[tile][4 * i] = u.x; x.w[tile][4 * i + 1] = u.y; x.w[tile][4 * i + 2] = u.z; x.w[tile][4 * i + 3] = u.w;
    }
  }
  static __device__ __forceinline__ void load_v(const uint16_t* base, int64_t row, int c16, int tile, int i, Values& x) {
    const uint16_t* const p = base + row * D + VT * c16;
    if constexpr (VW == 4) {
      const u32x4 u = load_past<u32x4>(p);
      x.w[tile][i][0] = u.x; x.w[tile][i][1] = u.y; x.w[tile][i][2] = u.z; x.w[tile][i][3] = u.w;
    } else {
      const u32x2 u = load_past<u32x2>(p);
      x.w[tile][i][0] = u.x; x.w[tile][i][1] = u.y;
    }
  }
  // (the products of one sum are not next to each other)
  template <int N> static __device__ __forceinline__ void scores(const Queries (&q)[N], const Keys& x, float4v (&acc)[N][kTiles]) {
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j][0] = acc[j][1] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KW / 4; ++s)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int j = 0; j < N; ++j)
          acc[j][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(x.w[tt][4 * s], x.w[tt][4 * s + 1], x.w[tt][4 * s + 2], x.w[tt][4 * s + 3]),
                                                               as_bf16x8(q[j].w[4 * s], q[j].w[4 * s + 1], q[j].w[4 * s + 2], q[j].w[4 * s + 3]), acc[j][tt], 0, 0, 0);
  }
  static __device__ __forceinline__ void weights(const float (&p)[kTiles][4], Weights& w) {
    // each term is what the one before left, cut off to bf16: the third is exact
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float a = p[j / 2][j % 2 * 2], b = p[j / 2][j % 2 * 2 + 1];
#pragma unroll
      for (int n = 0; n < 3; ++n) {
        const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
        w.term[n][j] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
        if (n < 2) {
          a = less_low(a, w.term[n][j]);
          b = less_high(b, w.term[n][j]);
        }
      }
    }
  }
  // V's columns as the product takes them
  struct Operands { bf16x8 v[VT]; };
  static __device__ __forceinline__ void operands(const Values& x, Operands& o) {
#pragma unroll
    for (int t = 0; t < VT; ++t) {
      const uint32_t sel = (t & 1) ? 0x07060302u : 0x05040100u;
      const int w = t >> 1;
      auto two = [&](int tile, int i) { return __builtin_amdgcn_perm(x.w[tile][i + 1][w], x.w[tile][i][w], sel); };
      o.v[t] = as_bf16x8(two(0, 0), two(0, 2), two(1, 0), two(1, 2));
    }
  }
  static __device__ __forceinline__ void add(const Weights& p, const Operands& x, float4v (&out)[VT]) {
#pragma unroll
    for (int n = 0; n < 3; ++n)
#pragma unroll
      for (int t = 0; t < VT; ++t)
        out[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(p.term[n][0], p.term[n][1], p.term[n][2], p.term[n][3]), x.v[t], out[t], 0, 0, 0);
  }
  // ... from LDS, 16 bytes of a row a place: K's places are swapped within a row by its number, or the 16 lanes of a read would meet in the same banks
  static constexpr int kPieces = D / 8;
  static __device__ __forceinline__ int k_place(int row, int piece) { return row * kPieces + (piece ^ (row & (kPieces - 1))); }
  static __device__ __forceinline__ void read(const u32x4* k, int c16, int g4, Keys& x) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < KW / 4; ++i) {
        const u32x4 u = k[k_place(16 * tt + c16, g4 + 4 * i)];
        x.w[tt][4 * i] = u.x; x.w[tt][4 * i + 1] = u.y; x.w[tt][4 * i + 2] = u.z; x.w[tt][4 * i + 3] = u.w;
      }
  }
  static __device__ __forceinline__ void read(const u32x4* v, int c16, int g4, Values& x) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t* const p = reinterpret_cast<const uint32_t*>(v) + (16 * tt + 4 * g4 + i) * (D / 2) + VW * c16;
        if constexpr (VW == 4) {
          const u32x4 u = *reinterpret_cast<const u32x4*>(p);
          x.w[tt][i][0] = u.x; x.w[tt][i][1] = u.y; x.w[tt][i][2] = u.z; x.w[tt][i][3] = u.w;
        } else {
          const u32x2 u = *reinterpret_cast<const u32x2*>(p);
          x.w[tt][i][0] = u.x; x.w[tt][i][1] = u.y;
        }
      }
  }
  static __device__ __forceinline__ void negate(Queries& q) {
#pragma unroll
    for (int i = 0; i < KW; ++i) q.w[i] ^= 0x80008000u;
  }
};
template <int D> struct Form<float, D> {
  static constexpr int kTiles = 1, kRows = 16, KW = D / 4, VT = D / 16;
  struct Queries { float w[KW]; };
  struct Keys { float w[1][KW]; };
  struct Values { float w[1][4][VT]; };
  struct Weights { float p[4]; };
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
  static __device__ __forceinline__ void load_k(const float* base, int64_t row, int g4, int tile, Keys& x) {
    const float* const p = base + row * D + 4 * g4;
#pragma unroll
    for (int j = 0; j < KW / 4; ++j) {
      const float4v u = *reinterpret_cast<const float4v*>(p + 16 * j);
      x.w[tile][4 * j] = u.x; x.w[tile][4 * j + 1] = u.y; x.w[tile][4 * j + 2] = u.z; x.w[tile][4 * j + 3] = u.w;
    }
  }
  static __device__ __forceinline__ void load_v(const float* base, int64_t row, int c16, int tile, int i, Values& x) {
    const float* const p = base + row * D + 4 * c16;
#pragma unroll
    for (int j = 0; j < VT / 4; ++j) {
      const float4v u = load_past<float4v>(p + 64 * j);
      x.w[tile][i][4 * j] = u.x; x.w[tile][i][4 * j + 1] = u.y; x.w[tile][i][4 * j + 2] = u.z; x.w[tile][i][4 * j + 3] = u.w;
    }
  }
  template <int N> static __device__ __forceinline__ void scores(const Queries (&q)[N], const Keys& x, float4v (&acc)[N][kTiles]) {
    float4v odd[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j][0] = odd[j] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KW; i += 2)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        acc[j][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w[0][i], q[j].w[i], acc[j][0], 0, 0, 0);
        odd[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w[0][i + 1], q[j].w[i + 1], odd[j], 0, 0, 0);
      }
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][0][i] += odd[j][i];
  }
  static __device__ __forceinline__ void weights(const float (&p)[kTiles][4], Weights& w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w.p[i] = p[0][i];
  }
  typedef Values Operands;
  static __device__ __forceinline__ void operands(const Values& x, Operands& o) { o = x; }
  static __device__ __forceinline__ void add(const Weights& p, const Operands& x, float4v (&out)[VT]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < VT; ++t) out[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(p.p[i], x.w[0][i][t], out[t], 0, 0, 0);
  }
  static constexpr int kPieces = D / 4;
  static __device__ __forceinline__ int k_place(int row, int piece) { return row * kPieces + (piece ^ row); }      // (16 rows)
  static __device__ __forceinline__ void read(const u32x4* k, int c16, int g4, Keys& x) {
#pragma unroll
    for (int j = 0; j < KW / 4; ++j) {
      const float4v u = __builtin_bit_cast(float4v, k[k_place(c16, g4 + 4 * j)]);
      x.w[0][4 * j] = u.x; x.w[0][4 * j + 1] = u.y; x.w[0][4 * j + 2] = u.z; x.w[0][4 * j + 3] = u.w;
    }
  }
  static __device__ __forceinline__ void read(const u32x4* v, int c16, int g4, Values& x) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < VT / 4; ++j) {
        const float4v u = __builtin_bit_cast(float4v, v[(4 * g4 + i) * kPieces + 16 * j + c16]);
        x.w[0][i][4 * j] = u.x; x.w[0][i][4 * j + 1] = u.y; x.w[0][i][4 * j + 2] = u.z; x.w[0][i][4 * j + 3] = u.w;
      }
  }
  static __device__ __forceinline__ void negate(Queries& q) {
#pragma unroll
    for (int i = 0; i < KW; ++i) q.w[i] = -q.w[i];
  }
};

// The scale of scores in log2 units, above 0 (queries change their signs for a negative one), and how scores are compared with a reference.
struct Scale {
  float log2e, inverse;
  bool negate;
};

// A wave's online softmax over N tiles of queries that read the same rows: reference (in log2 units, common to the four lanes of a query), this lane's
// sum, weighted V of queries 4 g4 + i.  The reference is the largest score at first and is moved only when one exceeds it by 2^kSlack.
template <typename T, int D, int N> struct State {
  typedef Form<T, D> F;
  static constexpr uint32_t kAll = F::kRows == 32 ? 0xFFFFFFFFu : 0xFFFFu;
  float m[N], shift[N], limit[N], sum[N];                  // shift: the reference, or 0 before there is one; limit: where it is moved, in products
  float4v out[N][F::VT];
  __device__ __forceinline__ State() {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      m[j] = limit[j] = -INFINITY;
      shift[j] = sum[j] = 0.f;
#pragma unroll
      for (int t = 0; t < F::VT; ++t) out[j][t] = float4v{0.f, 0.f, 0.f, 0.f};
    }
  }
  // A step's products of K and queries: those of rows that are not there (`there`: a bit each for those that are) are left out, and the reference is moved
  // if one exceeds it.
  __device__ __forceinline__ void refer(int j, float4v (&acc)[F::kTiles], uint32_t there, const Scale& scale, int g4) {
    if (there != kAll)
#pragma unroll
      for (int tt = 0; tt < F::kTiles; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!((there >> (16 * tt + 4 * g4 + i)) & 1u)) acc[tt][i] = -INFINITY;
    float mx = -INFINITY;
#pragma unroll
    for (int tt = 0; tt < F::kTiles; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, acc[tt][i]);
    if (__any(mx > limit[j])) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float m_new = mx == -INFINITY ? m[j] : fmaxf(m[j], mx * scale.log2e);
      const float alpha = m_new == -INFINITY ? 1.f : exp2f(m[j] - m_new);
      m[j] = m_new;
      shift[j] = m_new == -INFINITY ? 0.f : m_new;
      limit[j] = (m_new + kSlack) * scale.inverse;
      sum[j] *= alpha;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = __shfl(alpha, 4 * g4 + i, 64);
#pragma unroll
        for (int t = 0; t < F::VT; ++t) out[j][t][i] *= a;
      }
    }
  }
  // ... as weights
  __device__ __forceinline__ void weigh(int j, const float4v (&acc)[F::kTiles], const Scale& scale, typename F::Weights& w) {
    float p[F::kTiles][4], more = 0.f;
#pragma unroll
    for (int tt = 0; tt < F::kTiles; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) p[tt][i] = __builtin_amdgcn_exp2f(fmaf(acc[tt][i], scale.log2e, -shift[j]));
#pragma unroll
    for (int tt = 0; tt < F::kTiles; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) more += p[tt][i];
    sum[j] += more;
    F::weights(p, w);
  }
};

// A wave's steps 0 .. n - 1, two under way.  `begin(step, r)` loads what leads to the place of row r of a step, `finish` takes that and loads the place
// (the cache row, or kNoRow): both for as many steps together as 64 lanes have rows of, and a turn ahead of their use.
template <typename T, int D, typename Begin, typename Finish>
__device__ __forceinline__ void walk(State<T, D, 1>& state, const typename Form<T, D>::Queries (&q)[1], const T* K, const T* V, int n, const Scale& scale, int lane,
                                     const Begin& begin, const Finish& finish) {
  typedef Form<T, D> F;
  constexpr int kTogether = 64 / F::kRows;                 // steps of a look-up
  const int c16 = lane & 15, g4 = lane >> 4, r = lane % F::kRows, of = lane / F::kRows;
  struct Step {
    typename F::Keys k;
    typename F::Values v;
    uint32_t there;
  } xa, xb;
  if (n <= 0) return;
  auto begin_group = [&](int group) { return begin(min(group * kTogether + of, n - 1), r); };
  auto finish_group = [&](int group, auto token) {
    const uint32_t place = finish(token, min(group * kTogether + of, n - 1), r);
    return group * kTogether + of < n ? place : kNoRow;
  };
  const auto t0 = begin_group(0), t1 = begin_group(1);
  auto ahead = begin_group(2);
  uint32_t now = finish_group(0, t0), next = finish_group(1, t1);
  int group = 0;
  // Rows that are not there are read as the step's first one that is: what a cache holds in other places may be anything.
  auto ask = [&](int st, Step& x) {
    if (st / kTogether != group) {
      now = next;
      next = finish_group(group + 2, ahead);
      ahead = begin_group(group + 3);
      ++group;
    }
    const int base = st % kTogether * F::kRows;
    const uint64_t found = __ballot(now != kNoRow) >> base;
    x.there = (uint32_t)found & State<T, D, 1>::kAll;
    if (x.there == 0) return;
    const uint32_t stand_in = (uint32_t)__builtin_amdgcn_readlane((int)now, base + __builtin_ctz(x.there));
    const uint32_t row = now == kNoRow ? stand_in : now;
#pragma unroll
    for (int tt = 0; tt < F::kTiles; ++tt) {
      F::load_k(K, (uint32_t)__shfl((int)row, base + 16 * tt + c16, 64), g4, tt, x.k);
#pragma unroll
      for (int i = 0; i < 4; ++i) F::load_v(V, (uint32_t)__shfl((int)row, base + 16 * tt + 4 * g4 + i, 64), c16, tt, i, x.v);
    }
  };
  ask(0, xa);
  if (n > 1) ask(1, xb);
  auto turn = [&](int st, Step& x) {
    if (x.there) {
      float4v acc[1][F::kTiles];
      F::template scores<1>(q, x.k, acc);
      state.refer(0, acc[0], x.there, scale, g4);
      typename F::Weights w;
      state.weigh(0, acc[0], scale, w);
      typename F::Operands v;
      F::operands(x.v, v);
      F::add(w, v, state.out[0]);
    }
    if (st + 2 < n) ask(st + 2, x);
  };
  for (int st = 0; st < n; st += 2) {
    turn(st, xa);
    if (st + 1 < n) turn(st + 1, xb);
  }
}

// What parts are weighted by, of the largest score that they have.  Without one (no rows, or scores that are not numbers, which no maximum takes) it is 0:
// parts without rows are zeros and stay so, and what is not a number stays that.
__device__ __forceinline__ float reference_of(float largest) { return largest > -INFINITY ? largest : 0.f; }

// The waves' states as one, through LDS in a fixed order: into a record of `rows` queries, or (whole) the result itself.
constexpr size_t merge_bytes(int d) { return (size_t)kAttWaves * 16 * (d + 2) * sizeof(float); }
template <typename T, int D>
__device__ __forceinline__ void merge_waves(State<T, D, 1>& state, int rows, float* lds, float* record, float* whole) {
  typedef Form<T, D> F;
  float(*const sm_m)[16] = reinterpret_cast<float(*)[16]>(lds);
  float(*const sm_l)[16] = sm_m + kAttWaves;
  float(*const sm_o)[16][D] = reinterpret_cast<float(*)[16][D]>(sm_l + kAttWaves);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c16 = lane & 15, g4 = lane >> 4;
  float sum = state.sum[0];
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  if (g4 == 0) { sm_m[wave][c16] = state.m[0]; sm_l[wave][c16] = sum; }
#pragma unroll
  for (int t = 0; t < F::VT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) sm_o[wave][4 * g4 + i][F::column(c16, t)] = state.out[0][t][i];
  __syncthreads();
  for (int item = tid; item < rows * D; item += kAttThreads) {
    const int g = item / D, dim = item % D;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w) M = fmaxf(M, sm_m[w][g]);
    const float ref = reference_of(M);
    float acc = 0.f, lt = 0.f;
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w) {
      const float f = exp2f(sm_m[w][g] - ref);
      acc = fmaf(sm_o[w][g][dim], f, acc);
      lt = fmaf(sm_l[w][g], f, lt);
    }
    if (whole) {
      whole[(int64_t)g * D + dim] = acc / (lt == 0.f ? 1.f : lt);
    } else {
      record[2 * rows + item] = acc;
      if (dim == 0) { record[g] = M; record[rows + g] = lt; }
    }
  }
}

// Tile j of a wave's state into a record of `queries`, from query `from` on.
template <typename T, int D, int N>
__device__ __forceinline__ void write_record(const State<T, D, N>& state, int j, int from, int queries, float* record, int lane) {
  typedef Form<T, D> F;
  const int c16 = lane & 15, g4 = lane >> 4;
  float sum = state.sum[j];
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  if (g4 == 0 && from + c16 < queries) {
    record[from + c16] = state.m[j];
    record[queries + from + c16] = sum;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int query = from + 4 * g4 + i;
    if (query < queries)
#pragma unroll
      for (int t = 0; t < F::VT; t += 2) {                 // (neighbouring columns; records' rows lie at multiples of 8 bytes)
        float* const to = record + 2 * queries + (int64_t)query * D + F::column(c16, t);
        *reinterpret_cast<float2v*>(to) = float2v{state.out[j][t][i], state.out[j][t + 1][i]};
      }
  }
}

// ---- pages that a list names -------------------------------------------------------------------
// grid = (parts, units): the waves of a unit's parts take its steps in turn, so that a list that ends early leaves none idle before the others.
template <typename T, int D>
__global__ __launch_bounds__(kAttThreads, 2) void attend_chosen_kernel(PagedArgs a, const T* __restrict__ Q, int G, const int32_t* __restrict__ chosen, int count,
                                                                       Scale scale, float* __restrict__ records, float* __restrict__ whole) {
  typedef Form<T, D> F;
  const int u = blockIdx.y, b = u / (a.L * a.H), in = u - b * a.L * a.H;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g4 = lane >> 4;
  const int rows = rows_of(a, b, in / a.H);
  const int32_t* const table = a.table + b * a.table_b + (int64_t)in * a.max_pages;
  const int32_t* const list = chosen + (int64_t)u * count;
  typename F::Queries q[1];
  F::queries(Q + ((int64_t)u * G + min(c16, G - 1)) * D, c16 < G, g4, q[0]);
  if (scale.negate) F::negate(q[0]);
  const int waves = gridDim.x * kAttWaves, wave = blockIdx.x * kAttWaves + uniform(threadIdx.x >> 6);
  const int steps = (count * a.page_size + F::kRows - 1) / F::kRows;
  // step i of the wave is step wave + i * waves of the unit
  auto begin = [&](int i, int r) { return list[min(a.pages.of((wave + i * waves) * F::kRows + r), count - 1)]; };
  auto finish = [&](int p, int i, int r) -> uint32_t {
    const int at = (wave + i * waves) * F::kRows + r, entry = a.pages.of(at), off = at - entry * a.page_size;
    const bool held = entry < count && p >= 0 && p < a.max_pages && (int64_t)p * a.page_size + off < rows;
    const int page = table[held ? p : 0];
    return held && page >= 0 && page < a.num_pages ? (uint32_t)page * (uint32_t)a.page_size + (uint32_t)off : kNoRow;
  };
  State<T, D, 1> state;
  walk<T, D>(state, q, static_cast<const T*>(a.K), static_cast<const T*>(a.V), (steps - wave + waves - 1) / waves, scale, lane, begin, finish);
  __shared__ __align__(16) float merged[merge_bytes(D) / sizeof(float)];
  merge_waves<T, D>(state, G, merged, records + ((int64_t)u * gridDim.x + blockIdx.x) * record_floats(G, D), whole ? whole + (int64_t)u * G * D : nullptr);
}

// What records hold of a query's row: largest score, sum, four columns of the weighted V.
struct Part {
  float m = -INFINITY, sum = 0.f;
  float4v o = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void join(float m2, float sum2, const float4v& o2) {
    const float M = fmaxf(m, m2), ref = reference_of(M);
    const float w1 = exp2f(m - ref), w2 = exp2f(m2 - ref);
    m = M;
    sum = sum * w1 + sum2 * w2;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * w1 + o2[i] * w2;
  }
  // records from, from + step, ... below end at `base`, each of `queries` rows, `size` floats; as many under way as there are, up to eight
  template <int D> __device__ __forceinline__ void join_records(const float* base, int from, int end, int step, int64_t size, int queries, int row, int c4) {
    const int n = end - from;
    if (n <= 0) return;
    if (n <= step) join_some<D, 1>(base, from, end, step, size, queries, row, c4);
    else if (n <= 2 * step) join_some<D, 2>(base, from, end, step, size, queries, row, c4);
    else if (n <= 4 * step) join_some<D, 4>(base, from, end, step, size, queries, row, c4);
    else join_some<D, 8>(base, from, end, step, size, queries, row, c4);
  }
  template <int D, int kAtOnce>
  __device__ __forceinline__ void join_some(const float* base, int from, int end, int step, int64_t size, int queries, int row, int c4) {
    for (int k0 = from; k0 < end; k0 += kAtOnce * step) {
      float ms[kAtOnce], sums[kAtOnce];
      float4v os[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const float* const rec = base + min(k0 + j * step, end - 1) * size;
        ms[j] = k0 + j * step < end ? rec[row] : -INFINITY;
        sums[j] = rec[queries + row];
        // (records' rows lie at multiples of 8 bytes)
        const float* const o = rec + 2 * queries + (int64_t)row * D + 4 * c4;
        const float2v a = *reinterpret_cast<const float2v*>(o), b = *reinterpret_cast<const float2v*>(o + 2);
        os[j] = float4v{a.x, a.y, b.x, b.y};
      }
      float M = m;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) M = fmaxf(M, ms[j]);
      const float ref = reference_of(M), w = exp2f(m - ref);
      m = M;
      sum *= w;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= w;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const float v = exp2f(ms[j] - ref);
        sum = fmaf(sums[j], v, sum);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(os[j][i], v, o[i]);
      }
    }
  }
};

// The parts that a workgroup's `slots` threads of each item have, in order, and the result of the first at `out`.
__device__ __forceinline__ void finish_parts(Part& part, int slots, int per_slot, int slot, bool has, float* lds, float* out) {
  if (slots > 1) {
    float* const mine = lds + threadIdx.x * 6;
    if (slot > 0 && has) {
      mine[0] = part.m;
      mine[1] = part.sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) mine[2 + i] = part.o[i];
    }
    __syncthreads();
    if (slot == 0 && has)
      for (int j = 1; j < slots; ++j) {
        const float* const x = mine + j * per_slot * 6;
        part.join(x[0], x[1], float4v{x[2], x[3], x[4], x[5]});
      }
  }
  if (slot == 0 && has) {
    const float sum = part.sum == 0.f ? 1.f : part.sum;    // (no rows: zeros)
    *reinterpret_cast<float4v*>(out) = float4v{part.o[0] / sum, part.o[1] / sum, part.o[2] / sum, part.o[3] / sum};
  }
}

// grid = (units, parts of a unit's items): an item is four columns of one query; a thread has every `slots`-th record of one.
template <int D> __global__ __launch_bounds__(1024) void chosen_merge_kernel(const float* __restrict__ records, int parts, int G, int slots, float* __restrict__ out) {
  extern __shared__ float joined[];
  const int u = blockIdx.x, per_slot = blockDim.x / slots, slot = threadIdx.x / per_slot, item = blockIdx.y * per_slot + threadIdx.x - slot * per_slot;
  const bool has = item < G * (D / 4);
  const int64_t size = record_floats(G, D);
  Part part;
  if (has) part.join_records<D>(records + (int64_t)u * parts * size, slot, parts, slots, size, G, item / (D / 4), item % (D / 4));
  finish_parts(part, slots, per_slot, slot, has, joined, out + (int64_t)u * G * D + 4 * item);
}

// ---- rows of a shared prompt, and of each sequence ---------------------------------------------
struct SharedArgs {
  PagedArgs common, own;         // of P prompts and of B sequences
  const int32_t* starts;         // [P + 1]
  int G, groups;                 // pieces of prompts that the launch aims at
  int most_common, common_groups;        // records of prompts that the workspace has; workgroups for them, the launch's first
  int record_rows;               // queries that a prompt's record has room for
  int own_parts, step_rows;      // waves of a sequence's unit, each with a record; rows of a step
  Scale scale;
  float* common_records;
  float* own_records;
  int2* span;                    // of each prompt's layers: first record, pieces of a unit
  float* out;
};

// Sequences of prompt p: [first, first + n)
struct Run { int first, n; };
__device__ __forceinline__ Run run_of(const SharedArgs& a, int p) {
  const int s0 = min(max(a.starts[p], 0), a.own.B), s1 = min(max(a.starts[p + 1], 0), a.own.B);
  return {s0, max(0, s1 - s0)};
}
__device__ __forceinline__ int tiles_of(const SharedArgs& a, int n) { return (n * a.G + kTileQueries - 1) / kTileQueries; }

// Entry e: a layer of a prompt.  Its rows, and how many units and query tiles have them to read.
struct Entry { int rows, times; };
__device__ __forceinline__ Entry entry_at(const SharedArgs& a, int e, int entries) {
  const int at = min(e, entries - 1), p = at / a.own.L;
  const Entry x{rows_of(a.common, p, at - p * a.own.L), a.own.H * tiles_of(a, run_of(a, p).n)};
  return e < entries ? x : Entry{0, 0};
}
template <int ROWS> __device__ __forceinline__ int steps_in(int rows) { return (rows + ROWS - 1) / ROWS; }

__device__ __forceinline__ int64_t wave_sum(int64_t v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_add(int v) {     // 0 where there is no source lane
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int v) {          // sums up to and with each lane
  v = dpp_add<0x111, 0xF>(v);      // row_shr:1, 2, 4, 8
  v = dpp_add<0x112, 0xF>(v);
  v = dpp_add<0x114, 0xF>(v);
  v = dpp_add<0x118, 0xF>(v);
  v = dpp_add<0x142, 0xA>(v);      // row_bcast:15 into rows 1 and 3
  return dpp_add<0x143, 0xC>(v);   // row_bcast:31 into rows 2 and 3
}

// Steps' rows of K and V in LDS, kStages of them; the places of 64 steps' rows, and which of them there are.
constexpr int kStages = 4;             // (three under way: request, wait and barrier below go by that)
template <typename T, int D> struct Staged {
  typedef Form<T, D> F;
  static constexpr int kVectors = F::kRows * F::kPieces;   // of 16 bytes, of K or V
  u32x4 k[kStages][kVectors], v[kStages][kVectors];
  uint32_t places[kStepsLooked * F::kRows];
  uint32_t there[kStepsLooked];
};

// 16 bytes a lane from memory into LDS, side by side from `to` on (the same for the wave); nothing for lanes that are off.  It counts as a load; what it
// writes is there behind a wait for it.  (Written out: behind the builtin the compiler waits for all loads under way before it reads LDS.  There is
// no output register that could be taken for written before it is, and these kernels use m0 for nothing else: it is reserved, so it cannot be named as written.)
__device__ __forceinline__ void load_to_lds(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ uint32_t lds_offset(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }
// All but the last `left` loads (an even number up to 8) are done with.
__device__ __forceinline__ void wait_for_loads(int left) {
  if (left == 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  else if (left == 6) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
  else if (left == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
  else if (left == 2) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Steps first .. end of a unit's rows for up to 64 N queries, N tiles a wave (tiles behind the last query are zeros).  Rows go from memory straight into
// LDS, three steps ahead, a quarter of them by each wave; one barrier a step.
template <typename T, int D, int N, typename Places, typename LoadQueries>
__device__ __forceinline__ void wide_piece(void* lds, const T* K, const T* V, int first, int end, int queries, const Scale& scale, float* record,
                                           const Places& place_of, const LoadQueries& load_queries) {
  typedef Form<T, D> F;
  typedef Staged<T, D> S;
  constexpr int kMine = S::kVectors / kAttThreads;         // vectors of K, and of V, a thread and step
  static_assert(S::kVectors % kAttThreads == 0 && 4 * kMine <= 8, "a thread has whole vectors; two steps' loads at most are waited for by number");
  S& s = *static_cast<S*>(lds);
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), c16 = lane & 15, g4 = lane >> 4;
  const int from = 16 * wave;                              // the wave's first query
  typename F::Queries q[N];
#pragma unroll
  for (int j = 0; j < N; ++j) load_queries(from + j * 16 * kAttWaves, q[j]);
  State<T, D, N> state;
  // (rows that are not there stay what LDS has: values, for which a weight of 0 has to make 0)
  u32x4* const all_v = &s.v[0][0];
  for (int i = tid; i < kStages * S::kVectors; i += kAttThreads) all_v[i] = u32x4{0u, 0u, 0u, 0u};
  const uint32_t k_at = lds_offset(&s.k[0][wave * 64]), v_at = lds_offset(&s.v[0][wave * 64]);
  uint32_t place[kMine];                                   // of this thread's vectors, of the step that is requested next
  auto look = [&](int at) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) place[i] = s.places[at * F::kRows + (i * kAttThreads + tid) / F::kPieces];
  };
  auto request = [&](int at) -> int {                      // step `at` of those that were looked up; how many loads of this wave that makes
    int loads = 0;
    const uint32_t stage = (uint32_t)(at % kStages) * (uint32_t)(S::kVectors * 16);
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int m = i * kAttThreads + tid, row = m / F::kPieces, piece = m % F::kPieces;
      if (place[i] != kNoRow) {
        const int64_t from = (int64_t)place[i] * (D * (int)sizeof(T));
        // (K's swapped places, the other way round)
        load_to_lds(reinterpret_cast<const char*>(K) + from + (F::k_place(row, piece) - row * F::kPieces) * 16, k_at + stage + i * kAttThreads * 16);
        load_to_lds(reinterpret_cast<const char*>(V) + from + piece * 16, v_at + stage + i * kAttThreads * 16);
      }
      loads += __any(place[i] != kNoRow) ? 2 : 0;          // (none without a lane that has a row)
    }
    look(min(at + 1, kStepsLooked - 1));
    return loads;
  };
  for (int base = first; base < end; base += kStepsLooked) {
    const int n = min(kStepsLooked, end - base);
    __syncthreads();                                       // (the steps before are done with)
    for (int r = tid; r < n * F::kRows; r += kAttThreads) {
      const uint32_t place = place_of(base * F::kRows + r);
      s.places[r] = place;
      const uint64_t found = __ballot(place != kNoRow);    // (whole steps a wave, or none)
      if constexpr (F::kRows == 32) {
        if ((lane & 31) == 0) s.there[r / 32] = (uint32_t)(found >> lane);
      } else {
        if ((lane & 15) == 0) s.there[r / 16] = (uint32_t)(found >> lane) & 0xFFFFu;
      }
    }
    __syncthreads();
    look(0);
    request(0);
    int after = n > 1 ? request(1) : 0, after_that = n > 2 ? request(2) : 0;     // loads of the steps behind the one that is waited for
    for (int at = 0; at < n; ++at) {
      const uint32_t there = (uint32_t)uniform((int)s.there[at]);
      // this wave's part of the step is in LDS; behind the barrier everybody's is, and the step before is done with
      wait_for_loads(after + after_that);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      after = after_that;
      after_that = at + kStages - 1 < n ? request(at + kStages - 1) : 0;
      if (there && from < queries) {
        const int stage = at % kStages;
        typename F::Keys k;
        typename F::Values v;
        F::read(s.k[stage], c16, g4, k);
        F::read(s.v[stage], c16, g4, v);
        float4v acc[N][F::kTiles];
        F::template scores<N>(q, k, acc);
#pragma unroll
        for (int j = 0; j < N; ++j) state.refer(j, acc[j], there, scale, g4);
        typename F::Operands o;
        F::operands(v, o);
        // a tile's products beside the next one's weights
        typename F::Weights w[N];
        state.weigh(0, acc[0], scale, w[0]);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          if (j + 1 < N) state.weigh(j + 1, acc[j + 1], scale, w[j + 1]);
          F::add(w[j], o, state.out[j]);
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) write_record<T, D, N>(state, j, from + j * 16 * kAttWaves, queries, record, lane);
}

template <typename T, int D> constexpr size_t shared_lds_bytes() { return sizeof(Staged<T, D>) > merge_bytes(D) ? sizeof(Staged<T, D>) : merge_bytes(D); }

// A sequence's own rows: a wave has every own_parts-th step of a unit.  (Nothing here depends on what other sequences hold: to find a place among them
// by their rows, as the prompts' pieces do, took longer than the rows.)
template <typename T, int D> __device__ __forceinline__ void own_part(const SharedArgs& a, const T* Q, int64_t wave) {
  typedef Form<T, D> F;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g4 = lane >> 4, L = a.own.L, H = a.own.H, G = a.G, parts = a.own_parts;
  const int u = uniform((int)(wave / parts)), part = uniform((int)(wave - (int64_t)u * parts));
  if (u >= a.own.B * L * H) return;
  const int b = u / (L * H), in = u - b * L * H, rows = uniform(rows_of(a.own, b, in / H));
  const int n = (steps_in<F::kRows>(rows) - part + parts - 1) / parts;
  if (n <= 0) return;
  const int32_t* const table = a.own.table + b * a.own.table_b + (int64_t)in * a.own.max_pages;
  typename F::Queries q[1];
  F::queries(Q + ((int64_t)u * G + min(c16, G - 1)) * D, c16 < G, g4, q[0]);
  if (a.scale.negate) F::negate(q[0]);
  State<T, D, 1> state;
  walk<T, D>(state, q, static_cast<const T*>(a.own.K), static_cast<const T*>(a.own.V), n, a.scale, lane,
             [&](int i, int r) { return table[a.own.pages.of(min((part + i * parts) * F::kRows + r, rows - 1))]; },
             [&](int page, int i, int r) {
               const int row = (part + i * parts) * F::kRows + r;
               return row < rows && page >= 0 && page < a.own.num_pages
                          ? (uint32_t)page * (uint32_t)a.own.page_size + (uint32_t)(row - a.own.pages.of(row) * a.own.page_size) : kNoRow;
             });
  write_record<T, D, 1>(state, 0, 0, G, a.own_records + wave * record_floats(G, D), lane);
}

// A piece of a prompt's rows for up to 128 queries of its sequences.  Pieces are as long as each other, whatever the layers hold: every wave finds out
// by itself how many pieces the layers before make.
template <typename T, int D> __device__ __forceinline__ void common_piece(const SharedArgs& a, const T* Q, int w, unsigned char* lds) {
  typedef Form<T, D> F;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g4 = lane >> 4, wave = uniform(threadIdx.x >> 6);
  const int L = a.own.L, H = a.own.H, G = a.G, entries = a.common.B * L;
  if (entries == 0) return;
  const Entry front = entry_at(a, lane, entries);          // (mostly all)
  int64_t total = (int64_t)steps_in<F::kRows>(front.rows) * front.times;
  int units = front.rows > 0 ? front.times : 0;
  for (int e0 = 64; e0 < entries; e0 += 64) {
    const Entry x = entry_at(a, e0 + lane, entries);
    total += (int64_t)steps_in<F::kRows>(x.rows) * x.times;
    units += x.rows > 0 ? x.times : 0;
  }
  total = wave_sum(total);
  units = (int)wave_sum(units);
  // a unit's last piece is part of one: as many pieces as are resident together, with one for each unit among them; of more units than that twice as many
  // as units at most
  const int64_t aim = max(a.groups - units, (units + 1) / 2);
  int each = (int)max((int64_t)kLeastSteps, (total + aim - 1) / max(aim, (int64_t)1));
  if (entries <= 64)                                       // the shortest that makes as many (units' last pieces are half of one in the mean)
    for (int least = (int)max((int64_t)kLeastSteps, (total + a.groups - 1) / a.groups); least < each;) {
      const int middle = (least + each) / 2;
      const int made = __builtin_amdgcn_readlane(wave_scan((steps_in<F::kRows>(front.rows) + middle - 1) / middle * front.times), 63);
      if (made <= a.groups) each = middle;
      else least = middle + 1;
    }
  int before = 0, entry = -1, rows = 0, pieces = 0, place = 0;     // (all pieces are fewer than most_common, below 2^31, unless starts fall)
  for (int e0 = 0; e0 < entries && entry < 0; e0 += 64) {
    const Entry x = e0 == 0 ? front : entry_at(a, e0 + lane, entries);
    const int mine = (steps_in<F::kRows>(x.rows) + each - 1) / each, all = mine * x.times, upto = before + wave_scan(all);
    const uint64_t past = __ballot(upto > w);
    if (past) {
      const int from = __builtin_ctzll(past);
      entry = e0 + from;
      rows = __builtin_amdgcn_readlane(x.rows, from);
      pieces = __builtin_amdgcn_readlane(mine, from);
      place = w - __builtin_amdgcn_readlane(upto - all, from);
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  if (entry < 0) return;
  if (place == 0 && threadIdx.x == 0) a.span[entry] = int2{w, pieces};
  const int unit = place / pieces, piece = place - unit * pieces;
  // the unit's head, and the tile's queries
  const int p = entry / L, l = entry - p * L;
  const Run run = run_of(a, p);
  const int tiles = tiles_of(a, run.n), h = unit / tiles, tile = unit - h * tiles, queries = min(kTileQueries, run.n * G - tile * kTileQueries);
  const PagedArgs& kv = a.common;
  const int32_t* const table = kv.table + p * kv.table_b + ((int64_t)l * H + h) * kv.max_pages;
  const T* const K = static_cast<const T*>(kv.K);
  const T* const V = static_cast<const T*>(kv.V);
  auto place_of = [&](int row) -> uint32_t {
    if (row >= rows) return kNoRow;
    const int at = kv.pages.of(row), page = table[at];
    return page >= 0 && page < kv.num_pages ? (uint32_t)page * (uint32_t)kv.page_size + (uint32_t)(row - at * kv.page_size) : kNoRow;
  };
  // query c16 of a tile of 16
  auto load_queries = [&](int from, typename F::Queries& q) {
    const bool has = from + c16 < queries;
    const int r = tile * kTileQueries + from + c16, b = has ? run.first + r / G : run.first, g = has ? r % G : 0;
    F::queries(Q + (((int64_t)b * L + l) * H * G + (int64_t)h * G + g) * D, has, g4, q);
    if (a.scale.negate) F::negate(q);
  };
  float* const record = a.common_records + w * record_floats(a.record_rows, D);
  const int steps = steps_in<F::kRows>(rows), s0 = (int)((int64_t)steps * piece / pieces), s1 = (int)((int64_t)steps * (piece + 1) / pieces);
  if (queries <= 16) {
    typename F::Queries q[1];
    load_queries(0, q[0]);
    State<T, D, 1> state;
    // the waves take the piece's steps in turn
    walk<T, D>(state, q, K, V, (s1 - s0 - wave + kAttWaves - 1) / kAttWaves, a.scale, lane,
               [&](int i, int r) { return table[kv.pages.of(min((s0 + wave + i * kAttWaves) * F::kRows + r, rows - 1))]; },
               [&](int page, int i, int r) {
                 const int row = (s0 + wave + i * kAttWaves) * F::kRows + r;
                 return row < rows && page >= 0 && page < kv.num_pages
                            ? (uint32_t)page * (uint32_t)kv.page_size + (uint32_t)(row - kv.pages.of(row) * kv.page_size) : kNoRow;
               });
    merge_waves<T, D>(state, queries, reinterpret_cast<float*>(lds), record, nullptr);
  } else if (queries <= 64) {
    wide_piece<T, D, 1>(lds, K, V, s0, s1, queries, a.scale, record, place_of, load_queries);
  } else {
    wide_piece<T, D, 2>(lds, K, V, s0, s1, queries, a.scale, record, place_of, load_queries);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kAttThreads, 2) void attend_shared_kernel(SharedArgs a, const T* __restrict__ Q) {
  extern __shared__ __align__(16) unsigned char lds[];
  if ((int)blockIdx.x < a.common_groups) common_piece<T, D>(a, Q, blockIdx.x, lds);
  else own_part<T, D>(a, Q, (int64_t)((int)blockIdx.x - a.common_groups) * kAttWaves + uniform(threadIdx.x >> 6));
}

// The records of the prompt's pieces and of the sequence's own, in order; grid and threads as of chosen_merge_kernel.
template <int D> __global__ __launch_bounds__(1024) void shared_merge_kernel(SharedArgs a, int slots) {
  extern __shared__ float joined[];
  const int L = a.own.L, H = a.own.H, G = a.G, u = blockIdx.x, lane = threadIdx.x & 63, P = a.common.B;
  const int b = u / (L * H), l = u / H % L, h = u % H;
  const int per_slot = blockDim.x / slots, slot = threadIdx.x / per_slot, item = blockIdx.y * per_slot + threadIdx.x - slot * per_slot;
  const int g = item / (D / 4), c4 = item % (D / 4);
  const bool has = item < G * (D / 4);
  const int own_rows = rows_of(a.own, b, l);
  // the prompt whose sequence this is, with what its layer holds: 64 prompts' together, a lane each, in one wait for memory
  Run run{0, 0};
  int2 span{0, 0};
  for (int p0 = 0; p0 < P; p0 += 64) {
    const int mine = min(p0 + lane, P - 1);
    const Run r = run_of(a, mine);
    const int rows = rows_of(a.common, mine, l);
    const int2 s = a.span[mine * L + l];
    const uint64_t found = __ballot(p0 + lane < P && b >= r.first && b < r.first + r.n);
    if (found) {
      const int from = __builtin_ctzll(found);
      run = Run{__builtin_amdgcn_readlane(r.first, from), __builtin_amdgcn_readlane(r.n, from)};
      if (__builtin_amdgcn_readlane(rows, from) > 0) span = int2{__builtin_amdgcn_readlane(s.x, from), __builtin_amdgcn_readlane(s.y, from)};
      break;
    }
  }
  Part part;
  if (span.y > 0 && span.x >= 0) {
    const int tiles = tiles_of(a, run.n), at = (b - run.first) * G + g, tile = at / kTileQueries;
    const int64_t index = span.x + (int64_t)(h * tiles + tile) * span.y, size = record_floats(a.record_rows, D);
    if (has && index + span.y <= a.most_common)
      part.join_records<D>(a.common_records + index * size, slot, span.y, slots, size, min(kTileQueries, run.n * G - tile * kTileQueries),
                           at - tile * kTileQueries, c4);
  }
  const int64_t size = record_floats(G, D);
  if (has)
    part.join_records<D>(a.own_records + (int64_t)u * a.own_parts * size, slot, min(a.own_parts, (own_rows + a.step_rows - 1) / a.step_rows), slots, size, G, g, c4);
  finish_parts(part, slots, per_slot, slot, has, joined, a.out + (int64_t)u * G * D + 4 * item);
}

// Shape of a merge: threads for all items of a unit, or, of few units, a wave's in each of several workgroups; more slots where there are many records.
struct MergeShape {
  int slots, threads, along;
  size_t lds;
};
MergeShape merge_shape(int units, int records, int G, int d) {
  const int items = G * (d / 4), all = (items + 63) / 64 * 64, per_slot = units >= 256 ? all : 64, along = (items + per_slot - 1) / per_slot;
  int slots = 1;
  while (slots < 16 && records > 4 * slots && (int64_t)units * along * 2 * slots * per_slot <= 256 * 1024 && 2 * slots * per_slot <= 1024) slots *= 2;
  return {slots, slots * per_slot, along, slots > 1 ? (size_t)slots * per_slot * 6 * sizeof(float) : 0};
}

Scale scale_of(float scale) {
  const float s = fmaxf(fabsf(scale) * 1.4426950408889634f, 1.17549435e-38f);    // (0 would make a number of what is not there)
  return Scale{s, 1.f / s, scale < 0.f};
}

// Query tiles of all prompts at most
int64_t most_tiles(int P, int B, int G) {
  const int runs = std::min(P, B);
  return runs + ((int64_t)B * G - runs) / kTileQueries;
}

struct SharedSizes {
  int groups, record_rows, own_parts;
  int64_t common, own, span, total;    // records, entries, bytes
};
SharedSizes shared_sizes(int P, int B, int L, int H, int G, int d, int dtype) {
  SharedSizes z;
  const int64_t units = (int64_t)B * L * H;
  // pieces of prompts: some less than as many workgroups as are resident together (two on a compute unit, three of 64 columns); how many less goes by one
  // measured case (16 answers to 28 layers: 512 of them 148 us, 480 138, 448 150); of sequences: parts for four times as many waves, 16 of a unit at most
  z.groups = d == 64 ? 720 : 480;
  z.own_parts = (int)std::max<int64_t>(1, std::min<int64_t>(16, 8192 / units));
  const int64_t tiles = (int64_t)L * H * most_tiles(P, B, G);
  z.common = P ? std::max<int64_t>(z.groups, tiles + tiles / 2 + 1) + 1 : 0;
  z.own = units * z.own_parts;
  z.span = (int64_t)P * L;
  z.record_rows = std::min(kTileQueries, B * G);
  z.total = (z.common * record_floats(z.record_rows, d) + z.own * record_floats(G, d)) * (int64_t)sizeof(float) + z.span * (int64_t)sizeof(int2);
  return z;
}

// Workgroups that a unit's `steps` are cut into.  512 are resident together; a round of them costs about two steps besides what its waves have to do, so
// that long lists are cut for one round and a step a wave is the least.
int chosen_parts(int units, int count, int page_size, int step_rows) {
  const int64_t steps = ((int64_t)count * page_size + step_rows - 1) / step_rows;
  int best = 1;
  int64_t least = INT64_MAX;
  for (int parts = 1; parts <= 64 && (parts == 1 || (int64_t)kAttWaves * (parts - 1) < steps); ++parts) {
    const int64_t rounds = ((int64_t)units * parts + kGroups - 1) / kGroups, cost = rounds * (2 + (steps + kAttWaves * parts - 1) / (kAttWaves * parts));
    if (cost < least) {
      least = cost;
      best = parts;
    }
  }
  return best;
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
      hipLaunchKernelGGL(kern, dim3(parts, units), dim3(kAttThreads), 0, s, a, static_cast<const T*>(Q), group, chosen, count, scale_of(scale), records,
                         parts == 1 ? out : nullptr);
    };
    if (kv.dtype == FC_BF16) d == 128 ? launch(attend_chosen_kernel<uint16_t, 128>, uint16_t{}) : launch(attend_chosen_kernel<uint16_t, 64>, uint16_t{});
    else d == 128 ? launch(attend_chosen_kernel<float, 128>, float{}) : launch(attend_chosen_kernel<float, 64>, float{});
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  ProfileScope ps("chosen_merge_kernel", s);
  const MergeShape m = merge_shape(units, parts, group, d);
  auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(units, m.along), dim3(m.threads), m.lds, s, records, parts, group, m.slots, out); };
  d == 128 ? launch(chosen_merge_kernel<128>) : launch(chosen_merge_kernel<64>);
  return hipGetLastError();
}

size_t attend_shared_workspace_bytes(int P, int B, int L, int H, int group, int d, int dtype) {
  return (size_t)shared_sizes(P, B, L, H, group, d, dtype).total;
}

hipError_t attend_shared_launch(const void* Q, int group, const fc_paged_kv& common, const int32_t* starts, const fc_paged_kv& own, float scale, float* out, void* ws,
                                hipStream_t s) {
  const int P = common.batch, B = own.batch, L = own.layers, H = own.kv_heads, d = own.head_dim;
  const SharedSizes z = shared_sizes(P, B, L, H, group, d, own.dtype);
  float* const records = static_cast<float*>(ws);
  float* const own_records = records + z.common * record_floats(z.record_rows, d);
  // ... for as many waves as are resident together, and where units are more, parts of four steps by what the tables reach: sequences hold different
  // numbers of rows, which shorter parts even out (432 units of up to 700 fp32 rows in 4 parts 94 us, in 11 89; 32 units of up to 256 bf16 rows in 2 parts 16.2,
  // in 10 13.2)
  const int step_rows = own.dtype == FC_BF16 ? 32 : 16;
  const int64_t units = (int64_t)B * L * H, reach = (int64_t)own.max_pages * own.page_size / step_rows;
  const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(z.own_parts, std::max(std::min(2048 / units, reach), reach / 4)));
  // (no more workgroups for prompts than the shortest pieces of all that the tables reach)
  const int64_t pieces = ((int64_t)common.max_pages * common.page_size + kLeastSteps * step_rows - 1) / (kLeastSteps * step_rows);
  const int64_t common_groups = P ? std::min<int64_t>(z.common, (int64_t)L * H * most_tiles(P, B, group) * pieces) : 0;
  SharedArgs a{paged_args(common), paged_args(own), starts, group, z.groups, (int)z.common, (int)common_groups, z.record_rows, parts, step_rows, scale_of(scale), records, own_records,
               reinterpret_cast<int2*>(own_records + z.own * record_floats(group, d)), out};
  {
    ProfileScope ps("attend_shared_kernel", s);
    const int64_t groups = common_groups + (units * parts + kAttWaves - 1) / kAttWaves;
    auto launch = [&](auto kern, size_t lds, auto type) {
      typedef decltype(type) T;
      hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kAttThreads), lds, s, a, static_cast<const T*>(Q));
    };
    if (own.dtype == FC_BF16)
      d == 128 ? launch(attend_shared_kernel<uint16_t, 128>, shared_lds_bytes<uint16_t, 128>(), uint16_t{})
               : launch(attend_shared_kernel<uint16_t, 64>, shared_lds_bytes<uint16_t, 64>(), uint16_t{});
    else
      d == 128 ? launch(attend_shared_kernel<float, 128>, shared_lds_bytes<float, 128>(), float{})
               : launch(attend_shared_kernel<float, 64>, shared_lds_bytes<float, 64>(), float{});
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ProfileScope ps("shared_merge_kernel", s);
  const MergeShape m = merge_shape(B * L * H, std::max(P ? z.groups / (L * H) : 1, parts), group, d);
  auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(B * L * H, m.along), dim3(m.threads), m.lds, s, a, m.slots); };
  d == 128 ? launch(shared_merge_kernel<128>) : launch(shared_merge_kernel<64>);
  return hipGetLastError();
}

}  // namespace fc
