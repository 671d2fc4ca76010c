// Decode-step attention over the 4-bit paged cache (one new token a sequence):  out = softmax(q K^T * scale) V  over the first `rows` rows of each
// (layer, KV head); query head g reads KV head g / G.
//
// Bound by memory: every row of K and V is read once, 17 D / 16 bytes.  The matrix cores do both products on bf16 operands, which hold an
// e2m1 value times a power of two exactly; fp32 is kept in the sums and the softmax.
//   scores:  A = K rows (row c16 of a tile of 16 slots, D / 4 neighbouring columns of it for each g4), B = queries (head c16, the same
//            columns; fp32 queries as three bf16 terms, 24 bits), so that a lane has the scores of rows 4 g4 + i and head c16
//   output:  A = probabilities (head c16, rows 4 g4 + i of both tiles of a step: as the scores come out), B = V (the same rows, column
//            D / 16 c16 + t for output tile t).  Probabilities are three bf16 terms, 24 bits: with two the result is off by 1e-6.
//
// Work is shared out by steps of 32 rows over all units at once: workgroup w has steps S w / W .. S (w + 1) / W of the launch's S, whichever
// units they belong to, so that no workgroup waits for a long layer.  Budgets are on the device; every wave sums them up by itself.  A unit
// that lies in one workgroup is finished there, the others' pieces (running maximum, sum, weighted V) are merged by a second kernel: piece
// w + u of the workspace, no two alike since both only grow along the steps.
#include <algorithm>
#include <type_traits>

#include "fc_common.h"
#include "mx.h"

namespace fc {

namespace {

constexpr int kMxdThreads = 256, kMxdWaves = 4;
constexpr int kMxdGroups = 512;        // workgroups of a launch, two a compute unit
constexpr int kMostRows = (1 << 25) - 1;
constexpr float kSlack = 16.f;         // how far scores (in log2) may exceed the running reference before it is moved

typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float float2v __attribute__((ext_vector_type(2)));

struct MxdArgs {
  const void* Q;
  const uint8_t* pages;
  const int32_t* rows;           // [B * L]
  const int32_t* table;          // [B * L * H][max_pages]
  int layers, H, G;              // (layers of all sequences)
  int page_tiles, max_pages;
  int64_t num_pages;
  int groups;                    // workgroups of the launch
  float scale_log2e;
  float* pieces;
  int2* span;                    // first and last workgroup of each unit
  float* out;
};

__host__ __device__ inline size_t piece_floats(int G, int d) { return (size_t)G * (d + 2); }

__device__ __forceinline__ bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8, (u32x4{a, b, c, d}));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {        // to nearest
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{a, b}), bf16x2));
}
template <int BYTE> __device__ __forceinline__ uint32_t two_values(uint32_t code, float unit) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, unit, BYTE));
}
__device__ __forceinline__ void eight_values(uint32_t code, float unit, uint32_t (&o)[4]) {
  o[0] = two_values<0>(code, unit);
  o[1] = two_values<1>(code, unit);
  o[2] = two_values<2>(code, unit);
  o[3] = two_values<3>(code, unit);
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ int rows_at(const MxdArgs& a, int bl) {
  return min(min(max(a.rows[bl], 0), kMostRows), (int)min((int64_t)kMostRows, (int64_t)a.max_pages * a.page_tiles * 16));
}
__device__ __forceinline__ int steps_of(int rows) { return (rows + 31) >> 5; }

// A step's codes and scales of one lane.
template <int D> struct Step {
  static constexpr int kWords = D / 32;
  uint32_t k[2][kWords], v[2][kWords];
  uint32_t ks[2], vs[2];
};

template <int D, int QTERMS>
__global__ __launch_bounds__(kMxdThreads, 2) void mx_decode_partial_kernel(MxdArgs a) {
  typedef MxTile<D> Tile;
  constexpr int KW = D / 32;             // dwords of K and of V a lane and tile; 32-column products of a score
  constexpr int VT = D / 16;             // output tiles
  __shared__ float sm_m[kMxdWaves][16], sm_l[kMxdWaves][16];
  __shared__ float sm_o[kMxdWaves][16][D];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), c16 = lane & 15, g4 = lane >> 4, G = a.G;

  // ---- this workgroup's steps, and the unit that they begin in
  const int per = (a.layers + 63) >> 6, first = min(a.layers, lane * per), last = min(a.layers, first + per);
  int64_t mine = 0;
  for (int i = first; i < last; ++i) mine += (int64_t)steps_of(rows_at(a, i)) * a.H;
  int64_t upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up(upto, d, 64);
    if (lane >= d) upto += o;
  }
  const int64_t all = __shfl(upto, 63, 64);
  if (all == 0) return;
  // (four steps a workgroup at least, one for each wave)
  const int64_t groups = min((int64_t)a.groups, (all + 3) >> 2), w = blockIdx.x;
  if (w >= groups) return;
  int64_t at = all * w / groups;
  const int64_t end = all * (w + 1) / groups;
  int bl;                                // layer that step `at` is in
  int64_t begin_of;                      // and `at`'s place in it (beyond 31 bits where heads have many rows)
  {
    const uint64_t behind = __ballot(upto > at);
    const int owner = __builtin_ctzll(behind);
    int64_t before = upto - mine;
    int found = first;
    if (lane == owner)
      for (; found < last; ++found) {
        const int64_t n = (int64_t)steps_of(rows_at(a, found)) * a.H;
        if (before + n > at) break;
        before += n;
      }
    bl = __builtin_amdgcn_readlane(found, owner);
    const uint64_t in = (uint64_t)(at - before);
    begin_of = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(in >> 32), owner) << 32 |
                         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)in, owner));
  }
  int rows = uniform(rows_at(a, bl)), steps = steps_of(rows);
  int h = uniform((int)(begin_of / steps)), s = uniform((int)(begin_of - (int64_t)h * steps));

  // ---- pieces of units, one after another
  while (at < end) {
    const int unit = bl * a.H + h;
    const int n = (int)min((int64_t)(steps - s), end - at), s_end = s + n;
    const int s0 = s + (int)((int64_t)n * wave / kMxdWaves), s1 = s + (int)((int64_t)n * (wave + 1) / kMxdWaves);

    // queries: head c16 (zeros beyond G), columns D / 4 g4 + 8 i .. + 7
    uint32_t q[QTERMS][KW][4];
#pragma unroll
    for (int t = 0; t < QTERMS; ++t)
#pragma unroll
      for (int i = 0; i < KW; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) q[t][i][j] = 0u;
    if (c16 < G && s0 < s1) {
      const size_t at_q = ((size_t)unit * G + c16) * D + g4 * (D / 4);
      if constexpr (QTERMS == 1) {
#pragma unroll
        for (int i = 0; i < KW; ++i) {
          const u32x4 u = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.Q) + at_q + 8 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) q[0][i][j] = u[j];
        }
      } else {
#pragma unroll
        for (int i = 0; i < KW; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2v x = *reinterpret_cast<const float2v*>(static_cast<const float*>(a.Q) + at_q + 8 * i + 2 * j);
            float x0 = x[0], x1 = x[1];
#pragma unroll
            for (int t = 0; t < QTERMS; ++t) {
              // (the first two cut off, so that nothing overflows to infinity; the last to nearest)
              const uint32_t u0 = __float_as_uint(x0), u1 = __float_as_uint(x1);
              if (t == QTERMS - 1) {
                q[t][i][j] = pack_bf16(x0, x1);
              } else {
                q[t][i][j] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
                x0 -= __uint_as_float(u0 & 0xFFFF0000u);
                x1 -= __uint_as_float(u1 & 0xFFFF0000u);
              }
            }
          }
      }
    }

    float m = -INFINITY, ls = 0.f;       // reference of head c16 (the same in its four lanes), and this lane's sum
    float4v out[VT];
#pragma unroll
    for (int t = 0; t < VT; ++t) out[t] = float4v{0.f, 0.f, 0.f, 0.f};

    const int32_t* const entries = a.table + (int64_t)unit * a.max_pages;
    const int tiles = (rows + 15) >> 4;
    // address of a tile (the cache's first one if it has no page: masked)
    auto tile_at = [&](int t, bool& ok) -> const uint8_t* {
      t = min(t, tiles - 1);
      const int p = t / a.page_tiles;
      const int64_t page = entries[p];
      ok = page >= 0 && page < a.num_pages;
      return a.pages + (ok ? page * a.page_tiles + (t - p * a.page_tiles) : 0) * Tile::kBytes;
    };
    const int k_off = Tile::k_code(c16, g4 * (D / 8)), v_off = Tile::v_code(4 * g4, c16);
    const int ks_off = Tile::k_scale(c16, g4 * (D / 4) / 32), vs_off = Tile::v_scale(4 * g4, c16 * (D / 16) / 32);
    auto load_step = [&](int st, Step<D>& x) -> unsigned {
      unsigned ok2 = 0;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        bool ok;
        const uint8_t* tile = tile_at(2 * st + tt, ok);
        ok2 |= (ok ? 1u : 0u) << tt;
        if constexpr (D == 128) {
          const u32x4 k = *reinterpret_cast<const u32x4*>(tile + k_off), v = *reinterpret_cast<const u32x4*>(tile + v_off);
#pragma unroll
          for (int i = 0; i < KW; ++i) { x.k[tt][i] = k[i]; x.v[tt][i] = v[i]; }
        } else {
          const u32x2 k = *reinterpret_cast<const u32x2*>(tile + k_off), v = *reinterpret_cast<const u32x2*>(tile + v_off);
#pragma unroll
          for (int i = 0; i < KW; ++i) { x.k[tt][i] = k[i]; x.v[tt][i] = v[i]; }
        }
        x.ks[tt] = tile[ks_off];
        x.vs[tt] = *reinterpret_cast<const uint32_t*>(tile + vs_off);
      }
      return ok2;
    };
    auto work = [&](int st, unsigned ok2, Step<D>& x) {
      float sc[2][4];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const float unit_k = __uint_as_float(x.ks[tt] << 23);
        float4v acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KW; ++i) {
          uint32_t kv[4];
          eight_values(x.k[tt][i], unit_k, kv);
          const bf16x8 ka = as_bf16x8(kv[0], kv[1], kv[2], kv[3]);
#pragma unroll
          for (int t = QTERMS - 1; t >= 0; --t)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, as_bf16x8(q[t][i][0], q[t][i][1], q[t][i][2], q[t][i][3]), acc, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[tt][i] = acc[i] * a.scale_log2e;
      }
      const int rb = 32 * st + 4 * g4;
      if (ok2 != 3u || 32 * st + 32 > rows) {              // (the same for the wave)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (rb + 16 * tt + i >= rows || !((ok2 >> tt) & 1u)) {
              sc[tt][i] = -INFINITY;
              x.vs[tt] = (x.vs[tt] & ~(0xFFu << (8 * i))) | (127u << (8 * i));     // (no NaN from a row that is not there)
            }
      }
      float mx = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                       fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
      if (__ballot(mx > m + kSlack)) {                     // (-inf + 16: any score at all)
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx), alpha = m_new > m ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
        m = m_new;
        ls *= alpha;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a_i = __shfl(alpha, 4 * g4 + i, 64);
#pragma unroll
          for (int t = 0; t < VT; ++t) out[t][i] *= a_i;
        }
      }
      const float ref = m > -INFINITY ? m : 0.f;
      uint32_t hi[4], mid[4], lo[4];
      float psum = 0.f;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          float p0 = __builtin_amdgcn_exp2f(sc[tt][i] - ref), p1 = __builtin_amdgcn_exp2f(sc[tt][i + 1] - ref);
          psum += p0;
          psum += p1;
          const int w2 = 2 * tt + i / 2;
          uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
          hi[w2] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
          p0 -= __uint_as_float(u0 & 0xFFFF0000u);
          p1 -= __uint_as_float(u1 & 0xFFFF0000u);
          u0 = __float_as_uint(p0);
          u1 = __float_as_uint(p1);
          mid[w2] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
          lo[w2] = pack_bf16(p0 - __uint_as_float(u0 & 0xFFFF0000u), p1 - __uint_as_float(u1 & 0xFFFF0000u));
        }
      ls += psum;
      const bf16x8 ph = as_bf16x8(hi[0], hi[1], hi[2], hi[3]), pm = as_bf16x8(mid[0], mid[1], mid[2], mid[3]),
                   pl = as_bf16x8(lo[0], lo[1], lo[2], lo[3]);
      float unit_v[2][4];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        unit_v[tt][0] = __uint_as_float((x.vs[tt] << 23) & 0x7F800000u);
        unit_v[tt][1] = __uint_as_float((x.vs[tt] << 15) & 0x7F800000u);
        unit_v[tt][2] = __uint_as_float((x.vs[tt] << 7) & 0x7F800000u);
        unit_v[tt][3] = __uint_as_float((x.vs[tt] >> 1) & 0x7F800000u);
      }
      // byte c of a row's D / 32 bytes has the columns of output tiles 2 c and 2 c + 1
      auto tiles_of = [&](auto byte) {
        constexpr int c = decltype(byte)::value;
        uint32_t r[2][4];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (D == 128) r[tt][i] = two_values<c>(x.v[tt][i], unit_v[tt][i]);
            else r[tt][i] = i & 1 ? two_values<c + 2>(x.v[tt][i / 2], unit_v[tt][i]) : two_values<c>(x.v[tt][i / 2], unit_v[tt][i]);
          }
#pragma unroll
        for (int o = 0; o < 2; ++o) {
          const uint32_t sel = o ? 0x07060302u : 0x05040100u;
          const bf16x8 vb = as_bf16x8(__builtin_amdgcn_perm(r[0][1], r[0][0], sel), __builtin_amdgcn_perm(r[0][3], r[0][2], sel),
                                      __builtin_amdgcn_perm(r[1][1], r[1][0], sel), __builtin_amdgcn_perm(r[1][3], r[1][2], sel));
          float4v acc = out[2 * c + o];
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ph, vb, acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pm, vb, acc, 0, 0, 0);
          out[2 * c + o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pl, vb, acc, 0, 0, 0);
        }
      };
      tiles_of(std::integral_constant<int, 0>{});
      tiles_of(std::integral_constant<int, 1>{});
      if constexpr (D == 128) {
        tiles_of(std::integral_constant<int, 2>{});
        tiles_of(std::integral_constant<int, 3>{});
      }
    };
    {
      Step<D> xa, xb;
      unsigned oka = 0, okb = 0;
      if (s0 < s1) oka = load_step(s0, xa);
      for (int st = s0; st < s1; st += 2) {
        if (st + 1 < s1) okb = load_step(st + 1, xb);
        work(st, oka, xa);
        if (st + 1 >= s1) break;
        if (st + 2 < s1) oka = load_step(st + 2, xa);
        work(st + 1, okb, xb);
      }
    }

    // the four lanes of a head add their sums; then the waves merge through LDS in a fixed order
    ls += __shfl_xor(ls, 16, 64);
    ls += __shfl_xor(ls, 32, 64);
    if (g4 == 0) { sm_m[wave][c16] = m; sm_l[wave][c16] = ls; }
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) sm_o[wave][4 * g4 + i][VT * c16 + t] = out[t][i];
    __syncthreads();
    const bool whole = n == steps;
    float* const piece = a.pieces + (size_t)(w + unit) * piece_floats(G, D);
    for (int item = tid; item < G * D; item += kMxdThreads) {
      const int g = item / D, dim = item % D;
      float top = -INFINITY;
#pragma unroll
      for (int v = 0; v < kMxdWaves; ++v) top = fmaxf(top, sm_m[v][g]);
      const float ref = top > -INFINITY ? top : 0.f;       // (none has a finite score: zeros, or NaN)
      float acc = 0.f, lt = 0.f;
#pragma unroll
      for (int v = 0; v < kMxdWaves; ++v) {
        const float wt = __builtin_amdgcn_exp2f(sm_m[v][g] - ref);
        acc = fmaf(sm_o[v][g][dim], wt, acc);
        lt = fmaf(sm_l[v][g], wt, lt);
      }
      if (whole) {
        a.out[((size_t)unit * G + g) * D + dim] = lt == 0.f ? 0.f : acc / lt;
      } else {
        piece[2 * G + (size_t)g * D + dim] = acc;
        if (dim == 0) { piece[g] = top; piece[G + g] = lt; }
      }
    }
    if (tid == 0) {
      if (s == 0) a.span[unit].x = (int)w;
      if (s_end == steps) a.span[unit].y = (int)w;
    }
    // on to the next unit that has rows
    at += n;
    if (at < end) {
      __syncthreads();                                     // (the LDS arrays are still being read)
      s = 0;
      if (++h == a.H) {
        h = 0;
        do {
          ++bl;
          rows = uniform(rows_at(a, bl));
        } while (rows == 0);
        steps = steps_of(rows);
      }
    }
  }
}

// out[unit][g][:] of units that several workgroups had a piece of, and zeros for those without rows.  grid = (G, units), a thread for each
// column and every kMergeSets-th piece.
constexpr int kMergeSets = 4;
__global__ void mx_decode_merge_kernel(MxdArgs a, int d) {
  extern __shared__ float lds[];                           // [kMergeSets][2][d]
  const int g = blockIdx.x, unit = blockIdx.y, dim = threadIdx.x % d, set = threadIdx.x / d, G = a.G;
  float* const out = a.out + ((size_t)unit * G + g) * d;
  if (rows_at(a, unit / a.H) == 0) {
    if (set == 0) out[dim] = 0.f;
    return;
  }
  const int2 span = a.span[unit];
  if (span.x == span.y) return;                            // (written by its workgroup)
  const size_t stride = piece_floats(G, d);
  const float* const base = a.pieces + (size_t)(span.x + unit) * stride;
  const int n = span.y - span.x + 1;
  float top = -INFINITY;
  for (int i = 0; i < n; ++i) top = fmaxf(top, base[i * stride + g]);
  const float ref = top > -INFINITY ? top : 0.f;
  float acc = 0.f, lt = 0.f;
  for (int i = set; i < n; i += kMergeSets) {
    const float* const piece = base + i * stride;
    const float wt = __builtin_amdgcn_exp2f(piece[g] - ref);
    acc = fmaf(piece[2 * G + (size_t)g * d + dim], wt, acc);
    lt = fmaf(piece[G + g], wt, lt);
  }
  lds[(set * 2) * d + dim] = acc;
  lds[(set * 2 + 1) * d + dim] = lt;
  __syncthreads();
  if (set > 0) return;
  for (int v = 1; v < kMergeSets; ++v) {
    acc += lds[(v * 2) * d + dim];
    lt += lds[(v * 2 + 1) * d + dim];
  }
  out[dim] = lt == 0.f ? 0.f : acc / lt;
}

}  // namespace

bool mx_decode_supported(int group, int d) { return (d == 64 || d == 128) && group >= 1 && group <= 16; }

size_t mx_decode_workspace_bytes(int units, int group, int d) {
  return units == 0 ? 0 : ((size_t)(units + kMxdGroups) * piece_floats(group, d) * sizeof(float) + 15) / 16 * 16 + (size_t)units * sizeof(int2);
}

hipError_t mx_decode_launch(const void* Q, const void* pages, const int32_t* table, int page_size, int max_pages, int64_t num_pages,
                            int B, int L, int H, int group, int d, int dtype, const int32_t* rows, float scale, float* out, void* ws,
                            hipStream_t s) {
  const int units = B * L * H;
  // no more workgroups than the rows that tables and pages have room for make
  const int64_t room = std::min((int64_t)units * (((int64_t)max_pages * page_size + 31) / 32), num_pages * (page_size / 16) + units);
  const int groups = (int)std::min<int64_t>(kMxdGroups, (room + 3) / 4);
  float* const pieces = static_cast<float*>(ws);
  int2* const span = reinterpret_cast<int2*>(static_cast<char*>(ws) + ((size_t)(units + kMxdGroups) * piece_floats(group, d) * sizeof(float) + 15) / 16 * 16);
  const MxdArgs a{Q, static_cast<const uint8_t*>(pages), rows, table, B * L, H, group, page_size / 16, max_pages, num_pages, groups,
                  scale * 1.4426950408889634f, pieces, span, out};
  {
    ProfileScope ps("mx_decode_partial_kernel", s);
    auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(groups), dim3(kMxdThreads), 0, s, a); };
    if (dtype == FC_BF16) d == 128 ? launch(mx_decode_partial_kernel<128, 1>) : launch(mx_decode_partial_kernel<64, 1>);
    else d == 128 ? launch(mx_decode_partial_kernel<128, 3>) : launch(mx_decode_partial_kernel<64, 3>);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ProfileScope ps("mx_decode_merge_kernel", s);
  hipLaunchKernelGGL(mx_decode_merge_kernel, dim3(group, units), dim3(kMergeSets * d), (size_t)kMergeSets * 2 * d * sizeof(float), s, a, d);
  return hipGetLastError();
}

}  // namespace fc
