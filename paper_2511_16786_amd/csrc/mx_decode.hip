// Decode-step attention over the 4-bit paged cache (one new token a sequence):  out = softmax(q K^T * scale) V  over the first `rows` rows of each
// (layer, KV head); query head g reads KV head g / G.
//
// Bound by memory: every row of K and V is read once, 17 D / 16 bytes.  The matrix cores do both products on bf16 operands, which hold an
// e2m1 value times a power of two exactly; fp32 is kept in the sums and the softmax.
//   scores:  A = K rows (row c16 of a tile of 16 slots, D / 4 neighbouring columns of it for each g4), B = queries (head c16, the same
//            columns; fp32 queries as three bf16 terms, 24 bits), so that a lane has the scores of rows 4 g4 + i and head c16
//   output:  A = probabilities (head c16, rows 4 g4 + i of both tiles of a step: as the scores come out), B = V (the same rows, column
//            D / 16 c16 + t for output tile t).  Probabilities are three bf16 terms, 24 bits: with two the result is off by 1e-6.
// Up to eight heads leave half of the sixteen lanes, columns and rows of these products idle (FOLD): lanes 8 .. 15 then have the second tile's
// scores, half the exponentials and splits each; rows 8 .. 15 of A are the probabilities' second term, two products in place of three, added up
// once at the end; and columns 8 .. 15 of B an fp32 query's second term.  (28 layers that keep 29 500 of 32 768 rows, 7 heads: bf16 88.5 us / 84.5
// so, the second tile's scores alone 87; 6554 rows fp32 30.5 / 28.6, 64 columns 21.4 / 20.5.)
//
// A workgroup has a piece of one unit, in steps of 32 rows of which each of its waves takes a quarter; the waves merge in LDS, the pieces of a
// unit in a second kernel.  Budgets are on the device, so that every wave finds out by itself how many pieces the layers make and which of
// them is its own.  A unit's piece is never shared with another unit's: equal runs of steps over all units at once, whichever they
// belong to, leave no workgroup waiting, but most of them then have two units, load twice from nothing and write two pieces (512 units
// of 3600 rows 58 us, a workgroup each 48; 448 of 300 rows 18.6 and 9.8).  A single kernel whose last workgroup merges would need a
// release of the L2 by each of them: 155 us instead of 30.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "fc_common.h"
#include "mx.h"

namespace fc {

namespace {

constexpr int kMxdThreads = 256, kMxdWaves = 4;
constexpr int kAhead = 2;              // steps of rows under way in a wave
constexpr int kLeastSteps = 4;         // of a piece
// Waves that a SIMD holds by the registers of each form, and as many workgroups a compute unit, which all are resident together.  (With one step
// under way and four workgroups in place of three: 28 layers of 4 heads that keep 6554 rows 29.2 us, 28.2 so; four of the folded form 32.6 and 27.4,
// three of fp32's in place of two 30.9 and 28.6.)
constexpr int waves_held(int d, int terms) { return d == 64 ? 4 : terms > 1 ? 2 : 3; }
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
  int groups;                    // pieces that the launch aims at
  bool whole;                    // a workgroup for each unit
  float scale_log2e, limit_scale;        // of scores, above 0; its reciprocal
  bool negate;                           // the scale is negative: queries change their signs
  float* pieces;
  int2* span;                    // first piece of each unit and how many it has
  float* out;
};

// a part of a unit, or a workgroup's piece: weighted V [G][d], references [G], sums [G]
__host__ __device__ inline size_t piece_floats(int G, int d) { return ((size_t)G * (d + 2) + 3) / 4 * 4; }

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
// Of each sixteen lanes the upper eight, or the lower eight, take b's from the lane eight below, or above; the others keep a.
__device__ __forceinline__ uint32_t upper_half(uint32_t a, uint32_t b) { return (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)b, 0x118, 0xF, 0xC, false); }
__device__ __forceinline__ uint32_t lower_half(uint32_t a, uint32_t b) { return (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)b, 0x108, 0xF, 0x3, false); }
// the lower eight's own, and zeros
__device__ __forceinline__ uint32_t lower_half_alone(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xE4, 0xF, 0x3, false); }
__device__ __forceinline__ float other_half(float v) {     // eight lanes further round
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x128, 0xF, 0xF, false));
}
// in a scalar register
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
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

// Past the last-level cache: a step reads each row once, and before the next step a model's weights have been through it.  (Three caches in turn,
// claiming it / not: 200 MB 58 / 54 us, 449 MB 96 / 86, 100 MB the same; one cache again and again, 200 MB 48 / 51.)
template <typename V> __device__ __forceinline__ V load_past(const void* p) { return __builtin_nontemporal_load(static_cast<const V*>(p)); }

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

__device__ __forceinline__ int rows_within(const MxdArgs& a, int rows) {
  return min(min(max(rows, 0), kMostRows), (int)min((int64_t)kMostRows, (int64_t)a.max_pages * a.page_tiles * 16));
}
__device__ __forceinline__ int rows_at(const MxdArgs& a, int bl) { return rows_within(a, a.rows[bl]); }
__device__ __forceinline__ int steps_of(int rows) { return (rows + 31) >> 5; }

// Steps of a piece, for a launch of `all` steps: as many pieces as stay resident together, a part of one more for each unit among them; where
// there are more units than that, pieces twice as long as a unit on average, so that only the longest are cut.
__host__ __device__ inline int most_pieces(int groups, int units) { return groups > units + units / 2 ? groups : units + units / 2; }
__device__ __forceinline__ int steps_a_piece(int all, int groups, int units) {
  const int pieces = max(1, most_pieces(groups, units) - units);
  return max(kLeastSteps, all / pieces + (all % pieces != 0));
}

// A step's codes and scales of one lane.
template <int D> struct Step {
  static constexpr int kWords = D / 32;
  uint32_t k[2][kWords], v[2][kWords];
  uint32_t ks[2], vs[2];
  int gone[2], missing;          // negative: the tile, either tile has no page
};

template <int D, int QTERMS, bool FOLD>
__global__ __launch_bounds__(kMxdThreads, waves_held(D, QTERMS)) void mx_decode_partial_kernel(MxdArgs a) {
  typedef MxTile<D> Tile;
  constexpr int KW = D / 32;             // dwords of K and of V a lane and tile; 32-column products of a score
  constexpr int VT = D / 16;             // output tiles
  extern __shared__ __align__(16) float parts[];       // [kMxdWaves][piece_floats]
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), c16 = lane & 15, g4 = lane >> 4, G = a.G;
  const int w = blockIdx.x, part_floats = (int)piece_floats(G, D);
  int bl = 0, h = 0, rows = 0, piece = 0, pieces = 1;    // layer, head and rows of the unit; which of its pieces
  if (a.whole) {
    bl = w / a.H;
    h = w - bl * a.H;
    rows = uniform(rows_at(a, bl));
  } else {
    // steps and pieces of all layers, each head of which has as many (all units' steps fit 31 bits: mx_decode_reach)
    constexpr int kChunks = 8;           // 64 layers each, whose rows are under way together and stay in registers
    int held[kChunks];
    auto load_rows = [&](int base) {
#pragma unroll
      for (int j = 0; j < kChunks; ++j) held[j] = 0;
      auto load = [&](int j) { held[j] = a.rows[min(base + 64 * j + lane, a.layers - 1)]; };
      load(0);
      if (a.layers > base + 64) { load(1); load(2); load(3); }                 // (no use of one before the next)
      if (a.layers > base + 256) { load(4); load(5); load(6); load(7); }
#pragma unroll
      for (int j = 0; j < kChunks; ++j) held[j] = base + 64 * j + lane < a.layers ? rows_within(a, held[j]) : 0;
    };
    int total = 0;
    for (int base = 0; base < a.layers; base += 64 * kChunks) {
      load_rows(base);
      int sum = 0;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) sum += steps_of(held[j]);
      total += __builtin_amdgcn_readlane(wave_scan(sum), 63);
    }
    const int each = steps_a_piece(total * a.H, a.groups, a.layers * a.H), in_heads = w / a.H;
    int before = 0;
    bool found = false;
    for (int base = 0; base < a.layers && !found; base += 64 * kChunks) {
      if (a.layers > 64 * kChunks) load_rows(base);
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        if (!found && base + 64 * j < a.layers) {
          const int mine = (steps_of(held[j]) + each - 1) / each;
          const int upto = wave_scan(mine), chunk = __builtin_amdgcn_readlane(upto, 63);
          if (before + chunk > in_heads) {
            found = true;
            const int owner = __builtin_ctzll(__ballot(before + upto > in_heads));
            bl = base + 64 * j + owner;
            rows = __builtin_amdgcn_readlane(held[j], owner);
            pieces = __builtin_amdgcn_readlane(mine, owner);
            const int place = w - (before + __builtin_amdgcn_readlane(upto, owner) - pieces) * a.H;
            h = place / pieces;
            piece = place - h * pieces;
          }
          before += chunk;
        }
      }
    }
    if (!found) return;
  }
  const int unit = bl * a.H + h, steps = steps_of(rows);
  const int share = steps / pieces, over = steps - share * pieces, first = piece * share + min(piece, over), n = share + (piece < over ? 1 : 0);
  const int s0 = first + n * wave / kMxdWaves, s1 = first + n * (wave + 1) / kMxdWaves;
  if (!a.whole && piece == 0 && tid == 0) a.span[unit] = int2{w, pieces};
  const int32_t* const entries = a.table + (int64_t)unit * a.max_pages;
  const int last_tile = min((rows + 15) >> 4, 2 * s1);
  const uint32_t k_off = Tile::k_code(c16, g4 * (D / 8)), v_off = Tile::v_code(4 * g4, c16);
  const uint32_t ks_off = Tile::k_scale(c16, g4 * (D / 4) / 32), vs_off = Tile::v_scale(4 * g4, c16 * (D / 16) / 32);
  // The tile to be loaded next, its page and its place there.  Lane i holds the first tile of page page0 + i of the table (-1: it has none), so
  // that no load waits for a lookup.
  int tile = 2 * s0, in_page, page;    // (page: counted from page0)
  int page0 = uniform(tile / a.page_tiles);
  in_page = tile - page0 * a.page_tiles;
  page = 0;
  auto lookup = [&]() -> int32_t {
    const int32_t id = entries[min(page0 + lane, a.max_pages - 1)];
    return id >= 0 && id < a.num_pages ? id * a.page_tiles : -1;
  };
  int32_t entry = lookup();
  // queries: head c16 (zeros beyond G), columns D / 4 g4 + 8 i .. + 7; on the way as the page numbers are, and made operands of behind the first tiles
  constexpr int kQ = FOLD && QTERMS == 3 ? 2 : QTERMS;
  typedef std::conditional_t<QTERMS == 1, uint16_t, float> Query;
  const int head = FOLD && QTERMS == 3 ? c16 & 7 : c16;
  u32x4 raw[KW][sizeof(Query) / 2];
  {
    const Query* const from = static_cast<const Query*>(a.Q) + ((size_t)unit * G + min(head, G - 1)) * D + g4 * (D / 4);
#pragma unroll
    for (int i = 0; i < KW; ++i)
#pragma unroll
      for (int j = 0; j < (int)sizeof(Query) / 2; ++j) raw[i][j] = reinterpret_cast<const u32x4*>(from + 8 * i)[j];
  }

  // reference of head c16 (the same in its four lanes), in log2 units, and this lane's sum; the product from which on the reference is moved
  float m = -INFINITY, ref = 0.f, ls = 0.f, limit = -INFINITY;
  float4v out[VT];
#pragma unroll
  for (int t = 0; t < VT; ++t) out[t] = float4v{0.f, 0.f, 0.f, 0.f};

  auto load_step = [&](Step<D>& x) {
    x.missing = 0;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int first_tile = __builtin_amdgcn_readlane(entry, page);
      x.missing |= first_tile;                           // (negative if either is)
      x.gone[tt] = first_tile;
      // (the cache's first tiles in place of those that have no page: masked)
      const uint8_t* const at_tile = a.pages + (uint64_t)(uint32_t)(max(first_tile, 0) + in_page) * Tile::kBytes;
      if (tile + 1 < last_tile) {                        // (behind the last tile it comes again)
        ++tile;
        if (++in_page == a.page_tiles) {
          in_page = 0;
          if (++page == 64) {
            page0 += 64;
            page = 0;
            entry = lookup();
            asm volatile("" : "+v"(entry));              // (waited for here, not before every use)
          }
        }
      }
      if constexpr (D == 128) {
        const u32x4 k = load_past<u32x4>(at_tile + k_off), v = load_past<u32x4>(at_tile + v_off);
#pragma unroll
        for (int i = 0; i < KW; ++i) { x.k[tt][i] = k[i]; x.v[tt][i] = v[i]; }
      } else {
        const u32x2 k = load_past<u32x2>(at_tile + k_off), v = load_past<u32x2>(at_tile + v_off);
#pragma unroll
        for (int i = 0; i < KW; ++i) { x.k[tt][i] = k[i]; x.v[tt][i] = v[i]; }
      }
      x.ks[tt] = load_past<uint8_t>(at_tile + ks_off);
      x.vs[tt] = load_past<uint32_t>(at_tile + vs_off);
    }
  };
  Step<D> x[kAhead];                   // (of a wave without steps: what is at that place, or the cache's first tile)
#pragma unroll
  for (int i = 0; i < kAhead; ++i) load_step(x[i]);
  uint32_t q[kQ][KW][4];
#pragma unroll
  for (int i = 0; i < KW; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t there = head < G ? ~0u : 0u;
      if constexpr (QTERMS == 1) {
        q[0][i][j] = (raw[i][0][j] ^ (a.negate ? 0x80008000u : 0u)) & there;
      } else {
        const uint32_t flip = a.negate ? 0x80000000u : 0u;
        const uint32_t pair0 = raw[i][j / 2][2 * (j % 2)], pair1 = raw[i][j / 2][2 * (j % 2) + 1];
        float x0 = __uint_as_float((pair0 ^ flip) & there), x1 = __uint_as_float((pair1 ^ flip) & there);
        uint32_t term[QTERMS];
#pragma unroll
        for (int t = 0; t < QTERMS; ++t) {
          // (the first two cut off, so that nothing overflows to infinity; the last to nearest)
          const uint32_t u0 = __float_as_uint(x0), u1 = __float_as_uint(x1);
          if (t == QTERMS - 1) {
            term[t] = pack_bf16(x0, x1);
          } else {
            term[t] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
            x0 -= __uint_as_float(u0 & 0xFFFF0000u);
            x1 -= __uint_as_float(u1 & 0xFFFF0000u);
          }
        }
        if constexpr (FOLD) {
          q[0][i][j] = c16 < 8 ? term[0] : term[1];
          q[1][i][j] = c16 < 8 ? term[2] : 0u;
        } else {
#pragma unroll
          for (int t = 0; t < QTERMS; ++t) q[t][i][j] = term[t];
        }
      }
    }
  auto work = [&](int st, Step<D>& x) {
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
        for (int t = kQ - 1; t >= 0; --t)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, as_bf16x8(q[t][i][0], q[t][i][1], q[t][i][2], q[t][i][3]), acc, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[tt][i] = kQ < QTERMS ? acc[i] + other_half(acc[i]) : acc[i];
    }
    const int rb = 32 * st + 4 * g4;
    if (x.missing < 0 || 32 * st + 32 > rows) {              // (the same for the wave)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (rb + 16 * tt + i >= rows || x.gone[tt] < 0) {
            sc[tt][i] = -INFINITY;
            x.vs[tt] = (x.vs[tt] & ~(0xFFu << (8 * i))) | (127u << (8 * i));     // (no NaN from a row that is not there)
          }
    }
    constexpr int kTiles = FOLD ? 1 : 2;
    if constexpr (FOLD) {
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[0][i] = __uint_as_float(upper_half(__float_as_uint(sc[0][i]), __float_as_uint(sc[1][i])));
    }
    float mx = fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3]));
    if constexpr (!FOLD) mx = fmaxf(mx, fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
    if (__ballot(mx > limit)) {
      if constexpr (FOLD) mx = fmaxf(mx, __shfl_xor(mx, 8, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float m_new = fmaxf(m, mx * a.scale_log2e), alpha = m_new > m ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
      m = m_new;
      limit = (m + kSlack) * a.limit_scale;
      ref = m > -INFINITY ? m : 0.f;
      ls *= alpha;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a_i = __shfl(alpha, 4 * g4 + i, 64);
#pragma unroll
        for (int t = 0; t < VT; ++t) out[t][i] *= a_i;
      }
    }
    uint32_t hi[4], mid[4], lo[4];
#pragma unroll
    for (int tt = 0; tt < kTiles; ++tt)
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        float p0 = __builtin_amdgcn_exp2f(fmaf(sc[tt][i], a.scale_log2e, -ref)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[tt][i + 1], a.scale_log2e, -ref));
        ls += p0;
        ls += p1;
        const int w2 = 2 * tt + i / 2;
        hi[w2] = __builtin_amdgcn_perm(__float_as_uint(p1), __float_as_uint(p0), 0x07060302u);
        p0 = less_low(p0, hi[w2]);
        p1 = less_high(p1, hi[w2]);
        mid[w2] = __builtin_amdgcn_perm(__float_as_uint(p1), __float_as_uint(p0), 0x07060302u);
        lo[w2] = pack_bf16(less_low(p0, mid[w2]), less_high(p1, mid[w2]));
      }
    constexpr int kP = FOLD ? 2 : 3;
    bf16x8 terms[kP];
    if constexpr (FOLD) {
      terms[0] = as_bf16x8(upper_half(hi[0], mid[0]), upper_half(hi[1], mid[1]), lower_half(mid[0], hi[0]), lower_half(mid[1], hi[1]));
      terms[1] = as_bf16x8(lower_half_alone(lo[0]), lower_half_alone(lo[1]), lower_half(0u, lo[0]), lower_half(0u, lo[1]));
    } else {
      terms[0] = as_bf16x8(hi[0], hi[1], hi[2], hi[3]);
      terms[1] = as_bf16x8(mid[0], mid[1], mid[2], mid[3]);
      terms[kP - 1] = as_bf16x8(lo[0], lo[1], lo[2], lo[3]);
    }
    float unit_v[2][4];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      // (the conversion looks at the exponent alone)
      unit_v[tt][0] = __uint_as_float(x.vs[tt] << 23);
      unit_v[tt][1] = __uint_as_float(x.vs[tt] << 15);
      unit_v[tt][2] = __uint_as_float(x.vs[tt] << 7);
      unit_v[tt][3] = __uint_as_float(x.vs[tt] >> 1);
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
#pragma unroll
        for (int t = 0; t < kP; ++t) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(terms[t], vb, acc, 0, 0, 0);
        out[2 * c + o] = acc;
      }
    };
    tiles_of(std::integral_constant<int, 0>{});
    tiles_of(std::integral_constant<int, 1>{});
    if constexpr (D == 128) {
      tiles_of(std::integral_constant<int, 2>{});
      tiles_of(std::integral_constant<int, 3>{});
    }
  };
  // kAhead steps under way; a step's registers are filled again in place.  (Loads without conditions, behind the wave's last step of that
  // step's last tile again: where a load may or may not have been made the next wait is for all of them.)
  for (int st = s0; st < s1; st += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (st + i < s1) work(st + i, x[i]);
      load_step(x[i]);
    }
  }

  if constexpr (FOLD) {                                    // heads' second terms, eight rows below
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t u = __float_as_uint(out[t][i]);
        const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        out[t][i] = __uint_as_float(both[0]) + __uint_as_float(both[1]);
      }
  }
  // the lanes of a head add their sums
  if constexpr (FOLD) ls += __shfl_xor(ls, 8, 64);
  ls += __shfl_xor(ls, 16, 64);
  ls += __shfl_xor(ls, 32, 64);
  float* const mine = parts + wave * part_floats;
  if (g4 == 0 && c16 < G) { mine[G * D + c16] = m; mine[G * D + G + c16] = ls; }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (4 * g4 + i < G)
#pragma unroll
      for (int t = 0; t < VT; t += 4)
        *reinterpret_cast<float4v*>(mine + (4 * g4 + i) * D + VT * c16 + t) = float4v{out[t][i], out[t + 1][i], out[t + 2][i], out[t + 3][i]};
  __syncthreads();

  // the waves' parts, in their order
  float* const record = a.pieces + (size_t)w * part_floats;
  for (int item = tid; item < G * D / 4; item += kMxdThreads) {         // four columns
    const int g = item / (D / 4);
    float m[kMxdWaves], l[kMxdWaves], top = -INFINITY;
    float4v o[kMxdWaves];
#pragma unroll
    for (int v = 0; v < kMxdWaves; ++v) {
      const float* const one = parts + v * part_floats;
      m[v] = one[G * D + g];
      l[v] = one[G * D + G + g];
      o[v] = *reinterpret_cast<const float4v*>(one + 4 * item);
      top = fmaxf(top, m[v]);
    }
    const float ref = top > -INFINITY ? top : 0.f;         // (none has a finite score: zeros, or NaN)
    float4v acc = {0.f, 0.f, 0.f, 0.f};
    float lt = 0.f;
#pragma unroll
    for (int v = 0; v < kMxdWaves; ++v) {
      const float wt = __builtin_amdgcn_exp2f(m[v] - ref);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(o[v][i], wt, acc[i]);
      lt = fmaf(l[v], wt, lt);
    }
    if (pieces == 1) {
      const float part = lt == 0.f ? 0.f : 1.f / lt;       // (1 and more, if there is a row at all)
      *reinterpret_cast<float4v*>(a.out + (size_t)unit * G * D + 4 * item) = acc * part;
    } else {
      *reinterpret_cast<float4v*>(record + 4 * item) = acc;
      if (4 * item % D == 0) { record[G * D + g] = top; record[G * D + G + g] = lt; }
    }
  }
}

// out[unit][g][:] of units of several pieces, and zeros for those without rows.  grid = (slices of the heads, units); `sets` groups of d threads have
// kAtOnce pieces each at a time, all of them under way together.
constexpr int kAtOnce = 8;
__global__ void mx_decode_merge_kernel(MxdArgs a, int d, int heads) {
  extern __shared__ float lds[];                           // [sets][3][d]: largest reference, sum, weighted sum
  const int unit = blockIdx.y, dim = threadIdx.x % d, set = threadIdx.x / d, sets = blockDim.x / d, G = a.G;
  const int g0 = blockIdx.x * heads, g1 = min(G, g0 + heads);
  const int2 span = a.span[unit];
  if (rows_at(a, unit / a.H) == 0) {
    for (int g = g0 + set; g < g1; g += sets) a.out[((size_t)unit * G + g) * d + dim] = 0.f;
    return;
  }
  if (span.y <= 1) return;                                 // (written by its workgroup)
  const size_t stride = piece_floats(G, d);
  // (within the workspace whatever it holds)
  const int most = most_pieces(a.groups, a.layers * a.H), first = min(max(span.x, 0), most - 1), n = min(span.y, most - first);
  const float* const base = a.pieces + (size_t)first * stride;
  for (int g = g0; g < g1; ++g) {
    float top = -INFINITY, acc = 0.f, lt = 0.f;
    for (int i0 = set * kAtOnce; i0 < n; i0 += sets * kAtOnce) {
      float m[kAtOnce], l[kAtOnce], o[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const float* const piece = base + (size_t)min(i0 + i, n - 1) * stride;
        const bool have = i0 + i < n;
        m[i] = have ? piece[G * d + g] : -INFINITY;
        l[i] = have ? piece[G * d + G + g] : 0.f;
        o[i] = have ? piece[g * d + dim] : 0.f;
      }
      float up = top;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) up = fmaxf(up, m[i]);
      const float ref = up > -INFINITY ? up : 0.f, before = __builtin_amdgcn_exp2f(top - ref);
      acc *= before;
      lt *= before;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const float wt = __builtin_amdgcn_exp2f(m[i] - ref);
        acc = fmaf(o[i], wt, acc);
        lt = fmaf(l[i], wt, lt);
      }
      top = up;
    }
    if (sets > 1) {
      float* const mine = lds + (size_t)set * 3 * d + dim;
      if (g > g0) __syncthreads();    // (the head before is still being read)
      mine[0] = top;
      mine[d] = lt;
      mine[2 * d] = acc;
      __syncthreads();
      if (set == 0) {
        float up = top;
        for (int v = 1; v < sets; ++v) up = fmaxf(up, mine[v * 3 * d]);
        const float ref = up > -INFINITY ? up : 0.f;
        acc = lt = 0.f;
        for (int v = 0; v < sets; ++v) {
          const float wt = __builtin_amdgcn_exp2f(mine[v * 3 * d] - ref);
          acc = fmaf(mine[(v * 3 + 2) * d], wt, acc);
          lt = fmaf(mine[(v * 3 + 1) * d], wt, lt);
        }
      }
    }
    if (set == 0) a.out[((size_t)unit * G + g) * d + dim] = lt == 0.f ? 0.f : acc / lt;
  }
}

}  // namespace

bool mx_decode_supported(int group, int d) { return (d == 64 || d == 128) && group >= 1 && group <= 16; }

// Whether the steps of the rows that the tables reach are counted in 31 bits.
bool mx_decode_reach(int64_t units, int64_t max_pages, int64_t page_size) {
  return units * ((std::min<int64_t>(kMostRows, max_pages * page_size) + 31) / 32) < (1ll << 31);
}

constexpr int groups_held(int d, int dtype) { return 256 * waves_held(d, dtype == FC_BF16 ? 1 : 3); }
static size_t pieces_bytes(int units, int group, int d) {               // (bf16's: they hold more)
  return ((size_t)most_pieces(groups_held(d, FC_BF16), units) * piece_floats(group, d) * sizeof(float) + 15) / 16 * 16;
}
size_t mx_decode_workspace_bytes(int units, int group, int d) {
  return units == 0 ? 0 : pieces_bytes(units, group, d) + (size_t)units * sizeof(int2);
}

hipError_t mx_decode_launch(const void* Q, const void* pages, const int32_t* table, int page_size, int max_pages, int64_t num_pages,
                            int B, int L, int H, int group, int d, int dtype, const int32_t* rows, float scale, float* out, void* ws,
                            hipStream_t s) {
  const int units = B * L * H;
  // Tables that reach no further than kWholeSteps, and more units than four rounds of workgroups: one for each unit, and no merge.  (4 units of
  // 115, 460 and 921 rows 12.6, 12.0, 12.0 us with pieces of four steps, 9.8, 9.5, 10.0 whole; 64 units of 921 13.2 and 10.7, of 1843 15.2 and
  // 15.7; 4 of 1843 12.3 and 15.2; 3584 of 1500 177 and 151.  1792 of 1500 are 83 and 80, but a layer far longer than the others would keep a
  // single workgroup busy.  From 4 * groups units on it does so here: a layer of 131 072 rows among 895 of 100, four heads each, takes 640 us.)
  constexpr int64_t kWholeSteps = 32;
  const int64_t reach = ((int64_t)max_pages * page_size + 31) / 32;
  const int groups = groups_held(d, dtype);
  const bool whole = reach <= kWholeSteps || units >= 4 * groups;
  // (a scale of zero: the smallest there is, which leaves all scores as alike as they can be told)
  const float positive = std::max(std::fabs(scale) * 1.4426950408889634f, 1.17549435e-38f);
  const MxdArgs a{Q, static_cast<const uint8_t*>(pages), rows, table, B * L, H, group, page_size / 16, max_pages, num_pages, groups, whole,
                  positive, std::min(1.f / positive, 3.4e38f), scale < 0.f, static_cast<float*>(ws),
                  reinterpret_cast<int2*>(static_cast<char*>(ws) + pieces_bytes(units, group, d)), out};
  {
    ProfileScope ps("mx_decode_partial_kernel", s);
    // no more workgroups than the rows that the tables have room for make
    const int grid = whole ? units : (int)std::min<int64_t>(most_pieces(groups, units), units * ((reach + kLeastSteps - 1) / kLeastSteps));
    const size_t lds = kMxdWaves * piece_floats(group, d) * sizeof(float);
    auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(grid), dim3(kMxdThreads), lds, s, a); };
    auto folded = [&](auto fold) {
      constexpr bool kFold = decltype(fold)::value;
      if (dtype == FC_BF16) d == 128 ? launch(mx_decode_partial_kernel<128, 1, kFold>) : launch(mx_decode_partial_kernel<64, 1, kFold>);
      else d == 128 ? launch(mx_decode_partial_kernel<128, 3, kFold>) : launch(mx_decode_partial_kernel<64, 3, kFold>);
    };
    group <= 8 ? folded(std::true_type{}) : folded(std::false_type{});
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || whole) return e;
  // sets for the pieces of a unit if all units are alike; a workgroup for each head where that is no more than a few thousand
  const int sets = std::min(1024 / d, std::max(1, (groups / units + kAtOnce - 1) / kAtOnce));
  const int heads = std::min(group, std::max(1, units * group / 2048)), slices = (group + heads - 1) / heads;
  ProfileScope ps("mx_decode_merge_kernel", s);
  hipLaunchKernelGGL(mx_decode_merge_kernel, dim3(slices, units), dim3(sets * d), (size_t)sets * 3 * d * sizeof(float), s, a, d, heads);
  return hipGetLastError();
}

}  // namespace fc
