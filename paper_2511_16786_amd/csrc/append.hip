// New tokens' rows into a paged cache: queries and keys turned by their positions (the rotation of rotary.hip), keys and values into the slots of
// their pages, and, where a program ranks pages by their keys' bounds, each touched page's lowest and largest key of every column.
//
// Bound by memory: every element is read and written once, in one launch.  Without bounds, queries, keys and values of a token are heads in a row of
// which the last are copied, as in rotary.hip, up to five heads of a token under way together: 32768 tokens of 28, 4 and 4 heads of 128 bf16 columns (0.61 GB)
// 105 us, 5.8 TB/s (four heads together, the fifth's loads behind the stores of these, 137; with the code for bounds in the same kernel, whose registers leave
// fewer waves, 114).  With bounds a workgroup has a stretch of one KV head's tokens: it stores their keys and keeps the least and largest of what it stores
// (rounded values: rounding keeps the order) until the page changes, so that no page has two writers and no row is read back.  2 x 1003 tokens of 32, 8
// and 8 heads (0.05 GB) 16 us, of which keys and the rest would take 12 each by themselves, both little more than their chains of loads (a wave a stretch in
// place of a workgroup 30); the kernel has the arguments of both kinds, and keeps up to 106 scalar registers in lanes of vector ones.  Of a single token a wave
// has a key: eight sequences' step with bounds 5.4 us.
#include <algorithm>
#include <type_traits>
#include <math.h>

#include "fc_common.h"
#include "rotary.h"

namespace fc {

namespace {

constexpr int kAppThreads = 256, kAppWaves = kAppThreads / 64;
constexpr int kHeadsAtOnce = 5, kMostPairs = 4, kMostAbreast = 8, kMostTurns = 8;
constexpr int kTokensAtOnce = 2;       // of a lane, with bounds
constexpr int kLooked = kAppThreads;   // tokens whose slots a workgroup looks up together

struct NewRows {                 // strides in bytes
  const char* in;
  int64_t sb, st, sh;
  int heads;
};
struct AppendArgs {
  NewRows q, k, v;
  char* q_out;
  int64_t ob, ot, oh;
  char* k_pages;
  char* v_pages;
  char* bounds;
  const int64_t* slots;
  int64_t slots_b, slots_h;      // strides of the slot map
  int64_t num_slots;
  const int32_t* positions;      // [streams][batch * tokens]
  int tokens, rows;              // tokens of a sequence, of all sequences
  int half, chunks, turned;      // pairs; chunks of a head; those that are turned
  int row_bytes;                 // of a head
  int page_size;
  // rows of tokens
  int per_group;                 // tokens of a workgroup
  uint32_t chunks_inverse, abreast_inverse;
  int abreast, turns, across;    // heads of a token side by side; how many of them a thread has; workgroups side by side
  int at_once;                   // of the turns, under way together
  int turning;                   // heads of the first part that are turned; the keys among them unless there are bounds
  // keys with bounds
  int stretches, stretch;        // of a head; tokens of one
  int bound_groups;              // workgroups, the launch's first
  int streams, end0, end1, end2; // first pair behind the first, second and third stream
  float magnitude;
};

__device__ __forceinline__ float as_float(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float as_float(float x) { return x; }
template <typename T> __device__ __forceinline__ T as_type(float x) {      // (of a value that the type has)
  if constexpr (sizeof(T) == 2) return (T)(__float_as_uint(x) >> 16);
  else return x;
}

// A token's positions in all streams.
struct Positions { int32_t at[4]; };
__device__ __forceinline__ Positions positions_of(const AppendArgs& a, int row) {
  Positions p;
  p.at[0] = a.positions[row];
#pragma unroll
  for (int k = 1; k < 4; ++k) p.at[k] = a.streams > 1 && k < a.streams ? a.positions[(int64_t)k * a.rows + row] : 0;
  return p;
}
template <int P> __device__ __forceinline__ void sines_of(const AppendArgs& a, const fc_rotary_plan& plan, const Positions& p, int first, float (&sn)[P], float (&cs)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int pair = first + i;
    int32_t where = p.at[0];
    if (a.streams > 1) where = pair < a.end0 ? where : pair < a.end1 ? p.at[1] : pair < a.end2 ? p.at[2] : p.at[3];
    sine_cosine(turned_by(where, plan.turns[pair]), sn[i], cs[i]);
    sn[i] *= a.magnitude;
    cs[i] *= a.magnitude;
  }
}

// A chunk's pieces, turned.
template <typename T, int P, bool INTERLEAVED, int PIECES, int PIECE>
__device__ __forceinline__ void turn(Vec<T, PIECE> (&v)[PIECES], const float (&sn)[P], const float (&cs)[P]) {
  float x[PIECES][PIECE], y[PIECES][PIECE];
#pragma unroll
  for (int j = 0; j < PIECES; ++j) widen<T, PIECE>(v[j], x[j]);
#pragma unroll
  for (int k = 0; k < P; ++k) {
    constexpr int j = INTERLEAVED ? 0 : 1;
    const int c0 = INTERLEAVED ? 2 * k : k, c1 = INTERLEAVED ? 2 * k + 1 : k;
    y[0][c0] = fmaf(x[0][c0], cs[k], -(x[j][c1] * sn[k]));  // (fused by hand: the same roundings in all forms of the kernel)
    y[j][c1] = fmaf(x[0][c0], sn[k], x[j][c1] * cs[k]);
  }
#pragma unroll
  for (int j = 0; j < PIECES; ++j) v[j] = narrow<T, PIECE>(y[j]);
}

// Bytes of a chunk's first piece from the head's begin on, and from it to the second.
template <typename T, int P, int PIECE> __device__ __forceinline__ void place_of_chunk(const AppendArgs& a, int chunk, int& at, int& apart) {
  const bool turned = chunk < a.turned;
  at = (turned ? chunk * PIECE : 2 * a.half + (chunk - a.turned) * PIECE) * (int)sizeof(T);
  apart = (turned ? a.half : (a.chunks - a.turned) * P) * (int)sizeof(T);
}

// Tokens' heads side by side.
template <typename T, int P, bool INTERLEAVED, bool PAST>
__device__ __forceinline__ void append_rows(const AppendArgs& a, const fc_rotary_plan& plan, int group) {
  constexpr int kPieces = INTERLEAVED ? 1 : 2, kPiece = 2 * P / kPieces;     // pieces of a chunk, columns of a piece
  const int along = group / a.across, part = group - along * a.across;
  const int place = quotient(threadIdx.x, a.chunks_inverse), chunk = (int)threadIdx.x - place * a.chunks;
  const int own = quotient(place, a.abreast_inverse), beside = place - own * a.abreast;
  const int64_t row64 = (int64_t)along * a.per_group + own;
  if (own >= a.per_group || row64 >= a.rows) return;
  const int row = (int)row64, b = a.tokens == 1 ? row : row / a.tokens, t = row - b * a.tokens;
  const int heads = a.turning + a.v.heads;
  const int h0 = part * a.abreast * a.turns, h1 = min(heads, h0 + a.abreast * a.turns);
  int at, apart;
  place_of_chunk<T, P, kPiece>(a, chunk, at, apart);
  const bool turned = chunk < a.turned && h0 + beside < a.turning;
  float sn[P], cs[P];
  if (turned) sines_of<P>(a, plan, positions_of(a, row), chunk * P, sn, cs);
  // head `beside` of the queries, and what would be that of queries, keys and values as one: the rest of a head's place is the same for the wave
  const char* const q_in = a.q.in + b * a.q.sb + t * a.q.st + beside * a.q.sh + at;
  const char* const k_in = a.k.in + b * a.k.sb + t * a.k.st + (beside - a.q.heads) * a.k.sh + at;
  const char* const v_in = a.v.in + b * a.v.sb + t * a.v.st + (beside - a.turning) * a.v.sh + at;
  char* const q_out = a.q_out + b * a.ob + t * a.ot + beside * a.oh + at;
  const int64_t* const slots = a.slots + b * a.slots_b + t;
  for (int hw = h0; hw < h1; hw += a.at_once * a.abreast) {
    Vec<T, kPiece> v[kHeadsAtOnce][kPieces];
    int64_t slot[kHeadsAtOnce];
#pragma unroll
    for (int i = 0; i < kHeadsAtOnce; ++i) {
      const int hu = hw + i * a.abreast, h = hu + beside;
      if (i >= a.at_once || h >= h1) break;
      const char* in;
      if (h < a.q.heads) {
        in = q_in + hu * a.q.sh;
      } else {
        const bool key = h < a.turning;
        slot[i] = slots[(h - (key ? a.q.heads : a.turning)) * a.slots_h];
        in = key ? k_in + hu * a.k.sh : v_in + hu * a.v.sh;
      }
#pragma unroll
      for (int j = 0; j < kPieces; ++j) v[i][j] = get<PAST, T, kPiece>(in + j * apart);
    }
#pragma unroll
    for (int i = 0; i < kHeadsAtOnce; ++i) {
      const int hu = hw + i * a.abreast, h = hu + beside;
      if (i >= a.at_once || h >= h1) break;
      if (turned && h < a.turning) turn<T, P, INTERLEAVED>(v[i], sn, cs);
      char* out;
      if (h < a.q.heads) {
        out = q_out + hu * a.oh;
      } else {
        if (slot[i] < 0 || slot[i] >= a.num_slots) continue;
        out = (h < a.turning ? a.k_pages : a.v_pages) + (uint64_t)(uint32_t)slot[i] * (uint32_t)a.row_bytes + at;
      }
#pragma unroll
      for (int j = 0; j < kPieces; ++j) put<PAST>(out + j * apart, v[i][j]);
    }
  }
}

// A stretch of a KV head's tokens: the runs of tokens with a page in common that begin in it, up to their ends.  ALONE: a wave has it (a single token),
// else the workgroup, whose lane groups' results meet in LDS.
template <typename T, int P, bool INTERLEAVED, bool ALONE>
__device__ __forceinline__ void append_keys(const AppendArgs& a, const fc_rotary_plan& plan, int group, T* lds) {
  constexpr int kPieces = INTERLEAVED ? 1 : 2, kPiece = 2 * P / kPieces, kCols = 2 * P;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), item = ALONE ? group * kAppWaves + wave : group;
  const int head = item / a.stretches, b = head / a.k.heads, h = head - b * a.k.heads;
  if (b * a.tokens >= a.rows) return;
  const int t0 = (item - head * a.stretches) * a.stretch, t1 = min(a.tokens, t0 + a.stretch);
  const int64_t* const slots = a.slots + b * a.slots_b + h * a.slots_h;
  const char* const in = a.k.in + b * a.k.sb + h * a.k.sh;
  const int lanes = min(64, a.chunks), of_wave = 64 / lanes, abreast = ALONE ? of_wave : kAppWaves * of_wave;
  const int in_wave = lane / lanes, mine = ALONE ? in_wave : wave * of_wave + in_wave;       // lane group: tokens mine, mine + abreast, ... of a look-up
  // the page of a token, -1 without one
  auto page_of = [&](int64_t slot) { return slot >= 0 && slot < a.num_slots ? (int)((uint32_t)slot / (uint32_t)a.page_size) : -1; };
  for (int first = 0; first < a.chunks; first += lanes) {  // (one turn: a head's chunks but those of narrow pieces fit a wave)
    const int chunk = first + lane - in_wave * lanes;
    const bool has = in_wave < of_wave && chunk < a.chunks;
    int at, apart;
    place_of_chunk<T, P, kPiece>(a, has ? chunk : 0, at, apart);
    float low[kPieces][kPiece], high[kPieces][kPiece];
    // pages and places of the tokens from `looked` on, a thread each: one wait for memory for the pages that begin in a stretch
    __shared__ int look_page[kLooked], look_place[kLooked];
    int looked = t0 - 1;
    auto look_up = [&]() {
      const int64_t slot = slots[min(max(looked + (int)threadIdx.x, 0), a.tokens - 1)];
      const int page = page_of(slot);
      look_page[threadIdx.x] = page;
      look_place[threadIdx.x] = (int)((uint32_t)slot - (uint32_t)page * (uint32_t)a.page_size);
      __syncthreads();
    };
    if constexpr (!ALONE) {
      if (first) __syncthreads();                          // (the look-up before is done with)
      look_up();
    }
    int run = t0 == 0 ? -1 : ALONE ? page_of(slots[t0 - 1]) : look_page[0];      // page that the tokens before have
    bool open = false, begun = false;                      // whether the run is this one's; whether it has the page's first row
    // what the page's bounds are, with those of before
    auto write = [&](char* to, float l, float g, int which, int c) {
      T* const low_at = reinterpret_cast<T*>(to) + c;
      if (which == 0) {
        if (!begun) l = fminf(l, as_float(*low_at));
        *low_at = as_type<T>(l);
      } else {
        T* const high_at = reinterpret_cast<T*>(to + a.row_bytes) + c;
        if (!begun) g = fmaxf(g, as_float(*high_at));
        *high_at = as_type<T>(g);
      }
    };
    auto flush = [&]() {
      if (!open) return;
      open = false;
      char* const to = a.bounds + 2 * (int64_t)run * a.row_bytes;
      if constexpr (ALONE) {                               // (a token: the first lane group has it)
        if (has && mine == 0)
#pragma unroll
          for (int j = 0; j < kPieces; ++j) {
            if (!begun) {
              float l[kPiece], g[kPiece];
              widen<T, kPiece>(get<false, T, kPiece>(to + at + j * apart), l);
              widen<T, kPiece>(get<false, T, kPiece>(to + a.row_bytes + at + j * apart), g);
#pragma unroll
              for (int c = 0; c < kPiece; ++c) {
                low[j][c] = fminf(low[j][c], l[c]);
                high[j][c] = fmaxf(high[j][c], g[c]);
              }
            }
            put<false>(to + at + j * apart, narrow<T, kPiece>(low[j]));
            put<false>(to + a.row_bytes + at + j * apart, narrow<T, kPiece>(high[j]));
          }
      } else {
        const int cols = lanes * kCols;                    // (of a lane group, chunk by chunk)
        if (has)
#pragma unroll
          for (int j = 0; j < kPieces; ++j)
#pragma unroll
            for (int c = 0; c < kPiece; ++c) {
              T* const place = lds + mine * 2 * cols + (chunk - first) * kCols + j * kPiece + c;
              place[0] = as_type<T>(low[j][c]);
              place[cols] = as_type<T>(high[j][c]);
            }
        __syncthreads();
        const int groups = abreast;
        for (int i = threadIdx.x; i < 2 * cols; i += kAppThreads) {
          const int which = i >= cols ? 1 : 0, col = i - which * cols, ch = first + col / kCols, k = col % kCols;
          if (ch >= a.chunks) continue;
          float v = as_float(lds[i]);
#pragma unroll 4
          for (int r = 1; r < groups; ++r) {
            const float w = as_float(lds[r * 2 * cols + i]);
            v = which ? fmaxf(v, w) : fminf(v, w);
          }
          int from, between;
          place_of_chunk<T, P, kPiece>(a, ch, from, between);
          write(to + from + k / kPiece * between, v, v, which, k % kPiece);
        }
        __syncthreads();
      }
    };
    int cur = t0;
    while (cur < a.tokens) {
      // the next tokens' slots, a lane each, and how many of them are of the same page
      int page_mine, offset;
      if constexpr (ALONE) {
        const int64_t slot = slots[min(cur + lane, a.tokens - 1)];
        page_mine = page_of(slot);
        offset = (int)((uint32_t)slot - (uint32_t)page_mine * (uint32_t)a.page_size);
      } else {
        if (cur + 64 > looked + kLooked && looked + kLooked < a.tokens) {
          __syncthreads();
          looked = cur;
          look_up();
        }
        const int at = min(cur + lane, a.tokens - 1) - looked;
        page_mine = look_page[at];
        offset = look_place[at];
      }
      const int page = __builtin_amdgcn_readfirstlane(page_mine);
      const uint64_t other = __ballot(page_mine != page || cur + lane >= a.tokens);
      const int n = other ? __builtin_ctzll(other) : 64;
      if (page != run || page < 0) {                       // a new run
        flush();
        if (cur >= t1) break;
        run = page;
        open = page >= 0;
        begun = false;
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
#pragma unroll
          for (int c = 0; c < kPiece; ++c) { low[j][c] = INFINITY; high[j][c] = -INFINITY; }
      } else if (!open && cur >= t1) {
        break;
      }
      if (open) {
        begun = begun || __ballot(lane < n && offset == 0) != 0;
        for (int i = 0; i < n; i += kTokensAtOnce * abreast) {
          // (all loads before the first store: a load's wait behind one is for its end, too)
          Vec<T, kPiece> v[kTokensAtOnce][kPieces];
          Positions where[kTokensAtOnce];
#pragma unroll
          for (int u = 0; u < kTokensAtOnce; ++u) {
            const int t = min(i + u * abreast + mine, n - 1);
#pragma unroll
            for (int j = 0; j < kPieces; ++j) v[u][j] = get<false, T, kPiece>(in + (int64_t)(cur + t) * a.k.st + at + j * apart);
            where[u] = positions_of(a, b * a.tokens + cur + t);
          }
#pragma unroll
          for (int u = 0; u < kTokensAtOnce; ++u) {
            const int t = i + u * abreast + mine;
            const int off = __shfl(offset, min(t, 63), 64);
            if (has && t < n) {
              if (chunk < a.turned) {
                float sn[P], cs[P];
                sines_of<P>(a, plan, where[u], chunk * P, sn, cs);
                turn<T, P, INTERLEAVED>(v[u], sn, cs);
              }
              char* const to = a.k_pages + ((int64_t)page * a.page_size + off) * a.row_bytes + at;
#pragma unroll
              for (int j = 0; j < kPieces; ++j) {
                put<false>(to + j * apart, v[u][j]);
                float x[kPiece];
                widen<T, kPiece>(v[u][j], x);
#pragma unroll
                for (int c = 0; c < kPiece; ++c) {
                  low[j][c] = fminf(low[j][c], x[c]);
                  high[j][c] = fmaxf(high[j][c], x[c]);
                }
              }
            }
          }
        }
      }
      cur += n;
    }
    flush();
  }
}

template <typename T, int P, bool INTERLEAVED, bool PAST, bool BOUNDS>
__global__ __launch_bounds__(kAppThreads) void append_kernel(AppendArgs a, const fc_rotary_plan plan) {
  if constexpr (BOUNDS) {
    extern __shared__ __align__(16) unsigned char lds[];
    if ((int)blockIdx.x < a.bound_groups) {
      if (a.tokens == 1) append_keys<T, P, INTERLEAVED, true>(a, plan, blockIdx.x, nullptr);
      else append_keys<T, P, INTERLEAVED, false>(a, plan, blockIdx.x, reinterpret_cast<T*>(lds));
      return;
    }
  }
  append_rows<T, P, INTERLEAVED, PAST>(a, plan, (int)blockIdx.x - (BOUNDS ? a.bound_groups : 0));
}

}  // namespace

hipError_t append_launch(const fc_rotary_plan& plan, const int32_t* positions, const void* Q, void* Q_out, const fc_heads_desc& q, const void* K,
                         const fc_heads_desc& k, const void* V, const fc_heads_desc& v, const int64_t* slots, int64_t slots_b, int64_t slots_h,
                         int page_size, int64_t num_pages, void* K_pages, void* V_pages, void* bounds, hipStream_t s) {
  const int e = q.dtype == FC_BF16 ? 2 : 4, half = plan.rotary_dim / 2, rest = q.head_dim - plan.rotary_dim;
  // (the step of an axis of one says nothing: left out, as it would count in what addresses are multiples of)
  auto step = [&](int n, int64_t stride) { return n > 1 ? stride * e : 0; };
  auto side = [&](const void* in, const fc_heads_desc& d) {
    return NewRows{static_cast<const char*>(in), step(d.batch, d.stride_b), step(d.tokens, d.stride_t), step(d.heads, d.stride_h), d.heads};
  };
  AppendArgs a{};
  a.q = side(Q, q);
  a.k = side(K, k);
  a.v = side(V, v);
  a.q_out = static_cast<char*>(Q_out);
  a.ob = step(q.batch, q.out_stride_b);
  a.ot = step(q.tokens, q.out_stride_t);
  a.oh = step(q.heads, q.out_stride_h);
  a.k_pages = static_cast<char*>(K_pages);
  a.v_pages = static_cast<char*>(V_pages);
  a.bounds = static_cast<char*>(bounds);
  a.slots = slots;
  a.slots_b = slots_b;
  a.slots_h = slots_h;
  a.num_slots = num_pages * page_size;
  a.page_size = page_size;
  a.row_bytes = q.head_dim * e;
  // the widest parts that every address is a multiple of
  uint64_t bits = (uint64_t)(uintptr_t)K_pages | (uint64_t)(uintptr_t)V_pages | (uint64_t)(uintptr_t)bounds | (uint64_t)a.row_bytes;
  if (q.heads) bits |= (uint64_t)(uintptr_t)a.q_out | (uint64_t)(a.ob | a.ot | a.oh);
  for (const NewRows* r : {&a.q, &a.k, &a.v})
    if (r->heads) bits |= (uint64_t)(uintptr_t)r->in | (uint64_t)(r->sb | r->st | r->sh);
  const int pieces = plan.interleaved ? 1 : 2;             // (of a chunk: 16 bytes at most)
  int pairs = std::min(8 * pieces / e, kMostPairs);
  while (pairs > 1 && (half % pairs || rest % (2 * pairs) || (bits & (uint64_t)(2 * pairs / pieces * e - 1)))) pairs /= 2;
  a.positions = positions;
  a.tokens = q.tokens;
  a.rows = q.batch * q.tokens;
  a.half = half;
  a.turned = half / pairs;
  a.chunks = a.turned + rest / (2 * pairs);
  a.streams = plan.streams;
  a.end0 = plan.stream_end[0];
  a.end1 = plan.stream_end[1];
  a.end2 = plan.stream_end[2];
  a.magnitude = plan.magnitude;
  a.turning = q.heads + (bounds ? 0 : k.heads);
  const int heads = a.turning + v.heads, places = kAppThreads / a.chunks;
  int64_t row_groups = 0;
  if (heads) {
    const int64_t one_turn = ((int64_t)a.rows * heads + places - 1) / places;  // workgroups if every thread has a single head
    // few tokens: all heads side by side; else at least four turns, for which the sines are made once (see rotary.hip)
    int abreast = 1;
    while (abreast < kMostAbreast && 8 * abreast <= heads) abreast *= 2;
    a.abreast = std::min(std::min(heads, places), one_turn > 2048 ? abreast : heads);
    a.turns = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(kMostTurns, (heads + a.abreast - 1) / a.abreast), one_turn / 2048));
    const int batches = (a.turns + kHeadsAtOnce - 1) / kHeadsAtOnce;
    a.at_once = (a.turns + batches - 1) / batches;
    a.per_group = places / a.abreast;
    a.chunks_inverse = inverse_of(a.chunks);
    a.abreast_inverse = inverse_of(a.abreast);
    a.across = (heads + a.abreast * a.turns - 1) / (a.abreast * a.turns);
    row_groups = (((int64_t)a.rows + a.per_group - 1) / a.per_group) * a.across;
  } else {
    a.across = 1;
  }
  size_t lds = 0;
  if (bounds && k.heads) {
    a.stretch = a.tokens == 1 ? 1 : std::min(64, std::max(16, page_size));
    a.stretches = (a.tokens + a.stretch - 1) / a.stretch;
    const int64_t items = (int64_t)k.batch * k.heads * a.stretches;
    if (items >= 1 << 24) return hipErrorInvalidConfiguration;
    a.bound_groups = (int)(a.tokens == 1 ? (items + kAppWaves - 1) / kAppWaves : items);
    // a lane group's columns, least and largest, of as many groups as the waves have
    const int lanes = std::min(64, a.chunks);
    if (a.tokens > 1) lds = (size_t)kAppWaves * (64 / lanes) * 2 * lanes * 2 * pairs * e;
  }
  const int64_t groups = a.bound_groups + row_groups;
  if (groups == 0) return hipSuccess;
  if (groups >= 1 << 24) return hipErrorInvalidConfiguration;                // (2^32 threads)
  ProfileScope ps("append_kernel", s);
  auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kAppThreads), lds, s, a, plan); };
  // what is read and written exceeds the cache, in pieces of whole lines (see rotary.hip)
  const bool past = 2LL * a.rows * (q.heads + k.heads + v.heads) * a.row_bytes > 256000000 && (plan.interleaved || half * e % 128 == 0);
  auto with = [&](auto type, auto n, auto interleaved) {
    typedef decltype(type) T;
    constexpr int kN = decltype(n)::value;
    constexpr bool kInterleaved = decltype(interleaved)::value;
    if (a.bound_groups) past ? launch(append_kernel<T, kN, kInterleaved, true, true>) : launch(append_kernel<T, kN, kInterleaved, false, true>);
    else past ? launch(append_kernel<T, kN, kInterleaved, true, false>) : launch(append_kernel<T, kN, kInterleaved, false, false>);
  };
  typedef std::integral_constant<int, 4> Four;
  typedef std::integral_constant<int, 2> Two;
  typedef std::integral_constant<int, 1> One;
  auto sized = [&](auto type, auto interleaved) {          // (interleaved fp32: two pairs are 16 bytes)
    constexpr bool kFour = !decltype(interleaved)::value || sizeof(type) == 2;
    if (pairs == 1) with(type, One{}, interleaved);
    else if (!kFour || pairs == 2) with(type, Two{}, interleaved);
    else with(type, std::conditional_t<kFour, Four, Two>{}, interleaved);
  };
  auto of = [&](auto type) { plan.interleaved ? sized(type, std::true_type{}) : sized(type, std::false_type{}); };
  q.dtype == FC_BF16 ? of(uint16_t{}) : of(float{});
  return hipGetLastError();
}

}  // namespace fc
