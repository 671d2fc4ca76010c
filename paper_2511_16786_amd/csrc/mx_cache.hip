// Rows into the 4-bit paged cache, out of it, and the selection's rows straight into it.
//
// Blocks of 32 columns share a power of two; a value is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), rounded to nearest with ties to the
// even code by the conversion instruction.  Both steps are exact apart from that rounding: x / 2^k has no error.
//
// Bound by memory: a row of K and V is read once (4 D or 8 D bytes) and 17 D / 16 bytes are written.  A lane has 16 bytes of a row (fp32: of each
// half), so that what a wave loads or stores at a time are whole lines; the four (eight) lanes of a block find its largest magnitude by lane
// exchanges.  (32 bytes of an fp32 row together: 256 000 rows stored in 61 us, 52 so, loaded in 107 and 44.)  A thread has all of its rows under
// way together and ends with them: the next row's loads would wait for this one's stores.  734 000 bf16 rows of 128 columns: stored in 84 us
// (5.7 TB/s), loaded in 70 (6.8, what was stored is in the last-level cache still; the writes alone take as long).
#include <algorithm>
#include <type_traits>

#include "fc_common.h"
#include "mx.h"

namespace fc {

namespace {

constexpr int kMxThreads = 256;
constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E, kHalfMirror = 0x141;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int CTRL> __device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
  return v > o ? v : o;
}

// A lane's 16 bytes: the largest magnitude's bits as fp32 has them, and codes.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename T> struct Piece;
template <> struct Piece<uint16_t> {
  u32x4 raw;
  __device__ __forceinline__ uint32_t top() const {        // two columns at once
    u16x2 m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = __builtin_bit_cast(u16x2, raw[i] & 0x7FFF7FFFu);
    m[0] = __builtin_elementwise_max(__builtin_elementwise_max(m[0], m[1]), __builtin_elementwise_max(m[2], m[3]));
    return (uint32_t)max(m[0][0], m[0][1]) << 16;
  }
  __device__ __forceinline__ uint32_t codes(float unit) const {
    auto two = [](uint32_t bits) { return __builtin_bit_cast(bf16x2, bits); };     // (of a vector's element itself it would be the first's)
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(raw[0]), unit, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(raw[1]), unit, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(raw[2]), unit, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(raw[3]), unit, 3);
  }
};
template <> struct Piece<float> {
  u32x4 raw;
  __device__ __forceinline__ uint32_t top() const {
    return max(max(raw[0] & 0x7FFFFFFFu, raw[1] & 0x7FFFFFFFu), max(raw[2] & 0x7FFFFFFFu, raw[3] & 0x7FFFFFFFu));
  }
  __device__ __forceinline__ uint32_t codes(float unit) const {
    auto f = [](uint32_t bits) { return __uint_as_float(bits); };
    const uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, f(raw[0]), f(raw[1]), unit, 0);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(raw[2]), f(raw[3]), unit, 1);
  }
};

// D / 8 lanes have a row: piece j of lane `part` are the columns from j * D / kPieces + kCols * part on.
template <int D, typename T> struct Split {
  typedef MxTile<D> Tile;
  static constexpr int kLanes = D / 8, kAtOnce = kMxThreads / kLanes, kPieces = sizeof(T) / 2, kCols = 16 / sizeof(T);
  static __device__ __forceinline__ int column(int j, int part) { return j * (D / kPieces) + kCols * part; }
  static __device__ __forceinline__ int bytes(int j, int part) { return column(j, part) * (int)sizeof(T); }
  static __device__ __forceinline__ int k_code(int row, int col) { return Tile::k_code(row, col / 2); }
  static __device__ __forceinline__ int v_code(int row, int col) { return Tile::v_code(row, col / (D / 16)) + col % (D / 16) / 2; }
  static __device__ __forceinline__ int k_scale(int row, int col) { return Tile::k_scale(row, col / 32); }
  static __device__ __forceinline__ int v_scale(int row, int col) { return Tile::v_scale(row, col / 32); }
};

// Codes of a lane's piece and E of its block.
template <typename T> __device__ __forceinline__ uint32_t encode(const Piece<T>& x, uint32_t& E) {
  uint32_t top = dpp_max<kQuadXor2>(dpp_max<kQuadXor1>(x.top()));
  if constexpr (sizeof(T) == 4) top = dpp_max<kHalfMirror>(top);           // (the other quad of the eight)
  E = mx_scale(top);
  const uint32_t c = x.codes(__uint_as_float(E << 23));
  return E == 255u ? 0u : c;
}

// A lane's piece j of row `row` of the tile, K and V.
template <int D, typename T>
__device__ __forceinline__ void write_piece(uint8_t* tile, int row, int j, int part, const Piece<T>& k, const Piece<T>& v) {
  typedef Split<D, T> S;
  const int col = S::column(j, part);
  uint32_t ke, ve;
  const uint32_t kc = encode(k, ke), vc = encode(v, ve);
  if constexpr (S::kCols == 4) {
    *reinterpret_cast<uint16_t*>(tile + S::k_code(row, col)) = (uint16_t)kc;
    *reinterpret_cast<uint16_t*>(tile + S::v_code(row, col)) = (uint16_t)vc;
  } else {
    *reinterpret_cast<uint32_t*>(tile + S::k_code(row, col)) = kc;
    if constexpr (D == 128) {
      *reinterpret_cast<uint32_t*>(tile + S::v_code(row, col)) = vc;
    } else {                                               // four columns a place: two of them
      *reinterpret_cast<uint16_t*>(tile + S::v_code(row, col)) = (uint16_t)vc;
      *reinterpret_cast<uint16_t*>(tile + S::v_code(row, col + 4)) = (uint16_t)(vc >> 16);
    }
  }
  if (col % 32 == 0) {
    tile[S::k_scale(row, col)] = (uint8_t)ke;
    tile[S::v_scale(row, col)] = (uint8_t)ve;
  }
}

// Where the rows of a launch come from and go: row i of sequence b, bytes from the base, and a slot (negative: it is left out).
struct RowsOf {                  // rows [B][R][D] with strides, and a slot for each
  int64_t sb, sr;
  const int64_t* slots;
  size_t lds_bytes() const { return 0; }
  __device__ __forceinline__ void stage(int, int64_t*) const {}
  __device__ __forceinline__ int64_t look(int b, int64_t i, int64_t rows) const { return slots[(int64_t)b * rows + i]; }
  __device__ __forceinline__ void where(int b, int64_t i, int64_t seen, int64_t num_slots, const int64_t*, int64_t& from, int64_t& slot) const {
    slot = seen < num_slots ? seen : -1;
    from = b * sb + i * sr;
  }
};
struct KeptRows {                // kept rows of a cache [B][L][H][N][D], in the order of layer, head and token
  KvStrides st;
  int n, elem_bytes, page_size, max_pages;
  const int32_t* budgets;
  const int64_t* offsets;
  const int32_t* idx;
  const int32_t* table;
  size_t lds_bytes() const { return (size_t)(st.L + 1) * sizeof(int64_t) + (size_t)st.L * sizeof(int32_t); }
  // the sequence's offsets and budgets in LDS (read from there by every row's search for its layer: 5 loads one after another)
  __device__ __forceinline__ void stage(int b, int64_t* offs) const {
    int32_t* const kept = reinterpret_cast<int32_t*>(offs + st.L + 1);
    for (int l = threadIdx.x; l <= st.L; l += kMxThreads) offs[l] = offsets[(int64_t)b * (st.L + 1) + l];
    for (int l = threadIdx.x; l < st.L; l += kMxThreads) kept[l] = budgets[(int64_t)b * st.L + l];
  }
  __device__ __forceinline__ int look(int b, int64_t i, int64_t rows) const { return idx[(int64_t)b * rows + i]; }
  __device__ __forceinline__ void where(int b, int64_t i, int token, int64_t num_slots, const int64_t* offs, int64_t& from, int64_t& slot) const {
    slot = -1;
    from = 0;
    if (token < 0 || token >= n || i < offs[0] || i >= offs[st.L]) return;
    int lo = 0, hi = st.L;                                 // largest l with offs[l] <= i
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (offs[mid] <= i) lo = mid; else hi = mid;
    }
    const int k = reinterpret_cast<const int32_t*>(offs + st.L + 1)[lo];
    const int64_t in = i - offs[lo];
    if (k <= 0 || k > n || in >= (int64_t)st.H * k) return;      // (bad budgets; H * n is below 2^32)
    const int h = (int)((uint32_t)in / (uint32_t)k), j = (int)(in - (int64_t)h * k), p = j / page_size;
    if (p >= max_pages) return;
    const int64_t page = table[(((int64_t)b * st.L + lo) * st.H + h) * max_pages + p];
    from = ((int64_t)b * st.sb + (int64_t)lo * st.sl + (int64_t)h * st.sh + (int64_t)token * st.sn) * elem_bytes;
    slot = page * page_size + (j - p * page_size);
    if (page < 0 || slot >= num_slots) slot = -1;
  }
};

// Keeps loads where they are: the compiler would move a row's to where it is stored, behind the stores of the row before.
template <typename T, int R, int P> __device__ __forceinline__ void all_here(Piece<T> (&x)[R][P]) {
#pragma unroll
  for (int u = 0; u < R; ++u)
#pragma unroll
    for (int j = 0; j < P; ++j) asm volatile("" : "+v"(x[u][j].raw));
}
template <int R, int P> __device__ __forceinline__ void all_here(uint32_t (&x)[R][P]) {
#pragma unroll
  for (int u = 0; u < R; ++u)
#pragma unroll
    for (int j = 0; j < P; ++j) asm volatile("" : "+v"(x[u][j]));
}

// grid = (runs of rows, sequences), `ROWS` rows for each group of lanes.  A thread finds out where one of the workgroup's rows is and goes; then
// D / 8 lanes have a row.
template <int D, typename T, typename Source, int ROWS>
__global__ __launch_bounds__(kMxThreads) void mx_store_kernel(const char* __restrict__ K, const char* __restrict__ V, Source src,
                                                              int64_t rows, int64_t num_slots, uint8_t* __restrict__ pages) {
  typedef Split<D, T> S;
  constexpr int kShare = ROWS * S::kAtOnce;
  __shared__ int64_t from[kShare], to[kShare];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int64_t first = (int64_t)blockIdx.x * kShare;
  extern __shared__ int64_t staged[];
  src.stage(b, staged);
  const bool mine = tid < kShare && first + tid < rows;
  const auto seen = mine ? src.look(b, first + tid, rows) : -1;
  if constexpr (!std::is_same<Source, RowsOf>::value) __syncthreads();
  if (tid < kShare) {
    int64_t f = 0, s = -1;
    if (mine) src.where(b, first + tid, seen, num_slots, staged, f, s);
    from[tid] = f;
    to[tid] = s < 0 ? -1 : (s >> 4) * (MxTile<D>::kBytes * 16) + (s & 15);     // the tile's place, and the row in its last four bits
  }
  __syncthreads();
  const int part = tid % S::kLanes, group = tid / S::kLanes;
  Piece<T> k[ROWS][S::kPieces], v[ROWS][S::kPieces];
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {                         // (a row that goes nowhere: what is at its place all the same, or the first row)
    const int64_t at = from[group + u * S::kAtOnce];
#pragma unroll
    for (int j = 0; j < S::kPieces; ++j) {
      k[u][j].raw = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(K + at + S::bytes(j, part)));
      v[u][j].raw = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(V + at + S::bytes(j, part)));
    }
  }
  all_here(k);
  all_here(v);
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    const int64_t place = to[group + u * S::kAtOnce];
    if (place < 0) continue;                               // (the same for a block's lanes)
#pragma unroll
    for (int j = 0; j < S::kPieces; ++j) write_piece<D>(pages + (place >> 4), (int)(place & 15), j, part, k[u][j], v[u][j]);
  }
}

// 16 bytes of what the codes stand for: exact in bf16.
template <typename T> __device__ __forceinline__ u32x4 decode(uint32_t code, uint32_t E) {
  const float unit = __uint_as_float(E << 23);
  const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, unit, 0));
  const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, unit, 1));
  if constexpr (sizeof(T) == 4) {
    return u32x4{a << 16, a & 0xFFFF0000u, b << 16, b & 0xFFFF0000u};
  } else {
    const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, unit, 2));
    const uint32_t d = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, unit, 3));
    return u32x4{a, b, c, d};
  }
}

// Past the last-level cache.  (The value is made first: taken together with its conversions the store lost the hint.)
__device__ __forceinline__ void put_past(char* p, u32x4 v) {
  asm volatile("" : "+v"(v));
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
}

// grid = (runs of rows, sequences), ROWS rows for each group of lanes; rows without a slot become zeros.
template <int D, typename T, int ROWS>
__global__ __launch_bounds__(kMxThreads) void mx_load_kernel(const int64_t* __restrict__ slots, const uint8_t* __restrict__ pages,
                                                             int64_t rows, int64_t num_slots, int64_t sb, int64_t sr,
                                                             char* __restrict__ K, char* __restrict__ V) {
  typedef Split<D, T> S;
  constexpr int kShare = ROWS * S::kAtOnce;
  __shared__ int64_t from[kShare];
  const int b = blockIdx.y, tid = threadIdx.x, part = tid % S::kLanes, group = tid / S::kLanes;
  const int64_t first = (int64_t)blockIdx.x * kShare;
  if (tid < kShare) {
    const int64_t s = slots[(int64_t)b * rows + min(first + tid, rows - 1)];   // (behind the last row it comes again)
    from[tid] = s >= 0 && s < num_slots ? (s >> 4) * (MxTile<D>::kBytes * 16) + (s & 15) : -1;
  }
  __syncthreads();
  uint32_t kc[ROWS][S::kPieces], vc[ROWS][S::kPieces], ke[ROWS][S::kPieces], ve[ROWS][S::kPieces];
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    const int64_t place = max(from[group + u * S::kAtOnce], (int64_t)0);       // (the cache's first slot in place of none)
    const uint8_t* const tile = pages + (place >> 4);
    const int row = (int)(place & 15);
#pragma unroll
    for (int j = 0; j < S::kPieces; ++j) {
      const int col = S::column(j, part);
      if constexpr (S::kCols == 4) {
        kc[u][j] = *reinterpret_cast<const uint16_t*>(tile + S::k_code(row, col));
        vc[u][j] = *reinterpret_cast<const uint16_t*>(tile + S::v_code(row, col));
      } else {
        kc[u][j] = *reinterpret_cast<const uint32_t*>(tile + S::k_code(row, col));
        if constexpr (D == 128) vc[u][j] = *reinterpret_cast<const uint32_t*>(tile + S::v_code(row, col));
        else vc[u][j] = *reinterpret_cast<const uint16_t*>(tile + S::v_code(row, col)) |
                        (uint32_t)*reinterpret_cast<const uint16_t*>(tile + S::v_code(row, col + 4)) << 16;
      }
      ke[u][j] = tile[S::k_scale(row, col)];
      ve[u][j] = tile[S::v_scale(row, col)];
    }
  }
  all_here(kc);
  all_here(vc);
  all_here(ke);
  all_here(ve);
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    const int r = group + u * S::kAtOnce;
    const uint32_t held = from[r] >= 0 ? ~0u : 0u;
    const int64_t at = b * sb + min(first + r, rows - 1) * sr;
#pragma unroll
    for (int j = 0; j < S::kPieces; ++j) {
      put_past(K + at + S::bytes(j, part), decode<T>(kc[u][j] & held, ke[u][j] & held));
      put_past(V + at + S::bytes(j, part), decode<T>(vc[u][j] & held, ve[u][j] & held));
    }
  }
}

// Rows of each group of lanes: one where a launch is a few workgroups a compute unit at most, several where most workgroups wait for others to end
// (starting them counts then: some 430 a microsecond).  128 columns, bf16, us with 1, 2 and 4 rows: store of 4000 rows 3.3, 3.7, 3.6, 32 000
// 5.2, 5.4, 5.7, 64 000 9.7, 8.8, 9.2, 734 000 94, 85, 85; gather of 4000 8.4, 8.7, 9.3, 64 000 20.9, 19.1, 19.3, 734 000 114, 100, 96; load of 896 (in
// one pass with their store) 4.7, 5.3, 6.1, 8000 3.2, 3.1, 3.4, 16 000 4.1, 3.4, 3.7, 734 000 behind a gather 112, 69, 73.
constexpr int kStoreRows = 2, kGatherRows = 4, kLoadRows = 2;
constexpr int64_t kStoreOnes = 2048, kLoadOnes = 256;      // up to so many groups: one row
template <int MANY, typename Source>
hipError_t store(const void* K, const void* V, const Source& src, int B, int64_t rows, int d, int dtype, void* pages, int64_t num_slots,
                 const char* name, hipStream_t s) {
  const int at_once = kMxThreads / (d / 8);
  const bool many = rows * B > kStoreOnes * at_once;
  const int share = at_once * (many ? MANY : 1);
  const dim3 grid((unsigned)((rows + share - 1) / share), (unsigned)B);
  ProfileScope ps(name, s);
  auto launch = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(kMxThreads), src.lds_bytes(), s, static_cast<const char*>(K), static_cast<const char*>(V), src, rows,
                       num_slots, static_cast<uint8_t*>(pages));
  };
  auto of_type = [&](auto type) {
    typedef decltype(type) T;
    if (d == 128) many ? launch(mx_store_kernel<128, T, Source, MANY>) : launch(mx_store_kernel<128, T, Source, 1>);
    else many ? launch(mx_store_kernel<64, T, Source, MANY>) : launch(mx_store_kernel<64, T, Source, 1>);
  };
  dtype == FC_BF16 ? of_type(uint16_t{}) : of_type(float{});
  return hipGetLastError();
}

}  // namespace

hipError_t mx_store_launch(const void* K, const void* V, const fc_rows_desc& r, const int64_t* slots, void* pages, int64_t num_slots,
                           hipStream_t s) {
  const int e = r.dtype == FC_BF16 ? 2 : 4;
  return store<kStoreRows>(K, V, RowsOf{r.stride_b * e, r.stride_r * e, slots}, r.batch, r.rows, r.head_dim, r.dtype, pages, num_slots,
                           "mx_store_kernel", s);
}

hipError_t mx_load_launch(const fc_rows_desc& r, const int64_t* slots, const void* pages, int64_t num_slots, void* K, void* V,
                          hipStream_t s) {
  const int e = r.dtype == FC_BF16 ? 2 : 4, at_once = kMxThreads / (r.head_dim / 8);
  const bool many = r.rows * r.batch > kLoadOnes * at_once;
  const int share = at_once * (many ? kLoadRows : 1);
  const dim3 grid((unsigned)((r.rows + share - 1) / share), (unsigned)r.batch);
  ProfileScope ps("mx_load_kernel", s);
  auto launch = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(kMxThreads), 0, s, slots, static_cast<const uint8_t*>(pages), r.rows, num_slots,
                       r.stride_b * e, r.stride_r * e, static_cast<char*>(K), static_cast<char*>(V));
  };
  auto of_type = [&](auto type) {
    typedef decltype(type) T;
    if (r.head_dim == 128) many ? launch(mx_load_kernel<128, T, kLoadRows>) : launch(mx_load_kernel<128, T, 1>);
    else many ? launch(mx_load_kernel<64, T, kLoadRows>) : launch(mx_load_kernel<64, T, 1>);
  };
  r.dtype == FC_BF16 ? of_type(uint16_t{}) : of_type(float{});
  return hipGetLastError();
}

hipError_t mx_gather_launch(const void* K, const void* V, const fc_kv_desc& d, const int32_t* budgets, const int64_t* offsets,
                            int64_t rows_per_seq, const int32_t* idx, const int32_t* table, int32_t page_size, int32_t max_pages,
                            void* pages, int64_t num_slots, hipStream_t s) {
  const KeptRows src{strides_of(d), d.n_tokens, d.dtype == FC_BF16 ? 2 : 4, page_size, max_pages, budgets, offsets, idx, table};
  return store<kGatherRows>(K, V, src, d.batch, rows_per_seq, d.head_dim, d.dtype, pages, num_slots, "mx_gather_kernel", s);
}

}  // namespace fc
