// Rows into the 4-bit paged cache, out of it, and the selection's rows straight into it.
//
// Blocks of 32 columns share a power of two; a value is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), rounded to nearest with ties to the
// even code by the conversion instruction.  Both steps are exact apart from that rounding: x / 2^k has no error.
//
// Bound by memory: a row of K and V is read once (4 D or 8 D bytes) and 17 D / 16 bytes are written.  Eight columns a lane, so that a row's
// load is one run of 16-byte pieces (fp32: two), four lanes have a block in common and find its largest magnitude by two lane exchanges.
#include <algorithm>
#include <type_traits>

#include "fc_common.h"
#include "mx.h"

namespace fc {

namespace {

constexpr int kMxThreads = 256;
constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int CTRL> __device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
  return v > o ? v : o;
}

// Eight columns: the largest magnitude's bits as fp32 has them, and codes.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
  u32x4 raw;
  __device__ __forceinline__ void load(const char* p) { raw = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
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
template <> struct Eight<float> {
  u32x4 a, b;
  __device__ __forceinline__ void load(const char* p) {
    a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    b = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + 1);
  }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(a[i] & 0x7FFFFFFFu, b[i] & 0x7FFFFFFFu));
    return m;
  }
  __device__ __forceinline__ uint32_t codes(float unit) const {
    auto f = [](uint32_t bits) { return __uint_as_float(bits); };
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(a[0]), f(a[1]), unit, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(a[2]), f(a[3]), unit, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(b[0]), f(b[1]), unit, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(b[2]), f(b[3]), unit, 3);
  }
};

// Codes of a lane's eight columns and E of their block, which four lanes have.
template <typename T> __device__ __forceinline__ uint32_t encode(const Eight<T>& v, uint32_t& E) {
  E = mx_scale(dpp_max<kQuadXor2>(dpp_max<kQuadXor1>(v.top())));
  const uint32_t c = v.codes(__uint_as_float(E << 23));
  return E == 255u ? 0u : c;
}

// A lane's columns 8 part .. 8 part + 7 of row `row` of the tile, K and V.
template <int D, typename T>
__device__ __forceinline__ void write_row(uint8_t* tile, int row, int part, const Eight<T>& k, const Eight<T>& v) {
  typedef MxTile<D> Tile;
  uint32_t ke, ve;
  const uint32_t kc = encode(k, ke), vc = encode(v, ve);
  *reinterpret_cast<uint32_t*>(tile + Tile::k_code(row, 4 * part)) = kc;
  if constexpr (D == 128) {
    *reinterpret_cast<uint32_t*>(tile + Tile::v_code(row, part)) = vc;
  } else {                                                 // four columns a place: two of them
    *reinterpret_cast<uint16_t*>(tile + Tile::v_code(row, 2 * part)) = (uint16_t)vc;
    *reinterpret_cast<uint16_t*>(tile + Tile::v_code(row, 2 * part + 1)) = (uint16_t)(vc >> 16);
  }
  if (part % 4 == 0) {
    tile[Tile::k_scale(row, part / 4)] = (uint8_t)ke;
    tile[Tile::v_scale(row, part / 4)] = (uint8_t)ve;
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

// grid = (runs of `share` rows, sequences).  A thread finds out where one of the workgroup's rows is and goes; then D / 8 lanes have a row.
template <int D, typename T, typename Source>
__global__ __launch_bounds__(kMxThreads) void mx_store_kernel(const char* __restrict__ K, const char* __restrict__ V, Source src,
                                                              int64_t rows, int share, int64_t num_slots, uint8_t* __restrict__ pages) {
  constexpr int kLanes = D / 8, kAtOnce = kMxThreads / kLanes;
  __shared__ int64_t from[kMxThreads], to[kMxThreads];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int64_t first = (int64_t)blockIdx.x * share;
  extern __shared__ int64_t staged[];
  src.stage(b, staged);
  const bool mine = tid < share && first + tid < rows;
  const auto seen = mine ? src.look(b, first + tid, rows) : -1;
  if constexpr (!std::is_same<Source, RowsOf>::value) __syncthreads();
  if (tid < share) {
    int64_t f = 0, s = -1;
    if (mine) src.where(b, first + tid, seen, num_slots, staged, f, s);
    from[tid] = f;
    to[tid] = s < 0 ? -1 : (s >> 4) * (MxTile<D>::kBytes * 16) + (s & 15);     // the tile's place, and the row in its last four bits
  }
  __syncthreads();
  const int part = tid % kLanes;
  for (int r = tid / kLanes; r < share; r += kAtOnce) {
    const int64_t place = to[r];
    if (place < 0) continue;                               // (the same for a block's four lanes)
    Eight<T> k, v;
    k.load(K + from[r] + part * 8 * (int)sizeof(T));
    v.load(V + from[r] + part * 8 * (int)sizeof(T));
    write_row<D>(pages + (place >> 4), (int)(place & 15), part, k, v);
  }
}

// Eight columns of what the codes stand for: exact in bf16.
__device__ __forceinline__ void decode(uint32_t code, uint32_t E, uint32_t (&o)[4]) {
  const float unit = __uint_as_float(E << 23);
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, unit, 0));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, unit, 1));
  o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, unit, 2));
  o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, unit, 3));
}
template <typename T> __device__ __forceinline__ void put_eight(char* p, const uint32_t (&o)[4]) {
  if constexpr (sizeof(T) == 2) {
    __builtin_nontemporal_store((u32x4{o[0], o[1], o[2], o[3]}), reinterpret_cast<u32x4*>(p));
  } else {
    const u32x4 a = {o[0] << 16, o[0] & 0xFFFF0000u, o[1] << 16, o[1] & 0xFFFF0000u};
    const u32x4 b = {o[2] << 16, o[2] & 0xFFFF0000u, o[3] << 16, o[3] & 0xFFFF0000u};
    __builtin_nontemporal_store(a, reinterpret_cast<u32x4*>(p));
    __builtin_nontemporal_store(b, reinterpret_cast<u32x4*>(p) + 1);
  }
}

// grid = (runs of `share` rows, sequences); rows without a slot become zeros.
template <int D, typename T>
__global__ __launch_bounds__(kMxThreads) void mx_load_kernel(const int64_t* __restrict__ slots, const uint8_t* __restrict__ pages,
                                                             int64_t rows, int share, int64_t num_slots, int64_t sb, int64_t sr,
                                                             char* __restrict__ K, char* __restrict__ V) {
  typedef MxTile<D> Tile;
  constexpr int kLanes = D / 8, kAtOnce = kMxThreads / kLanes;
  const int b = blockIdx.y, part = threadIdx.x % kLanes;
  const int64_t first = (int64_t)blockIdx.x * share, last = first + share < rows ? first + share : rows;
  for (int64_t i = first + threadIdx.x / kLanes; i < last; i += kAtOnce) {
    const int64_t slot = slots[(int64_t)b * rows + i];
    const bool ok = slot >= 0 && slot < num_slots;
    uint32_t k[4] = {0u, 0u, 0u, 0u}, v[4] = {0u, 0u, 0u, 0u};
    if (ok) {
      const uint8_t* tile = pages + (slot >> 4) * Tile::kBytes;
      const int row = (int)(slot & 15);
      decode(*reinterpret_cast<const uint32_t*>(tile + Tile::k_code(row, 4 * part)), tile[Tile::k_scale(row, part / 4)], k);
      uint32_t code;
      if constexpr (D == 128) code = *reinterpret_cast<const uint32_t*>(tile + Tile::v_code(row, part));
      else code = *reinterpret_cast<const uint16_t*>(tile + Tile::v_code(row, 2 * part)) |
                  (uint32_t)*reinterpret_cast<const uint16_t*>(tile + Tile::v_code(row, 2 * part + 1)) << 16;
      decode(code, tile[Tile::v_scale(row, part / 4)], v);
    }
    const int64_t at = b * sb + i * sr + part * 8 * (int)sizeof(T);
    put_eight<T>(K + at, k);
    put_eight<T>(V + at, v);
  }
}

// Rows of a workgroup: a group of lanes has one at a time, several in turn where there are thousands of workgroups all the same.  `enough`
// workgroups: 734 000 rows stored from packed rows 93 us with 4096, 85 with 16384, loaded 75 / 72; gathered 98 / 104, whose threads look rows up.
int rows_a_group(int64_t rows, int B, int at_once, int enough) {
  const int64_t turns = rows * B / at_once / enough;
  return at_once * (int)std::min<int64_t>(kMxThreads / at_once, std::max<int64_t>(1, turns));
}

template <typename Source>
hipError_t store(const void* K, const void* V, const Source& src, int B, int64_t rows, int d, int dtype, void* pages, int64_t num_slots,
                 int enough, const char* name, hipStream_t s) {
  const int share = rows_a_group(rows, B, kMxThreads / (d / 8), enough);
  const dim3 grid((unsigned)((rows + share - 1) / share), (unsigned)B);
  ProfileScope ps(name, s);
  auto launch = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(kMxThreads), src.lds_bytes(), s, static_cast<const char*>(K), static_cast<const char*>(V), src, rows, share,
                       num_slots, static_cast<uint8_t*>(pages));
  };
  if (dtype == FC_BF16) d == 128 ? launch(mx_store_kernel<128, uint16_t, Source>) : launch(mx_store_kernel<64, uint16_t, Source>);
  else d == 128 ? launch(mx_store_kernel<128, float, Source>) : launch(mx_store_kernel<64, float, Source>);
  return hipGetLastError();
}

}  // namespace

hipError_t mx_store_launch(const void* K, const void* V, const fc_rows_desc& r, const int64_t* slots, void* pages, int64_t num_slots,
                           hipStream_t s) {
  const int e = r.dtype == FC_BF16 ? 2 : 4;
  return store(K, V, RowsOf{r.stride_b * e, r.stride_r * e, slots}, r.batch, r.rows, r.head_dim, r.dtype, pages, num_slots,
               16384, "mx_store_kernel", s);
}

hipError_t mx_load_launch(const fc_rows_desc& r, const int64_t* slots, const void* pages, int64_t num_slots, void* K, void* V,
                          hipStream_t s) {
  const int e = r.dtype == FC_BF16 ? 2 : 4, share = rows_a_group(r.rows, r.batch, kMxThreads / (r.head_dim / 8), 16384);
  const dim3 grid((unsigned)((r.rows + share - 1) / share), (unsigned)r.batch);
  ProfileScope ps("mx_load_kernel", s);
  auto launch = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(kMxThreads), 0, s, slots, static_cast<const uint8_t*>(pages), r.rows, share, num_slots,
                       r.stride_b * e, r.stride_r * e, static_cast<char*>(K), static_cast<char*>(V));
  };
  if (r.dtype == FC_BF16) r.head_dim == 128 ? launch(mx_load_kernel<128, uint16_t>) : launch(mx_load_kernel<64, uint16_t>);
  else r.head_dim == 128 ? launch(mx_load_kernel<128, float>) : launch(mx_load_kernel<64, float>);
  return hipGetLastError();
}

hipError_t mx_gather_launch(const void* K, const void* V, const fc_kv_desc& d, const int32_t* budgets, const int64_t* offsets,
                            int64_t rows_per_seq, const int32_t* idx, const int32_t* table, int32_t page_size, int32_t max_pages,
                            void* pages, int64_t num_slots, hipStream_t s) {
  const KeptRows src{strides_of(d), d.n_tokens, d.dtype == FC_BF16 ? 2 : 4, page_size, max_pages, budgets, offsets, idx, table};
  return store(K, V, src, d.batch, rows_per_seq, d.head_dim, d.dtype, pages, num_slots, 4096, "mx_gather_kernel", s);
}

}  // namespace fc
