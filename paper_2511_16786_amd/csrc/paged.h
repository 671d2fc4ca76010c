// A paged cache as the kernels take it.
#ifndef FC_PAGED_H_
#define FC_PAGED_H_

#include "fc_common.h"

namespace fc {

namespace {

constexpr int kMostPagedRows = (1 << 25) - 1;

// Quotients of numbers n below 2^31 by d: with l = ceil(log2 d) and m = floor(2^(31 + l) / d) + 1, the product m d is 2^(31 + l) + e with 0 < e <= d <= 2^l,
// so that n m / 2^(31 + l) = n / d + n e / (d 2^(31 + l)), and what is added is below 1 / d: the same whole part.  m has 32 bits for d > 1.
struct Divider {
  uint32_t m;
  int shift;                     // l - 1; negative: d is 1
  __device__ __forceinline__ int of(int n) const { return shift < 0 ? n : (int)(__umulhi((uint32_t)n, m) >> shift); }
};
inline Divider divider(int d) {
  if (d == 1) return {0u, -1};
  const int l = 32 - __builtin_clz((unsigned)(d - 1));
  return {(uint32_t)((1ull << (31 + l)) / (unsigned)d + 1), l - 1};
}

struct PagedArgs {
  const void* K;
  const void* V;
  const int32_t* rows;           // [B][L], rows_b between sequences
  const int32_t* table;          // [B][L][H][max_pages], table_b between sequences
  int64_t rows_b, table_b, num_pages;
  int B, L, H, page_size, max_pages;
  Divider pages;                 // by the page's size
};

inline PagedArgs paged_args(const fc_paged_kv& kv) {
  return PagedArgs{kv.K, kv.V, kv.rows, kv.block_table, kv.rows_stride_b, kv.table_stride_b, kv.num_pages,
                   kv.batch, kv.layers, kv.kv_heads, kv.page_size, kv.max_pages, divider(kv.page_size)};
}

// Rows of a layer that its table can reach.
__device__ __forceinline__ int rows_within(const PagedArgs& a, int rows) {
  return (int)min((int64_t)min(max(rows, 0), kMostPagedRows), (int64_t)a.max_pages * a.page_size);
}
__device__ __forceinline__ int rows_of(const PagedArgs& a, int b, int l) { return rows_within(a, a.rows[b * a.rows_b + l]); }
__device__ __forceinline__ int pages_of(const PagedArgs& a, int b, int l) { return (rows_of(a, b, l) + a.page_size - 1) / a.page_size; }

}  // namespace

}  // namespace fc
#endif
