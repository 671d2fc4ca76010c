// Block tables and slot maps of a paged cache, from the rows that the layers of each sequence hold and add (both on the device: budgets
// are made there).  Unit (b, l, h) has ceil(rows / page_size) pages; pages that the added rows begin are taken from a free list in the order
// of the units, so that the page of a unit's row is a prefix sum away and the result does not depend on how the work is shared out.
//
// One pass over the added rows writes both: a row's slot, and the table's entry by the row that begins a page.  A few bytes a row and no
// arithmetic to speak of: bound by its launch and by the chain of loads before the first store (rows, prefix sums, free list).
#include <algorithm>

#include "fc_common.h"

namespace fc {

namespace {

constexpr int kPageThreads = 256;
constexpr int kMostRows = (1 << 25) - 1;

struct PageArgs {
  const int32_t* rows;
  const int32_t* add;            // or nullptr: add_each
  int32_t* rows_out;
  const int32_t* free_pages;     // or nullptr: page i is i
  int32_t* table;
  const int64_t* cursor;
  int64_t* cursor_out;
  int64_t* slots;                // [B][slots_per_seq] or nullptr
  int64_t num_free, slots_per_seq;
  int B, L, H, page_size, page_shift, max_pages, add_each;         // (the shift: -1 if the size is no power of two)
  bool finish;                   // one workgroup, or outputs of their own: they are written here
};

struct Held { int rows, grown, first, fresh; };             // rows before and after, pages before, pages taken
__device__ __forceinline__ Held held_at(const PageArgs& a, int i) {
  Held x;
  x.rows = min(max(a.rows[i], 0), kMostRows);
  x.grown = min(x.rows + min(max(a.add ? a.add[i] : a.add_each, 0), kMostRows), kMostRows);
  x.first = min((x.rows + a.page_size - 1) / a.page_size, a.max_pages);
  x.fresh = min((x.grown + a.page_size - 1) / a.page_size, a.max_pages) - x.first;
  return x;
}

// grid = (shares of a sequence's rows, sequences)
template <bool SLOTS>
__global__ __launch_bounds__(kPageThreads) void assign_pages_kernel(PageArgs a) {
  extern __shared__ int64_t lds[];
  int64_t* const rows_before = lds;                        // [L + 1], all heads
  int64_t* const pages_before = lds + a.L + 1;             // [L + 1], all heads and the sequences before
  Held* const held = reinterpret_cast<Held*>(pages_before + a.L + 1);          // [L]
  __shared__ int64_t wave_rows[kPageThreads / 64], wave_pages[kPageThreads / 64], before_wave[kPageThreads / 64];
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // pages that earlier sequences take
  int64_t earlier = 0;
  for (int i = tid; i < b * a.L; i += kPageThreads) earlier += held_at(a, i).fresh;
#pragma unroll
  for (int d = 32; d; d >>= 1) earlier += __shfl_xor(earlier, d, 64);
  if (lane == 0) before_wave[wave] = earlier;
  // prefix sums over the layers, a thread's `per` neighbours at a time
  const int per = (a.L + kPageThreads - 1) / kPageThreads, l0 = min(a.L, tid * per), l1 = min(a.L, l0 + per);
  int64_t rows = 0, pages = 0;
  for (int l = l0; l < l1; ++l) {
    const Held x = held_at(a, b * a.L + l);
    held[l] = x;
    rows += x.grown - x.rows;
    pages += x.fresh;
  }
  int64_t rows_in = rows, pages_in = pages;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t r = __shfl_up(rows_in, d, 64), p = __shfl_up(pages_in, d, 64);
    if (lane >= d) { rows_in += r; pages_in += p; }
  }
  if (lane == 63) { wave_rows[wave] = rows_in; wave_pages[wave] = pages_in; }
  const int64_t cursor = a.cursor[0];
  __syncthreads();
  int64_t r = rows_in - rows, p = pages_in - pages;
  earlier = 0;
  for (int w = 0; w < kPageThreads / 64; ++w) {
    if (w < wave) { r += wave_rows[w]; p += wave_pages[w]; }
    earlier += before_wave[w];
  }
  for (int l = l0; l < l1; ++l) {
    const Held x = held[l];
    rows_before[l] = r * a.H;
    pages_before[l] = (earlier + p) * a.H;
    r += x.grown - x.rows;
    p += x.fresh;
    if (l == a.L - 1) {
      rows_before[a.L] = r * a.H;
      pages_before[a.L] = (earlier + p) * a.H;
    }
  }
  __syncthreads();
  auto page_at = [&](int64_t at) {                         // of the free list
    const int64_t i = cursor + at;
    return i >= 0 && i < a.num_free ? (a.free_pages ? a.free_pages[i] : (int32_t)i) : -1;
  };
  auto layer_of = [&](const int64_t* before, int64_t at) { // largest l with before[l] <= at < before[l + 1]
    int lo = 0, hi = a.L;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before[mid] <= at) lo = mid; else hi = mid;
    }
    return lo;
  };
  const int64_t step = (int64_t)gridDim.x * kPageThreads, begin = (int64_t)blockIdx.x * kPageThreads + tid;
  // (heads times rows of a layer are below 2^31 in all but caches that nobody has: 32-bit divisions)
  auto head_of = [](int64_t in, int each) { return in >> 31 ? (int)(in / each) : (int)((uint32_t)in / (uint32_t)each); };
  if constexpr (SLOTS) {
    const int64_t all = rows_before[a.L], end = all > a.slots_per_seq ? all : a.slots_per_seq;
    for (int64_t i = begin; i < end; i += step) {
      int64_t slot = -1;
      if (i < all) {
        const int l = layer_of(rows_before, i);
        const Held x = held[l];
        const int added = x.grown - x.rows;
        const int64_t in = i - rows_before[l];             // < H * added
        const int h = head_of(in, added), row = x.rows + (int)(in - (int64_t)h * added);
        const int page = a.page_shift >= 0 ? row >> a.page_shift : row / a.page_size, off = row - page * a.page_size;
        int32_t* const entry = a.table + ((int64_t)(b * a.L + l) * a.H + h) * a.max_pages + page;
        if (page < a.max_pages) {
          const int32_t id = page < x.first ? *entry : page_at(pages_before[l] + (int64_t)h * x.fresh + page - x.first);
          if (page >= x.first && off == 0) *entry = id;
          if (id >= 0) slot = (int64_t)id * a.page_size + off;
        }
      }
      if (i < a.slots_per_seq) a.slots[(int64_t)b * a.slots_per_seq + i] = slot;
    }
  } else {
    const int64_t first = pages_before[0], all = pages_before[a.L] - first;
    for (int64_t i = begin; i < all; i += step) {
      const int l = layer_of(pages_before, first + i);
      const Held x = held[l];
      const int64_t in = first + i - pages_before[l];      // < H * fresh
      const int h = head_of(in, x.fresh), page = x.first + (int)(in - (int64_t)h * x.fresh);
      a.table[((int64_t)(b * a.L + l) * a.H + h) * a.max_pages + page] = page_at(first + i);
    }
  }
  if (a.finish && blockIdx.x == 0) {                       // (outputs of their own, or no other workgroup reads the inputs)
    __syncthreads();
    for (int l = tid; l < a.L; l += kPageThreads) a.rows_out[b * a.L + l] = held[l].grown;
    if (b == a.B - 1 && tid == 0) a.cursor_out[0] = cursor + pages_before[a.L];
  }
}

// Rows and cursor in place, once every workgroup of the launch before has read them.
__global__ __launch_bounds__(kPageThreads) void grow_rows_kernel(PageArgs a) {
  __shared__ int64_t sums[kPageThreads / 64];
  int64_t pages = 0;
  for (int i = threadIdx.x; i < a.B * a.L; i += kPageThreads) {
    const Held x = held_at(a, i);
    pages += x.fresh;
    a.rows_out[i] = x.grown;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) pages += __shfl_xor(pages, d, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = pages;
  __syncthreads();
  if (threadIdx.x == 0) {
    pages = 0;
    for (int w = 0; w < kPageThreads / 64; ++w) pages += sums[w];
    a.cursor_out[0] = a.cursor[0] + pages * a.H;
  }
}

}  // namespace

hipError_t assign_pages_launch(const int32_t* rows, const int32_t* add, int32_t add_each, int B, int L, int H, int page_size,
                               int max_pages, const int32_t* free_pages, int64_t num_free, int32_t* table, const int64_t* cursor,
                               int64_t* slots, int64_t slots_per_seq, int32_t* rows_out, int64_t* cursor_out, hipStream_t s) {
  // a thread has up to four rows, or pages of a table whose units are full
  const int64_t work = slots ? slots_per_seq : (int64_t)L * H * max_pages;
  const unsigned shares = (unsigned)std::min<int64_t>(4096, std::max<int64_t>(1, (work + 4 * kPageThreads - 1) / (4 * kPageThreads)));
  const bool in_place = rows_out == rows || cursor_out == cursor, alone = shares == 1 && B == 1;
  PageArgs a{rows, add, rows_out, free_pages, table, cursor, cursor_out, slots, num_free, slots_per_seq, B, L, H, page_size,
             page_size & (page_size - 1) ? -1 : __builtin_ctz((unsigned)page_size), max_pages, add_each, !in_place || alone};
  const size_t lds = (size_t)(L + 1) * 2 * sizeof(int64_t) + (size_t)L * sizeof(Held);
  {
    ProfileScope ps("assign_pages_kernel", s);
    if (slots) hipLaunchKernelGGL(assign_pages_kernel<true>, dim3(shares, B), dim3(kPageThreads), lds, s, a);
    else hipLaunchKernelGGL(assign_pages_kernel<false>, dim3(shares, B), dim3(kPageThreads), lds, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.finish) return e;
  ProfileScope ps("grow_rows_kernel", s);
  hipLaunchKernelGGL(grow_rows_kernel, dim3(1), dim3(kPageThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace fc
