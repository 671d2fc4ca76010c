// Pieces of rows and the sines of positions, for the kernels that turn queries and keys.
#ifndef FC_ROTARY_H_
#define FC_ROTARY_H_

#include "fc_common.h"

namespace fc {

namespace {

// n / d for n and d up to 256, with d's inverse in 16 bits, rounded up
__host__ __device__ __forceinline__ uint32_t inverse_of(int d) { return (65536u + (uint32_t)d - 1u) / (uint32_t)d; }
__device__ __forceinline__ int quotient(uint32_t n, uint32_t inverse) { return (int)(n * inverse >> 16); }

template <int BYTES> struct Bytes;
template <> struct Bytes<2> { typedef uint16_t type; };
template <> struct Bytes<4> { typedef uint32_t type; };
template <> struct Bytes<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Bytes<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };

template <typename T, int N> struct Vec {
  typename Bytes<N * (int)sizeof(T)>::type raw;
};
template <typename T, int N> __device__ __forceinline__ void widen(const Vec<T, N>& v, float (&o)[N]) {
  if constexpr (sizeof(T) == 4) {
    struct F { float f[N]; };
    const F f = __builtin_bit_cast(F, v.raw);
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = f.f[i];
  } else {
    struct H { uint16_t h[N]; };
    const H h = __builtin_bit_cast(H, v.raw);
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = bf16_to_f32(h.h[i]);
  }
}
template <typename T, int N> __device__ __forceinline__ Vec<T, N> narrow(const float (&x)[N]) {
  Vec<T, N> v;
  if constexpr (sizeof(T) == 4) {
    struct F { float f[N]; } f;
#pragma unroll
    for (int i = 0; i < N; ++i) f.f[i] = x[i];
    v.raw = __builtin_bit_cast(decltype(v.raw), f);
  } else {                                                 // (the one rounding: to nearest)
    struct H { __bf16 h[N]; } h;
#pragma unroll
    for (int i = 0; i < N; ++i) h.h[i] = (__bf16)x[i];
    v.raw = __builtin_bit_cast(decltype(v.raw), h);
  }
  return v;
}

// PAST: past the last-level cache.
template <bool PAST, typename T, int N> __device__ __forceinline__ Vec<T, N> get(const char* p) {
  const Vec<T, N>* const at = reinterpret_cast<const Vec<T, N>*>(p);
  Vec<T, N> v;
  if constexpr (PAST) v.raw = __builtin_nontemporal_load(&at->raw);
  else v = *at;
  return v;
}
template <bool PAST, typename T, int N> __device__ __forceinline__ void put(char* p, const Vec<T, N>& v) {
  Vec<T, N>* const at = reinterpret_cast<Vec<T, N>*>(p);
  if constexpr (PAST) __builtin_nontemporal_store(v.raw, &at->raw);
  else *at = v;
}

// Sine and cosine of `turns` 2^-32 of a whole turn.
__device__ __forceinline__ void sine_cosine(uint32_t turns, float& s, float& c) {
  const uint32_t quarter = (turns + 0x20000000u) >> 30;
  const float t = (float)(int32_t)(turns - (quarter << 30)) * 1.4629180792671596e-9f;      // 2 pi / 2^32
  const float u = t * t;
  const float a = t * fmaf(u, fmaf(u, fmaf(u, fmaf(u, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
  const float b = fmaf(u, fmaf(u, fmaf(u, fmaf(u, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const float x = quarter & 1 ? b : a, y = quarter & 1 ? a : b;
  s = quarter & 2 ? -x : x;
  c = (quarter + 1) & 2 ? -y : y;
}

// The part of a turn, in units of 2^-32, that a pair of `turns` 2^-64 turns a position makes up to position `where`: the upper half of the product,
// rounded (what the lower halves' product carries, and less 2^32 times the turns for a negative position).
__device__ __forceinline__ uint32_t turned_by(int32_t where, uint64_t turns) {
  const uint32_t low = (uint32_t)turns, high = (uint32_t)(turns >> 32), pos = (uint32_t)where;
  const uint64_t carried = (uint64_t)pos * low + 0x80000000ull;
  return pos * high + (uint32_t)(carried >> 32) - (where < 0 ? low : 0u);
}

}  // namespace

}  // namespace fc
#endif
