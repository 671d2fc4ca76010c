// Rotary positions of the queries and keys that a step or a prompt brings: pair i of a head is turned by the angle
// position * frequency_i,
//   y0 = m (x0 cos - x1 sin),  y1 = m (x1 cos + x0 sin)        (transposed: sin -> -sin)
// where a pair is (x_i, x_{i + R/2}) or (x_2i, x_2i+1) of the first R columns; the other columns are copied.
//
// Angles: a frequency is kept as turns per position in units of 2^-64, so that position * frequency is one product of
// integers whose overflow drops the whole turns: exact to 2^-53 of the frequency for any int32 position, where an angle in
// fp32 is off by 0.06 rad at position 10^6.  32 bits of the turn are left to an octant and the series of sine and cosine
// on |theta| <= pi / 4 (terms up to theta^9 and theta^8, whose rest is below 2^-25).
//
// Bound by memory: every element is read and written once.  A thread keeps the sines of its pairs (about 35 operations each) for four heads and
// more of its token, whose pieces are all loaded before the first is stored (behind a store the next load's wait is for the store too).  Pieces
// side by side in a wave are whole lines: of the halves 8 bytes a lane, of interleaved pairs 16.  32768 tokens of 28 and 4 heads of 128 columns in
// bf16 (0.54 GB in all), us: a head at a time 112, eight heads side by side 105, past the last-level cache 97, four loaded together 92,
// four pairs a thread in place of eight 88, 6.1 TB/s; interleaved pairs as two pieces of 16 bytes 151, as one 87; fp32 (1.07 GB) as 32
// bytes a lane 224, as 16 180.  Integer products of 64 bits take four times as long as others: heads' places by the wave and sequences that
// follow each other as one made 8192 tokens of 5 and 1 heads 9.1 / 7.9 us, 2048 of 28 and 4 10.5 / 9.5.
#include <algorithm>
#include <type_traits>
#include <math.h>
#include <string.h>

#include "fc_common.h"
#include "rotary.h"

namespace fc {

namespace {

constexpr int kRotThreads = 256;
constexpr int kHeadsAtOnce = 4, kMostPairs = 4, kMostAbreast = 8, kMostTurns = 8;

struct RotSide {                 // Q or K
  const char* in;
  char* out;
  int64_t sb, st, sh, ob, ot, oh;    // strides in bytes
  int heads;
};
struct RotArgs {
  RotSide q, k;
  const int32_t* positions;      // [streams][batch * tokens]
  int tokens, rows;              // tokens of a sequence, of all sequences
  int half, chunks, turned;      // pairs; chunks of a head; those that are turned
  int per_group;                 // tokens of a workgroup
  uint32_t chunks_inverse, abreast_inverse;
  bool flat;                     // the sequences follow each other as tokens do
  int abreast, turns;            // heads of a token side by side; how many of them a thread has, one after another
  int streams, end0, end1, end2; // first pair behind the first, second and third stream
  float magnitude, sign;
};

// P pairs a thread and head: a piece of P columns and its partners' half a head away, or, interleaved, one of 2 P columns; chunks behind the
// turned ones are copied, as pieces of the same kind.
template <typename T, int P, bool INTERLEAVED, bool PAST>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotArgs a, const fc_rotary_plan plan) {
  constexpr int kPieces = INTERLEAVED ? 1 : 2, kPiece = 2 * P / kPieces;     // pieces of a chunk, columns of a piece
  const int place = quotient(threadIdx.x, a.chunks_inverse), chunk = (int)threadIdx.x - place * a.chunks;
  const int own = quotient(place, a.abreast_inverse), beside = place - own * a.abreast;
  const int64_t row64 = (int64_t)blockIdx.x * a.per_group + own;
  if (own >= a.per_group || row64 >= a.rows) return;
  const int row = (int)row64;
  const bool turned = chunk < a.turned;
  float sn[P], cs[P];
  // bytes of the first piece from the head's begin on, and from it to the second
  const int at = (turned ? chunk * kPiece : 2 * a.half + (chunk - a.turned) * kPiece) * (int)sizeof(T);
  const int apart = (turned ? a.half : (a.chunks - a.turned) * P) * (int)sizeof(T);
  if (turned) {
    const int first = chunk * P;
    int32_t where[P];
    where[0] = a.positions[row];
#pragma unroll
    for (int i = 1; i < P; ++i) where[i] = where[0];
    if (a.streams > 1) {
      int32_t other[3];
#pragma unroll
      for (int k = 0; k < 3; ++k) other[k] = k + 1 < a.streams ? a.positions[(int64_t)(k + 1) * a.rows + row] : 0;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int pair = first + i;
        where[i] = pair < a.end0 ? where[i] : pair < a.end1 ? other[0] : pair < a.end2 ? other[1] : other[2];
      }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      sine_cosine(turned_by(where[i], plan.turns[first + i]), sn[i], cs[i]);
      sn[i] *= a.magnitude * a.sign;
      cs[i] *= a.magnitude;
    }
  }
  const int heads = a.q.heads + a.k.heads, h0 = (int)blockIdx.y * a.abreast * a.turns, h1 = min(heads, h0 + a.abreast * a.turns);
  // head `beside` of Q, and what would be that of Q and K as one
  int b = 0, t = row;
  if (!a.flat) {
    b = row / a.tokens;
    t = row - b * a.tokens;
  }
  int64_t q_in = t * a.q.st + beside * a.q.sh + at, q_out = t * a.q.ot + beside * a.q.oh + at;
  int64_t k_in = t * a.k.st + (beside - a.q.heads) * a.k.sh + at, k_out = t * a.k.ot + (beside - a.q.heads) * a.k.oh + at;
  if (!a.flat) {
    q_in += b * a.q.sb;
    q_out += b * a.q.ob;
    k_in += b * a.k.sb;
    k_out += b * a.k.ob;
  }
  for (int hw = h0; hw < h1; hw += kHeadsAtOnce * a.abreast) {
    Vec<T, kPiece> v[kHeadsAtOnce][kPieces];
    char* out[kHeadsAtOnce];
#pragma unroll
    for (int i = 0; i < kHeadsAtOnce; ++i) {
      const int hu = hw + i * a.abreast, h = hu + beside;  // (the first is the same for the wave)
      if (h >= h1) break;
      const bool is_q = h < a.q.heads;
      const char* const in = is_q ? a.q.in + hu * a.q.sh + q_in : a.k.in + hu * a.k.sh + k_in;
      out[i] = is_q ? a.q.out + hu * a.q.oh + q_out : a.k.out + hu * a.k.oh + k_out;
#pragma unroll
      for (int j = 0; j < kPieces; ++j) v[i][j] = get<PAST, T, kPiece>(in + j * apart);
    }
#pragma unroll
    for (int i = 0; i < kHeadsAtOnce; ++i) {
      if (hw + i * a.abreast + beside >= h1) break;
      if (turned) {
        float x[kPieces][kPiece], y[kPieces][kPiece];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) widen<T, kPiece>(v[i][j], x[j]);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          const int j = INTERLEAVED ? 0 : 1, c0 = INTERLEAVED ? 2 * k : k, c1 = INTERLEAVED ? 2 * k + 1 : k;
          y[0][c0] = x[0][c0] * cs[k] - x[j][c1] * sn[k];
          y[j][c1] = x[j][c1] * cs[k] + x[0][c0] * sn[k];
        }
#pragma unroll
        for (int j = 0; j < kPieces; ++j) v[i][j] = narrow<T, kPiece>(y[j]);
      }
#pragma unroll
      for (int j = 0; j < kPieces; ++j) put<PAST>(out[i] + j * apart, v[i][j]);
    }
  }
}

}  // namespace

hipError_t rotary_launch(const fc_rotary_plan& plan, const int32_t* positions, const void* Q, void* Q_out, const fc_heads_desc& q,
                         const void* K, void* K_out, const fc_heads_desc* k, bool inverse, hipStream_t s) {
  const int e = q.dtype == FC_BF16 ? 2 : 4, half = plan.rotary_dim / 2, rest = q.head_dim - plan.rotary_dim;
  // (the step of an axis of one says nothing: left out, as it would count in what addresses are multiples of)
  auto step = [&](int n, int64_t stride) { return n > 1 ? stride * e : 0; };
  auto side = [&](const void* in, void* out, const fc_heads_desc& d) {
    return RotSide{static_cast<const char*>(in), static_cast<char*>(out),
                   step(d.batch, d.stride_b), step(d.tokens, d.stride_t), step(d.heads, d.stride_h),
                   step(d.batch, d.out_stride_b), step(d.tokens, d.out_stride_t), step(d.heads, d.out_stride_h), d.heads};
  };
  RotArgs a{};
  a.q = side(Q, Q_out, q);
  a.k = k && k->heads ? side(K, K_out, *k) : RotSide{};
  // the widest parts that every address is a multiple of
  uint64_t bits = 0;
  for (const RotSide* r : {&a.q, &a.k})
    bits |= (uint64_t)(uintptr_t)r->in | (uint64_t)(uintptr_t)r->out | (uint64_t)(r->sb | r->st | r->sh | r->ob | r->ot | r->oh);
  const int pieces = plan.interleaved ? 1 : 2;             // (of a chunk: 16 bytes at most)
  int pairs = std::min(8 * pieces / e, kMostPairs);
  while (pairs > 1 && (half % pairs || rest % (2 * pairs) || (bits & (uint64_t)(2 * pairs / pieces * e - 1)))) pairs /= 2;
  a.positions = positions;
  a.tokens = q.tokens;
  a.rows = q.batch * q.tokens;
  a.flat = true;
  for (RotSide* r : {&a.q, &a.k}) {
    if (q.tokens == 1) {
      r->st = r->sb;
      r->ot = r->ob;
    } else if (q.batch > 1 && r->heads) {
      a.flat = a.flat && r->sb == q.tokens * r->st && r->ob == q.tokens * r->ot;
    }
  }
  a.half = half;
  a.turned = half / pairs;
  a.chunks = a.turned + rest / (2 * pairs);
  a.streams = plan.streams;
  a.end0 = plan.stream_end[0];
  a.end1 = plan.stream_end[1];
  a.end2 = plan.stream_end[2];
  a.magnitude = plan.magnitude;
  a.sign = inverse ? -1.f : 1.f;
  const int heads = a.q.heads + a.k.heads, places = kRotThreads / a.chunks;
  const int64_t one_turn = ((int64_t)a.rows * heads + places - 1) / places;    // workgroups if every thread has a single head
  // few tokens: all heads side by side, so that a step's launch is spread over the chip; else at least four turns, for which the sines are made
  // once (32768 tokens, us with eight side by side whatever there is / so: 8 heads of 128 columns 44 / 30, 10 of 64 26 / 17)
  int abreast = 1;
  while (abreast < kMostAbreast && 2 * abreast * kHeadsAtOnce <= heads) abreast *= 2;
  a.abreast = std::min(std::min(heads, places), one_turn > 2048 ? abreast : heads);
  a.turns = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(kMostTurns, (heads + a.abreast - 1) / a.abreast), one_turn / 2048));
  a.per_group = places / a.abreast;
  a.chunks_inverse = inverse_of(a.chunks);
  a.abreast_inverse = inverse_of(a.abreast);
  const dim3 grid((unsigned)(((int64_t)a.rows + a.per_group - 1) / a.per_group), (unsigned)((heads + a.abreast * a.turns - 1) / (a.abreast * a.turns)));
  ProfileScope ps("rotary_kernel", s);
  auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(kRotThreads), 0, s, a, plan); };
  // what is read and written exceeds the cache, in pieces of whole lines (half lines: 32 and 8 heads of 128 columns, 64 of them turned, 147 / 136)
  const bool past = 2LL * a.rows * heads * q.head_dim * e > 256000000 && (plan.interleaved || half * e % 128 == 0);
  auto with = [&](auto type, auto n, auto interleaved) {
    typedef decltype(type) T;
    past ? launch(rotary_kernel<T, decltype(n)::value, decltype(interleaved)::value, true>)
         : launch(rotary_kernel<T, decltype(n)::value, decltype(interleaved)::value, false>);
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

using namespace fc;

extern "C" {

// Host only.  Frequencies f_i = theta^(-2i / R), rescaled for contexts longer than the one trained on:
//   linear  f_i / s
//   base    theta * s^(R / (R - 2)) in place of theta
//   parts   a pair that makes n turns over the original context keeps f_i if n >= beta_fast, takes f_i / s if n <= beta_slow and a
//           mixture linear in n between; magnitude 0.1 ln s + 1
fc_status flashcache_rotary_prepare(const fc_rotary_spec* spec, const double* frequencies, fc_rotary_plan* plan) {
  if (!spec || !plan) return FC_EINVAL;
  const int R = spec->rotary_dim;
  if (R < 2 || R % 2) return FC_EINVAL;
  if (R > 2 * FC_ROTARY_MAX_PAIRS) return FC_EUNSUPPORTED;
  if (spec->streams < 1 || spec->streams > 4) return FC_EINVAL;
  if (spec->scaling < FC_ROTARY_PLAIN || spec->scaling > FC_ROTARY_PARTS) return FC_EINVAL;
  if (!frequencies && !(spec->theta > 0.0 && isfinite(spec->theta))) return FC_EINVAL;
  const bool scaled = !frequencies && spec->scaling != FC_ROTARY_PLAIN;
  if (scaled && !(spec->factor >= 1.0 && isfinite(spec->factor))) return FC_EINVAL;
  const bool parts = scaled && spec->scaling == FC_ROTARY_PARTS;
  if (parts && (spec->original_tokens < 1 || !(spec->beta_fast > spec->beta_slow) || !isfinite(spec->beta_fast) || !isfinite(spec->beta_slow)))
    return FC_EINVAL;
  if (!(spec->magnitude >= 0.0 && isfinite(spec->magnitude))) return FC_EINVAL;
  fc_rotary_plan p;
  memset(&p, 0, sizeof(p));
  p.rotary_dim = R;
  p.interleaved = spec->interleaved != 0;
  p.streams = spec->streams;
  int end = 0;
  for (int k = 0; k < 4; ++k) {
    if (k < spec->streams) {
      const int n = spec->streams == 1 ? R / 2 : spec->stream_pairs[k];
      if (n < 0 || n > R / 2) return FC_EINVAL;
      end += n;
    }
    p.stream_end[k] = k < spec->streams - 1 ? end : R / 2;
  }
  if (end != R / 2) return FC_EINVAL;
  const double pi = 3.14159265358979323846, s = scaled ? spec->factor : 1.0;
  p.magnitude = (float)(spec->magnitude > 0.0 ? spec->magnitude : parts ? 0.1 * log(s) + 1.0 : 1.0);
  const double theta = scaled && spec->scaling == FC_ROTARY_BASE && R > 2 ? spec->theta * pow(s, (double)R / (R - 2)) : spec->theta;
  for (int i = 0; i < R / 2; ++i) {
    double f = frequencies ? frequencies[i] : pow(theta, -2.0 * i / R);
    if (!isfinite(f)) return FC_EINVAL;
    if (scaled && spec->scaling == FC_ROTARY_LINEAR) f /= s;
    if (parts) {
      const double n = spec->original_tokens * f / (2.0 * pi);
      const double keep = fmin(1.0, fmax(0.0, (n - spec->beta_slow) / (spec->beta_fast - spec->beta_slow)));
      f = f * keep + f / s * (1.0 - keep);
    }
    const double turns = f / (2.0 * pi), part = turns - floor(turns);      // (whole turns a position change nothing)
    const double units = ldexp(part, 64);
    p.turns[i] = units >= 18446744073709551616.0 ? 0u : (uint64_t)units;
  }
  p.magic = kWsMagic;
  *plan = p;
  return FC_OK;
}

}  // extern "C"
