// Rotary positions: the angle of a (position, frequency), its cosine and sine, and the
// rotation of channel pairs, shared by the query rotation, the appends that rotate their
// keys and the decode step that rotates both.
//
// Pair i of a head turns by th = fl64(pos[axis_i] * f_i): (x0, x1) -> m (x0 cos th - x1
// sin th, x1 cos th + x0 sin th).  Everything is fp64 and the result is rounded to bf16
// once, so that the same inputs give the same bits in every kernel here and in any other
// fp64 evaluation (an error of 2^-50 of a value crosses a bf16 rounding boundary once in
// 2^41), and the FP8 pages of a rotated append equal those of a rotation followed by a
// plain append.  In fp32 the angle of position 10^6 would be off by 2^-5.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mkv {

constexpr int ROPE_MAX_AXES = 4;

// One entry per frequency: what a lane needs of it in one 16-byte load.
struct RopeEntry {
  double freq;
  int32_t axis, pad;
};
struct RopeView {
  const RopeEntry* tab;  // device [rot / 2]
  double scale;          // m
  int rot, n_axes, interleaved;
};

// cos and sin of th in (-2^34, 2^34), times m.  k = the nearest multiple of pi/2; th - k
// P1 is exact (a multiple of 2^-52 below 1), k P2 corrects P1's rounding; then the Taylor
// series of both on |r| <= pi/4 to below 2^-58.
__device__ __forceinline__ void rope_cos_sin(double th, double m, double& c, double& s) {
#pragma clang fp contract(off)
  const double k = rint(th * 0x1.45f306dc9c883p-1);  // 2 / pi
  double r = __builtin_fma(-k, 0x1.921fb54442d18p+0, th);  // pi / 2 in two parts
  r = __builtin_fma(-k, 0x1.1a62633145c07p-54, r);
  const double z = r * r;
  double a = 1.0 / 355687428096000.0;  // 1 / 17!, 1 / 15!, ...
  a = __builtin_fma(a, z, -1.0 / 1307674368000.0);
  a = __builtin_fma(a, z, 1.0 / 6227020800.0);
  a = __builtin_fma(a, z, -1.0 / 39916800.0);
  a = __builtin_fma(a, z, 1.0 / 362880.0);
  a = __builtin_fma(a, z, -1.0 / 5040.0);
  a = __builtin_fma(a, z, 1.0 / 120.0);
  a = __builtin_fma(a, z, -1.0 / 6.0);
  const double sn = __builtin_fma(a * z, r, r);
  double b = 1.0 / 20922789888000.0;  // 1 / 16!, 1 / 14!, ...
  b = __builtin_fma(b, z, -1.0 / 87178291200.0);
  b = __builtin_fma(b, z, 1.0 / 479001600.0);
  b = __builtin_fma(b, z, -1.0 / 3628800.0);
  b = __builtin_fma(b, z, 1.0 / 40320.0);
  b = __builtin_fma(b, z, -1.0 / 720.0);
  b = __builtin_fma(b, z, 1.0 / 24.0);
  b = __builtin_fma(b, z, -0.5);
  const double cn = __builtin_fma(b, z, 1.0);
  // quadrant k mod 4 (|k| < 2^34): swap, then the signs
  const int q = (int)(int64_t)k & 3;
  const double cu = q & 1 ? sn : cn, su = q & 1 ? cn : sn;
  c = ((q + 1) & 2 ? -cu : cu) * m;
  s = (q & 2 ? -su : su) * m;
}

__device__ __forceinline__ void rope_rotate(double x0, double x1, double c, double s, double& y0, double& y1) {
#pragma clang fp contract(off)
  y0 = __builtin_fma(x0, c, -(x1 * s));
  y1 = __builtin_fma(x1, c, x0 * s);
}

// fp64 -> bf16 in one rounding, to nearest even, as the fp32 of that value.  Adding and
// taking away M = 1.5 * 2^(e + 45), e the exponent of x, leaves x rounded to multiples of
// 2^(e - 7): eight significant bits.  e is at least -126, where bf16's subnormals begin
// (their step is 2^-133), overflow is left to the conversion (the rounded value has eight
// bits, so it is exact or infinite), and x = inf or NaN survives both steps, whatever M.
// Seven instructions; through fp32 rounded to odd it took fourteen.
__device__ __forceinline__ float f64_round_bf16(double x) {
#pragma clang fp contract(off)
  const uint32_t h = (uint32_t)(__builtin_bit_cast(uint64_t, x) >> 32);
  const uint32_t e = max(h & 0x7FF00000u, (1023u - 126u) << 20);
  const double m = __builtin_bit_cast(double, (uint64_t)(e + (45u << 20) + 0x80000u) << 32);
  return __builtin_copysignf((float)((x + m) - m), __uint_as_float(h));
}
// two such values -> bf16 bits, b above a
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ uint32_t f64_to_bf16(double x) { return __float_as_uint(f64_round_bf16(x)) >> 16; }

// position of a token on an axis: entry `row` of [n_axes][n], or its place in the cache
__device__ __forceinline__ double rope_pos(const int32_t* pos, int64_t n, int64_t row, int axis, int at) {
  return (double)(pos ? pos[(int64_t)axis * n + row] : at);
}

// where the pair of frequency i sits
__device__ __forceinline__ int2 rope_pair(const RopeView& R, int i) {
  return R.interleaved ? make_int2(2 * i, 2 * i + 1) : make_int2(i, i + R.rot / 2);
}
// and the pair of channel c: its frequency, the other channel, whether c is the upper one
__device__ __forceinline__ void rope_of_channel(const RopeView& R, int c, int& freq, int& partner, bool& upper) {
  const int m = R.rot / 2;
  if (R.interleaved) {
    freq = c >> 1;
    partner = c ^ 1;
    upper = c & 1;
  } else {
    upper = c >= m;
    freq = upper ? c - m : c;
    partner = upper ? c - m : c + m;
  }
}

// Rows by D / (2 V) lanes, V = 4, 2 or 1 (rot / 2 a multiple of V): lane j holds V whole
// pairs, in two groups of V neighbouring channels, so it turns them by itself: V j .. and
// rot / 2 + V j .. (halves), 2 V j .. and 2 V j + V .. (neighbours); lanes past the rotated
// channels hold the others, two groups each.
template <int V>
struct RopeGroup;
template <> struct RopeGroup<4> { typedef uint2 type; };
template <> struct RopeGroup<2> { typedef uint32_t type; };
template <> struct RopeGroup<1> { typedef uint16_t type; };

inline int rope_width(int rot) { return rot % 8 == 0 ? 4 : rot % 4 == 0 ? 2 : 1; }

template <int V>
__device__ __forceinline__ bool rope_lane(const RopeView& R, int j, int& ca, int& cb) {
  const int m = R.rot / 2;
  const bool turn = j < m / V;
  ca = 2 * V * j;
  cb = ca + V;
  if (!R.interleaved) {
    ca = turn ? V * j : R.rot + 2 * V * (j - m / V);
    cb = turn ? m + V * j : ca + V;
  }
  return turn;
}
// the two groups as V words of two values; these as 2 V fp32 values, and back
__device__ __forceinline__ void rope_words(uint2 a, uint2 b, uint32_t (&w)[4]) { w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y; }
__device__ __forceinline__ void rope_words(uint32_t a, uint32_t b, uint32_t (&w)[2]) { w[0] = a, w[1] = b; }
__device__ __forceinline__ void rope_words(uint16_t a, uint16_t b, uint32_t (&w)[1]) { w[0] = a | (uint32_t)b << 16; }
template <int V>
__device__ __forceinline__ void rope_groups(const uint32_t (&w)[V], typename RopeGroup<V>::type& a, typename RopeGroup<V>::type& b) {
  if constexpr (V == 4) a = make_uint2(w[0], w[1]), b = make_uint2(w[2], w[3]);
  else if constexpr (V == 2) a = w[0], b = w[1];
  else a = (uint16_t)w[0], b = (uint16_t)(w[0] >> 16);
}
template <int V>
__device__ __forceinline__ void rope_unpack(const uint32_t (&w)[V], float* x) {
#pragma unroll
  for (int q = 0; q < V; ++q) {
    x[2 * q] = __uint_as_float(w[q] << 16);
    x[2 * q + 1] = __uint_as_float(w[q] & 0xFFFF0000u);
  }
}
template <int V>
__device__ __forceinline__ void rope_pack(const float* x, uint32_t (&w)[V]) {
#pragma unroll
  for (int q = 0; q < V; ++q) w[q] = bf16_pair(x[2 * q], x[2 * q + 1]);
}
// the lane's pairs turned, cos_sin(q) those of pair q; the values are bf16 again
template <int V, bool NEAR, class F>
__device__ __forceinline__ void rope_turn(float* x, F cos_sin) {
#pragma unroll
  for (int q = 0; q < V; ++q) {
    constexpr int step = NEAR ? 2 : 1, other = NEAR ? 1 : V;
    const double2 cs = cos_sin(q);
    double y0, y1;
    rope_rotate((double)x[step * q], (double)x[step * q + other], cs.x, cs.y, y0, y1);
    x[step * q] = f64_round_bf16(y0);
    x[step * q + other] = f64_round_bf16(y1);
  }
}
template <int V, class F>
__device__ __forceinline__ void rope_turn(float* x, bool interleaved, F cos_sin) {
  if (interleaved) rope_turn<V, true>(x, cos_sin);
  else rope_turn<V, false>(x, cos_sin);
}

}  // namespace mkv
