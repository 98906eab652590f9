// Shaped attention scores: a cap by a tanh, a bias by the distance, the tokens that a query
// sees, a sink per head; shared by the decode and chunk kernels.  Scores are in base-2 units
// here, s log2(e).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mkv {

struct ShapeView {
  float cap, icap;        // cap in base-2 units (0: none) and its inverse
  float scale;            // softmax scale, 0: 1 / sqrt(d)
  int window;             // a query at p sees keys past p - window (0: all)
  const float* slopes;    // device [n_q_heads] or null
  const float* sinks;     // device [n_q_heads] or null
  const int32_t* first;   // device, per query row, or null: keys below are not seen
  const int32_t* prefix;  // device, per request, or null (chunk): length of the part seen from both sides
};

constexpr float LOG2E_F = 1.4426950408889634f;

// kinds of shaped instances: masks alone; a bias by the distance; a cap; any of them
enum { SHAPE_MASK = 1, SHAPE_BIAS = 2, SHAPE_CAP = 3, SHAPE_ALL = 4 };

// cap tanh(x / cap) in fp32.  Below 0.55 cap as x + x z p(z), z = (x / cap)^2, p the odd polynomial's rest
// (least squares of the relative error: 1.1 2^-24), so that only the sum's rounding is one of x's size;
// above as cap (1 - 2 / (e^2t + 1)), t = x / cap, where the quotient is at most half of the result's size, so
// the hardware's exponential and reciprocal (an ulp each) leave less than 2 ulp.
constexpr float TANH_SMALL = 0.55f;
__device__ __forceinline__ float shape_cap_small(float x, float t) {
  const float z = t * t;
  float p = -0x1.9a8aa8p-8f;
  p = fmaf(p, z, 0x1.591d64p-6f);
  p = fmaf(p, z, -0x1.b92442p-5f);
  p = fmaf(p, z, 0x1.110d0ap-3f);
  p = fmaf(p, z, -0x1.55554ap-2f);
  return fmaf(x * z, p, x);
}
__device__ __forceinline__ float shape_cap_large(float cap, float t) {
  const float e = __builtin_amdgcn_exp2f(fabsf(t) * (2.0f * LOG2E_F));
  return cap * copysignf(fmaf(-2.0f, __builtin_amdgcn_rcpf(e + 1.0f), 1.0f), t);  // (NaN stays)
}
// a score, capped
__device__ __forceinline__ float shape_cap(const ShapeView& s, float x) {
  const float t = x * s.icap;
  return fabsf(t) < TANH_SMALL ? shape_cap_small(x, t) : shape_cap_large(s.cap, t);
}
// N scores of every lane, capped, and a bias; the wave leaves the second form out where none of them
// takes it (a NaN may be either's)
template <int N>
__device__ __forceinline__ void shape_cap(const ShapeView& s, float* x, float bias) {
  float t[N], big = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    t[i] = x[i] * s.icap;
    big = fmaxf(big, fabsf(t[i]));
    x[i] = shape_cap_small(x[i], t[i]);
  }
  if (__any(!(big < TANH_SMALL))) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fabsf(t[i]) < TANH_SMALL ? x[i] : shape_cap_large(s.cap, t[i]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] += bias;
}

}  // namespace mkv
