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

// tanh in fp32: an odd polynomial below 0.55 (least squares of the relative error: 1.1 2^-24),
// 1 - 2 / (e^2x + 1) above, where the quotient is at most half of the result's size, so the
// hardware's exponential and reciprocal (an ulp each) leave less than 2 ulp.
__device__ __forceinline__ float shape_tanh(float x) {
  const float z = x * x;
  float p = -0x1.9a8aa8p-8f;
  p = fmaf(p, z, 0x1.591d64p-6f);
  p = fmaf(p, z, -0x1.b92442p-5f);
  p = fmaf(p, z, 0x1.110d0ap-3f);
  p = fmaf(p, z, -0x1.55554ap-2f);
  const float a = fabsf(x);
  const float e = __builtin_amdgcn_exp2f(a * (2.0f * LOG2E_F));
  const float t = fmaf(-2.0f, __builtin_amdgcn_rcpf(e + 1.0f), 1.0f);
  return a < 0.55f ? fmaf(x * z, p, x) : copysignf(t, x);  // (NaN stays)
}
// a score, capped where there is a cap
__device__ __forceinline__ float shape_cap(const ShapeView& s, float x) { return s.cap * shape_tanh(x * s.icap); }

}  // namespace mkv
