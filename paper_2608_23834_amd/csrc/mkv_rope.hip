// Rotation of bf16 rows by their tokens' positions (queries; keys where the caller keeps
// them elsewhere).  See mkv_rope.h for the mathematics and the precision.
#include <hip/hip_runtime.h>

#include "mkv_internal.h"
#include "mkv_rope.h"

namespace mkv {

// D / (2 V) lanes share a (token, block of hb heads): a lane evaluates the angles of its V
// pairs, keeps their cosines and sines in registers and turns its pairs of every head of the
// block; lanes past the rotated channels copy.  Each lane reads what it writes, so in place
// works.  Memory bound from some thousand rows on (16,384 tokens of 24 heads at d = 256: 403 MB
// in 86 us, a copy of them takes 74); with one head in flight instead of four it took 100.
template <int D, int V>
__global__ __launch_bounds__(256) void rope_apply_kernel(RopeView R, int64_t t0, int n_here, int n_tokens, int n_heads, int hb,
                                                         const uint16_t* x, int64_t xs, const int32_t* pos,
                                                         uint16_t* out, int64_t os) {
  typedef typename RopeGroup<V>::type group;
  constexpr int LT = D / (2 * V), HU = 4;  // lanes of a token; heads in flight
  const int nb = (n_heads + hb - 1) / hb;
  const int64_t unit = (int64_t)blockIdx.x * (256 / LT) + threadIdx.x / LT;
  if (unit >= (int64_t)n_here * nb) return;
  const int j = threadIdx.x % LT;
  const int64_t tu = unit / nb, t = t0 + tu;
  const int h0 = (int)(unit - tu * nb) * hb, h1 = min(h0 + hb, n_heads);
  int ca, cb;
  const bool turn = rope_lane<V>(R, j, ca, cb);
  double c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    c[i] = 1.0;
    s[i] = 0.0;
    if (turn) {
      const RopeEntry e = R.tab[V * j + i];
      rope_cos_sin((double)pos[(int64_t)e.axis * n_tokens + t] * e.freq, R.scale, c[i], s[i]);
    }
  }
  const uint16_t* xr = x + t * xs;
  uint16_t* orow = out + t * os;
  for (int hu = h0; hu < h1; hu += HU) {
    group a[HU], b[HU];
#pragma unroll
    for (int k = 0; k < HU; ++k) {
      const uint16_t* xh = xr + (int64_t)min(hu + k, h1 - 1) * D;
      a[k] = *reinterpret_cast<const group*>(xh + ca);
      b[k] = *reinterpret_cast<const group*>(xh + cb);
    }
#pragma unroll
    for (int k = 0; k < HU; ++k) {
      if (hu + k >= h1) break;
      if (turn) {
        float v[2 * V];
        uint32_t w[V];
        rope_words(a[k], b[k], w);
        rope_unpack<V>(w, v);
        rope_turn<V>(v, R.interleaved, [&](int i) { return make_double2(c[i], s[i]); });
        rope_pack<V>(v, w);
        rope_groups<V>(w, a[k], b[k]);
      }
      uint16_t* oh = orow + (int64_t)(hu + k) * D;
      *reinterpret_cast<group*>(oh + ca) = a[k];
      *reinterpret_cast<group*>(oh + cb) = b[k];
    }
  }
}

hipError_t launch_rope_apply(const RopeView& R, int d, int n_tokens, int n_heads, const uint16_t* x, int64_t xs,
                             const int32_t* pos, uint16_t* out, int64_t os, hipStream_t s) {
  // heads per lane group: all of them once that fills the chip (eight waves per SIMD), so
  // that an angle serves every head
  const int V = rope_width(R.rot), lt = d / (2 * V), per = 256 / lt;
  int64_t nb = ((int64_t)8192 * 64 / lt + n_tokens - 1) / n_tokens;
  if (nb > n_heads) nb = n_heads;
  const int hb = (int)((n_heads + nb - 1) / nb);
  auto go = [&](auto kern) {
    // (a launch holds 2^32 threads at most: 2^22 tokens and up to 8192 * 64 lanes' worth of
    // head blocks stay below 2^30)
    for (int64_t t0 = 0; t0 < n_tokens; t0 += 1 << 22) {
      const int n_here = (int)(n_tokens - t0 < 1 << 22 ? n_tokens - t0 : 1 << 22);
      const int64_t units = (int64_t)n_here * ((n_heads + hb - 1) / hb);
      hipLaunchKernelGGL(kern, dim3((unsigned)((units + per - 1) / per)), dim3(256), 0, s, R, t0, n_here, n_tokens,
                         n_heads, hb, x, xs, pos, out, os);
    }
  };
  if (d == 256)
    V == 4 ? go(rope_apply_kernel<256, 4>) : V == 2 ? go(rope_apply_kernel<256, 2>) : go(rope_apply_kernel<256, 1>);
  else
    V == 4 ? go(rope_apply_kernel<128, 4>) : V == 2 ? go(rope_apply_kernel<128, 2>) : go(rope_apply_kernel<128, 1>);
  return hipGetLastError();
}

}  // namespace mkv
