// Rotation of bf16 rows by their tokens' positions (queries; keys where the caller keeps
// them elsewhere).  See mkv_rope.h for the mathematics and the precision.
#include <hip/hip_runtime.h>

#include "mkv_internal.h"
#include "mkv_rope.h"

namespace mkv {

// D / 8 lanes share a (token, block of hb heads): a lane owns two groups of four channels,
// the two halves of four pairs where rot / 2 comes in fours (VEC), so it evaluates four
// angles, keeps their cosines and sines in registers and turns its pairs of every head of
// the block; lanes past the rotated channels copy.  !VEC: channels 8 j .., the other half
// of each pair is loaded again (by the same wave, before it stores: in place works).
template <int D, bool VEC>
__global__ __launch_bounds__(256) void rope_apply_kernel(RopeView R, int n_tokens, int n_heads, int hb,
                                                         const uint16_t* x, int64_t xs, const int32_t* pos,
                                                         uint16_t* out, int64_t os) {
  constexpr int LT = D / 8, NF = VEC ? 4 : 8;
  const int nb = (n_heads + hb - 1) / hb;
  const int64_t unit = (int64_t)blockIdx.x * (256 / LT) + threadIdx.x / LT;
  if (unit >= (int64_t)n_tokens * nb) return;
  const int j = threadIdx.x % LT, m = R.rot / 2;
  const int64_t t = unit / nb;
  const int h0 = (int)(unit - t * nb) * hb, h1 = min(h0 + hb, n_heads);
  const bool turn = VEC ? j < m / 4 : 8 * j < R.rot;
  int ca = 8 * j, cb = 8 * j + 4;
  if (VEC && !R.interleaved) {
    ca = turn ? 4 * j : R.rot + 8 * (j - m / 4);
    cb = turn ? m + 4 * j : ca + 4;
  }
  int pc[8];
  bool up[8];
  double c[NF], s[NF];
#pragma unroll
  for (int i = 0; i < NF; ++i) {
    c[i] = 1.0;
    s[i] = 0.0;
    int f = 4 * j + i;
    pc[i] = 8 * j + i;
    up[i] = false;
    const bool in = VEC ? turn : 8 * j + i < R.rot;
    if (!VEC && in) rope_of_channel(R, 8 * j + i, f, pc[i], up[i]);
    if (in) {
      const RopeEntry e = R.tab[f];
      rope_cos_sin((double)pos[(int64_t)e.axis * n_tokens + t] * e.freq, R.scale, c[i], s[i]);
    }
  }
  // the rows of HU heads are in flight together
  constexpr int HU = 4;
  const uint16_t* xr = x + t * xs;
  uint16_t* orow = out + t * os;
  for (int hu = h0; hu < h1; hu += HU) {
    uint2 a[HU], b[HU];
#pragma unroll
    for (int k = 0; k < HU; ++k) {
      const uint16_t* xh = xr + (int64_t)min(hu + k, h1 - 1) * D;
      a[k] = *reinterpret_cast<const uint2*>(xh + ca);
      b[k] = *reinterpret_cast<const uint2*>(xh + cb);
    }
#pragma unroll
    for (int k = 0; k < HU; ++k) {
      if (hu + k >= h1) break;
      const uint32_t w[4] = {a[k].x, a[k].y, b[k].x, b[k].y};
      uint32_t o[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[2 * i] = w[i] << 16;
        o[2 * i + 1] = w[i] & 0xFFFF0000u;
      }
      if (turn) {
        auto val = [&](int i) { return (double)__uint_as_float(o[i]); };
        auto put = [&](int i, double y) { o[i] = __float_as_uint(f64_round_bf16(y)); };
        if constexpr (VEC) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int u = 2 * i, v = 2 * i + 1;
            double y0, y1;
            if (R.interleaved) {
              rope_rotate(val(u), val(v), c[i], s[i], y0, y1);
              put(u, y0);
              put(v, y1);
            } else {
              rope_rotate(val(i), val(i + 4), c[i], s[i], y0, y1);
              put(i, y0);
              put(i + 4, y1);
            }
          }
        } else {
          const uint16_t* xh = xr + (int64_t)(hu + k) * D;
          uint16_t other[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) other[i] = xh[pc[i]];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (8 * j + i >= R.rot) continue;
            const double xo = val(i), xp = (double)bf16_to_f32(other[i]);
            double y0, y1;
            rope_rotate(up[i] ? xp : xo, up[i] ? xo : xp, c[i], s[i], y0, y1);
            put(i, up[i] ? y1 : y0);
          }
        }
      }
      uint16_t* oh = orow + (int64_t)(hu + k) * D;
      *reinterpret_cast<uint2*>(oh + ca) = make_uint2(o[0] >> 16 | o[1], o[2] >> 16 | o[3]);
      *reinterpret_cast<uint2*>(oh + cb) = make_uint2(o[4] >> 16 | o[5], o[6] >> 16 | o[7]);
    }
  }
}

hipError_t launch_rope_apply(const RopeView& R, int d, int n_tokens, int n_heads, const uint16_t* x, int64_t xs,
                             const int32_t* pos, uint16_t* out, int64_t os, hipStream_t s) {
  if (n_tokens == 0) return hipSuccess;
  // heads per lane group: all of them once that fills the chip (eight waves per SIMD), so
  // that an angle serves every head
  const int lt = d / 8, per = 256 / lt;
  int64_t nb = ((int64_t)8192 * 64 / lt + n_tokens - 1) / n_tokens;
  if (nb > n_heads) nb = n_heads;
  const int hb = (int)((n_heads + nb - 1) / nb);
  const int64_t units = (int64_t)n_tokens * ((n_heads + hb - 1) / hb);
  const dim3 grid((unsigned)((units + per - 1) / per));
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, R, n_tokens, n_heads, hb, x, xs, pos, out, os);
  };
  const bool vec = R.rot % 8 == 0;
  if (d == 256)
    vec ? go(rope_apply_kernel<256, true>) : go(rope_apply_kernel<256, false>);
  else
    vec ? go(rope_apply_kernel<128, true>) : go(rope_apply_kernel<128, false>);
  return hipGetLastError();
}

}  // namespace mkv
