// Rotation of bf16 rows by their tokens' positions (queries; keys where the caller keeps
// them elsewhere), alone or behind a norm of every head.  See mkv_rope.h for the mathematics and the precision.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "mkv_internal.h"
#include "mkv_norm.h"
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

// rope_apply_kernel with every head normed and weighted first.  The lanes of a row add up its
// squares over lane exchanges; U = 2 where a row has more lanes than a wave (d = 256, pairs of
// one): a lane then holds two of them.  Bound by the rows' way through memory, and behind it by the
// instructions of the norm: 16,384 tokens of 24 heads, d = 256, all channels turned (403 MB, 79 us
// of a copy's bandwidth): 95 us with weights of every head, 87 with shared ones.  Two heads in flight,
// because a third would not fit beside the converted values, which the sum of squares and the product
// both take (four in flight and the values converted twice: 112).
template <int D, int V, bool NEAR>
__global__ __launch_bounds__(256, 4) void norm_rope_apply_kernel(RopeView R, NormView N, int64_t t0, int n_here, int n_tokens,
                                                              int n_heads, int hb, const uint16_t* x, int64_t xs,
                                                              const int32_t* pos, uint16_t* out, int64_t os) {
  typedef typename RopeGroup<V>::type group;
  constexpr int U = D / (2 * V) > 64 ? 2 : 1, LT = D / (2 * V) / U, HU = 2;
  const int nb = (n_heads + hb - 1) / hb;
  const int64_t unit = (int64_t)blockIdx.x * (256 / LT) + threadIdx.x / LT;
  if (unit >= (int64_t)n_here * nb) return;  // (all lanes of a row, so exchanges stay among those that are here)
  const int lane = threadIdx.x & 63, j = threadIdx.x % LT;
  const int64_t tu = unit / nb, t = t0 + tu;
  const int h0 = (int)(unit - tu * nb) * hb, h1 = min(h0 + hb, n_heads);
  int ca[U], cb[U];
  bool turn[U];
#pragma unroll
  for (int u = 0; u < U; ++u) turn[u] = rope_lane<V>(R, j + u * LT, ca[u], cb[u]);
  const uint16_t* xr = x + t * xs;
  uint16_t* orow = out + t * os;
  uint32_t w[HU][U][V], ww[HU][U][V];  // two heads' values and weights, loaded while the two before are in work
  auto load = [&](int hu) {
#pragma unroll
    for (int k = 0; k < HU; ++k)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = min(hu + k, h1 - 1);
        const uint16_t* xh = xr + (int64_t)h * D;
        rope_words(*reinterpret_cast<const group*>(xh + ca[u]), *reinterpret_cast<const group*>(xh + cb[u]), w[k][u]);
        if (N.head) {
          const uint16_t* wh = N.w + h * N.head;
          rope_words(*reinterpret_cast<const group*>(wh + ca[u]), *reinterpret_cast<const group*>(wh + cb[u]), ww[k][u]);
        }
      }
  };
  load(h0);
  double wd[U][2 * V];  // weights of the head in work, of every head where they are the same
  auto weigh = [&](int u, const uint32_t (&a)[V]) {
    float f[2 * V];
    rope_unpack<V>(a, f);
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) wd[u][i] = (double)f[i] + N.add;
  };
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t one[V];
#pragma unroll
    for (int q = 0; q < V; ++q) one[q] = 0x3F803F80u;
    if (N.w && !N.head) rope_words(*reinterpret_cast<const group*>(N.w + ca[u]), *reinterpret_cast<const group*>(N.w + cb[u]), one);
    weigh(u, one);
  }
  double c[U][V], s[U][V];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      c[u][i] = 1.0;
      s[u][i] = 0.0;
      if (turn[u]) {
        const RopeEntry e = R.tab[V * (j + u * LT) + i];
        rope_cos_sin((double)pos[(int64_t)e.axis * n_tokens + t] * e.freq, R.scale, c[u][i], s[u][i]);
      }
    }
  for (int hu = h0; hu < h1; hu += HU) {
    double y[HU][U][2 * V], rs[HU];
#pragma unroll
    for (int k = 0; k < HU; ++k) {
      rs[k] = 0.0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[2 * V];
        rope_unpack<V>(w[k][u], v);
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) {
          y[k][u][i] = (double)v[i];
          rs[k] = __builtin_fma(y[k][u][i], y[k][u][i], rs[k]);
        }
      }
    }
    uint32_t wt[HU][U][V];
#pragma unroll
    for (int k = 0; k < HU; ++k)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < V; ++q) wt[k][u][q] = ww[k][u][q];
    if (hu + HU < h1) load(hu + HU);
#pragma unroll
    for (int k = 0; k < HU; ++k) rs[k] = norm_rstd(row_sum<LT>(rs[k], lane), D, N.eps);
#pragma unroll
    for (int k = 0; k < HU; ++k) {
      if (hu + k >= h1) break;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (N.head) weigh(u, wt[k][u]);
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) y[k][u][i] = y[k][u][i] * rs[k] * wd[u][i];
        if (turn[u]) {
          constexpr int step = NEAR ? 2 : 1, other = NEAR ? 1 : V;
#pragma unroll
          for (int q = 0; q < V; ++q) {
            const double x0 = y[k][u][step * q], x1 = y[k][u][step * q + other];
            rope_rotate(x0, x1, c[u][q], s[u][q], y[k][u][step * q], y[k][u][step * q + other]);
          }
        }
        float v[2 * V];
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) v[i] = f64_round_bf16(y[k][u][i]);
        uint32_t o[V];
        rope_pack<V>(v, o);
        group a, b;
        rope_groups<V>(o, a, b);
        uint16_t* oh = orow + (int64_t)(hu + k) * D;
        *reinterpret_cast<group*>(oh + ca[u]) = a;
        *reinterpret_cast<group*>(oh + cb[u]) = b;
      }
      __builtin_amdgcn_sched_barrier(0);  // one head at a time: bounded register use
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

hipError_t launch_norm_rope_apply(const RopeView& R, const NormView& N, int d, int n_tokens, int n_heads, const uint16_t* x,
                                  int64_t xs, const int32_t* pos, uint16_t* out, int64_t os, hipStream_t s) {
  // (lane groups and launches as launch_rope_apply's)
  const int V = rope_width(R.rot), lt = d / (2 * V) > 64 ? 64 : d / (2 * V), per = 256 / lt;
  int64_t nb = ((int64_t)8192 * 64 / lt + n_tokens - 1) / n_tokens;
  if (nb > n_heads) nb = n_heads;
  const int hb = (int)((n_heads + nb - 1) / nb);
  auto go = [&](auto kern) {
    for (int64_t t0 = 0; t0 < n_tokens; t0 += 1 << 22) {
      const int n_here = (int)(n_tokens - t0 < 1 << 22 ? n_tokens - t0 : 1 << 22);
      const int64_t units = (int64_t)n_here * ((n_heads + hb - 1) / hb);
      hipLaunchKernelGGL(kern, dim3((unsigned)((units + per - 1) / per)), dim3(256), 0, s, R, N, t0, n_here, n_tokens,
                         n_heads, hb, x, xs, pos, out, os);
    }
  };
  auto pick = [&](auto dc, auto vc) {
    constexpr int DD = decltype(dc)::value, VV = decltype(vc)::value;
    R.interleaved ? go(norm_rope_apply_kernel<DD, VV, true>) : go(norm_rope_apply_kernel<DD, VV, false>);
  };
  auto of_v = [&](auto dc) {
    V == 4   ? pick(dc, std::integral_constant<int, 4>{})
    : V == 2 ? pick(dc, std::integral_constant<int, 2>{}) : pick(dc, std::integral_constant<int, 1>{});
  };
  d == 256 ? of_v(std::integral_constant<int, 256>{}) : of_v(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace mkv
