// The cache read back: bf16 K and V rows of token ranges, out of FP8 and TQ3 pages.
//
//   FP8:  k = s_K code,  v = s_V code
//   TQ3:  k_c = gamma sigma_c (H mu)_c / sqrt(d),  v_c = zero_c + scale_c code
//
// evaluated in fp32 and rounded to bf16 once.  Bound by memory: a value costs 1 or 0.5 bytes
// read and 2 written.
//
// One wave per (page, layer, KV head), keys or values, the heads of a page side by side, so that the
// waves of a workgroup write neighbouring pieces of the same rows.  The waves find their
// request by a 64-way search over the slots cu[r] / 16 + 2 r: a request of n tokens touches
// at most n / 16 + 2 pages, so these never overlap, and nothing has to be planned before.
//  * FP8 keys lie as the rows do: 16 codes a lane, two conversions and a packing.
//  * Values, FP8 or TQ3, lie in lane-chunks of d / 16 channels by four tokens: lane (r, g)
//    turns its chunk into d / 16 neighbouring channels of four rows, 16-byte stores.
//  * TQ3 keys need the inverse Hadamard transform: on the matrix unit, as the product of the
//    matrix itself (rows = channels, E4M3 signs) with the code levels (columns = tokens), all
//    sums exact (multiples of 1/8 below 2^10).  With k = channel index of the codes and c of the
//    row, H = (-1)^popcount(c & k): the rows of a tile are numbered so that only the low five
//    bits of c and k enter the operand, the bits above flip a lane's whole operand, and the top
//    bit of d = 256 is a sum and a difference of two products: 16 registers hold the matrix,
//    and a lane ends with eight neighbouring channels of a token.  As butterflies the transform
//    would take eight additions and four lane exchanges a value.
// 8 requests of 12,001 to 20,011 tokens, four layers of four heads, d = 256 (2.71 GB, 533 us of a
// copy's bandwidth): 664 us; over FP8 pages alone 5.1 TB/s read and written, over TQ3 pages alone 4.0
// to 4.3 TB/s, against 5.1 of a large copy.  With the pages in cache keys or values alone take 194 to
// 206 us each: the writes bound it.  A grid of resident workgroups that loop took 670 us; stores past
// the cache, the rows through LDS, keys and values in one wave, and the next head's loads before this
// one's stores gained nothing.
#include <hip/hip_runtime.h>

#include "mkv_attn.h"
#include "mkv_internal.h"
#include "../../include/minima_kv.h"

namespace mkv {

namespace {

typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(8)));  // rows are 8-byte aligned
typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(8)));
typedef float f2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  const bf2 r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

struct ReadArgs {
  PoolView P;
  int layer, n_lcall, n_req, max_pages, n_total;
  const int32_t* bt;
  const uint8_t* tags;
  const int32_t* from;
  const int32_t* cu;
  uint16_t* k;
  uint16_t* v;
  int64_t kts, vts;
  uint32_t n_tasks;
};

// the last request whose first slot is at most `slot` (cu as a caller promises it; any cu
// gives a request of the call)
__device__ __forceinline__ int find_request(const int32_t* cu, int n_req, uint32_t slot, int lane) {
  int lo = 0, n = n_req;
  while (n > 1) {
    const int step = (n + 63) / 64, i = lane * step;
    bool le = false;
    if (i < n) le = (int64_t)(cu[lo + i] >> 4) + 2 * (int64_t)(lo + i) <= (int64_t)slot;
    const int c = max(__popcll(__ballot(le)) - 1, 0);
    lo += c * step;
    n = min(step, n - c * step);
  }
  return lo;
}

}  // namespace

// the wave's keys, or values
template <int D, bool KV>
__device__ __forceinline__ void read_rows(const ReadArgs& a) {
  constexpr int CL = D / 16, NDW = 3 * D / 128, NK8 = D / 128;
  const PoolView& P = a.P;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ln = lane & 15, lg = lane >> 4;
  const int H = P.n_kv_heads;
  if (a.cu[0] != 0 || a.cu[a.n_req] != a.n_total) {  // the same verdict in every wave
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(&P.ctrl[CTRL_ERR], (int)MKV_DEVERR_RANGE);
    return;
  }
  // rows 4 a + i of a tile are channels 8 a + i (+ 4 and + 32 m by the tile): signs of their low
  // five bits against a lane's 32 codes, and of the bits above against the lane's group
  [[maybe_unused]] uint32_t had[8];
#pragma unroll
  for (int w = 0; w < 8 && !KV; ++w) {
    had[w] = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b)
      had[w] |= (0x38u | (uint32_t)(__popc((8 * (ln >> 2) + (ln & 3)) & (4 * w + b)) & 1) << 7) << (8 * b);
  }
  // signs of the channels 32 m + 8 lg + e, over pairs of bf16
  [[maybe_unused]] uint32_t sgn[D / 32][4];
#pragma unroll
  for (int m = 0; m < D / 32 && !KV; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int8_t* s = P.sigma + 32 * m + 8 * lg + 2 * e;
      sgn[m][e] = (s[0] < 0 ? 0x8000u : 0u) | (s[1] < 0 ? 0x80000000u : 0u);
    }
  for (uint32_t task = blockIdx.x * 4u + wid; task < a.n_tasks; task += gridDim.x * 4u) {
    const int h = (int)(task % (uint32_t)H);
    const uint32_t rest = task / (uint32_t)H;
    const int li = (int)(rest % (uint32_t)a.n_lcall);
    const uint32_t slot = rest / (uint32_t)a.n_lcall;
    const int r = __builtin_amdgcn_readfirstlane(find_request(a.cu, a.n_req, slot, lane));
    const int c0 = a.cu[r], c1 = a.cu[r + 1], f = a.from[r];
    const int64_t j = (int64_t)slot - (c0 >> 4) - 2 * (int64_t)r;  // page of the request's range
    if (c0 < 0 || c1 < c0 || c1 > a.n_total) {
      if (lane == 0) atomicOr(&P.ctrl[CTRL_ERR], (int)MKV_DEVERR_RANGE);
      continue;
    }
    const int n = c1 - c0;
    if (j < 0) continue;
    uint16_t* const base = KV ? a.v : a.k;
    const int64_t ts = KV ? a.vts : a.kts;
    uint16_t* const out = base + (int64_t)li * a.n_total * ts + (int64_t)h * D;
    int tag = TAG_NONE, id = -1, t0, t1;  // slots [t0, t1) of the page
    int64_t row0;                         // row of slot 0
    if (f < 0 || (int64_t)f + n > (int64_t)a.max_pages * PAGE) {  // no such tokens: zeros
      if (16 * j >= n) continue;
      if (lane == 0) atomicOr(&P.ctrl[CTRL_ERR], (int)MKV_DEVERR_RANGE);
      row0 = c0 + 16 * j;
      t0 = 0;
      t1 = (int)min((int64_t)16, n - 16 * j);
    } else {
      const int64_t p = (f >> 4) + j;
      if (p * PAGE >= (int64_t)f + n) continue;  // past the range
      t0 = (int)max((int64_t)0, f - p * PAGE);
      t1 = (int)min((int64_t)PAGE, (int64_t)f + n - p * PAGE);
      if (t0 >= t1) continue;  // (an empty range inside a page)
      row0 = (int64_t)c0 + p * PAGE - f;
      const int64_t ix = (int64_t)r * a.max_pages + p;
      tag = __builtin_amdgcn_readfirstlane((int)a.tags[ix]);
      id = __builtin_amdgcn_readfirstlane(a.bt[ix]);
      const bool is3 = tag == TAG_S, is8 = tag == TAG_R || tag == TAG_A;
      int bad = 0;
      if (!is3 && !is8) bad = MKV_DEVERR_BAD_TAG;
      else if (id < 0 || id >= (is3 ? P.n_tq3 : P.n_fp8)) bad = MKV_DEVERR_RANGE;
      if (bad) {
        if (lane == 0) atomicOr(&P.ctrl[CTRL_ERR], bad);
        tag = TAG_NONE;
      }
    }
    uint8_t* const rows = reinterpret_cast<uint8_t*>(out + row0 * ts);  // slot t at t * 2 ts
    const int64_t tb = 2 * ts;
    if (tag == TAG_NONE) {
      for (int i = lane; i < 16 * (D / 8); i += 64) {
        const int t = i / (D / 8);
        if (t >= t0 && t < t1) *reinterpret_cast<u4*>(rows + t * tb + 16 * (i % (D / 8))) = u4{0u, 0u, 0u, 0u};
      }
      continue;
    }
    const int layer = a.layer < 0 ? li : a.layer;
    if (tag != TAG_S) {
      const int64_t ph = ((int64_t)layer * P.n_fp8 + id) * H + h;
      const uint8_t* reg = P.fp8 + ph * fp8_region_bytes(D) + KV * PAGE * D;
      const float s = P.fp8_scales[ph * 2 + KV];
      if constexpr (!KV) {
        constexpr int LT = D / 16, NP = PAGE * LT / 64;  // lanes a token, passes
        uint4 x[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) x[i] = reinterpret_cast<const uint4*>(reg)[lane + 64 * i];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int t = (lane + 64 * i) / LT, c = 16 * (lane % LT);
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
          uint32_t o[8];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[q], true);
            o[2 * q] = bf16x2(lo[0] * s, lo[1] * s);
            o[2 * q + 1] = bf16x2(hi[0] * s, hi[1] * s);
          }
          if (t >= t0 && t < t1) {
            u4* dst = reinterpret_cast<u4*>(rows + t * tb + 2 * c);
            dst[0] = u4{o[0], o[1], o[2], o[3]};
            dst[1] = u4{o[4], o[5], o[6], o[7]};
          }
        }
      } else {
        const int cr = lane >> 2, g = lane & 3;  // lane-chunk of the region: channels CL cr .., tokens 4 g ..
        uint32_t w[CL];
#pragma unroll
        for (int i = 0; i < CL / 4; ++i) {
          const uint4 x = reinterpret_cast<const uint4*>(reg)[lane * (CL / 4) + i];
          w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
        }
        uint32_t o[4][CL / 2];
#pragma unroll
        for (int m = 0; m < CL; m += 2) {
          const f2 a0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[m], false), a1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[m], true);
          const f2 b0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[m + 1], false), b1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[m + 1], true);
          o[0][m / 2] = bf16x2(a0[0] * s, b0[0] * s);
          o[1][m / 2] = bf16x2(a0[1] * s, b0[1] * s);
          o[2][m / 2] = bf16x2(a1[0] * s, b1[0] * s);
          o[3][m / 2] = bf16x2(a1[1] * s, b1[1] * s);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int t = 4 * g + u;
          if (t >= t0 && t < t1) {
            u4* dst = reinterpret_cast<u4*>(rows + t * tb + 2 * CL * cr);
#pragma unroll
            for (int i = 0; i < CL / 8; ++i) dst[i] = u4{o[u][4 * i], o[u][4 * i + 1], o[u][4 * i + 2], o[u][4 * i + 3]};
          }
        }
      }
      continue;
    }
    const uint8_t* reg = P.tq3 + (((int64_t)layer * P.n_tq3 + id) * H + h) * tq3_region_bytes(D);
    uint32_t dw[NDW];
    read_chunk<NDW>(dw, reg + KV * 6 * D, lane);
    if constexpr (!KV) {
      const float f0 = (float)reinterpret_cast<const _Float16*>(reg + 12 * D)[ln] * (D == 256 ? 0.0625f : 0x1.6a09e667f3bcdp-4f);
      v8i B[NK8];
#pragma unroll
      for (int s = 0; s < NK8; ++s)
#pragma unroll
        for (int w = 0; w < 8; ++w)
          B[s][w] = (int)__builtin_amdgcn_perm(KLUT_HI, KLUT_LO, quad_sel<NDW>(dw, 8 * s + w));
      const bool put = ln >= t0 && ln < t1;
      // (read again for each page: with every flip of it kept over the pages the matrix takes 64 registers)
#pragma unroll
      for (int w = 0; w < 8; ++w) asm volatile("" : "+v"(had[w]));
      int lgv = lg;
      asm volatile("" : "+v"(lgv));
      uint8_t* row = rows + ln * tb + 16 * lg;
#pragma unroll
      for (int mm = 0; mm < 4; ++mm) {
        const uint32_t flip = (__popc(mm & lgv) & 1) ? 0x80808080u : 0u;
        float4v X[2][NK8];  // [b][m bit 0]
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          v8i A;
#pragma unroll
          for (int w = 0; w < 8; ++w) A[w] = (int)(had[w] ^ flip ^ (b && (w & 1) ? 0x80808080u : 0u));
          const float4v z = {0.f, 0.f, 0.f, 0.f};
          X[b][0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B[0], z, 0, 0, 0, 0, 0, 0);
          if constexpr (NK8 == 2) {
            const float4v Q = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B[NK8 - 1], z, 0, 0, 0, 0, 0, 0);
            X[b][NK8 - 1] = X[b][0] - Q;
            X[b][0] = X[b][0] + Q;
          }
        }
#pragma unroll
        for (int m0 = 0; m0 < NK8; ++m0) {
          const int m = NK8 * mm + m0;
          uint32_t o[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[e] = bf16x2(X[e >> 1][m0][2 * (e & 1)] * f0, X[e >> 1][m0][2 * (e & 1) + 1] * f0) ^ sgn[m][e];
          if (put) *reinterpret_cast<u4*>(row + 64 * m) = u4{o[0], o[1], o[2], o[3]};
        }
        __builtin_amdgcn_sched_barrier(0);  // a few tiles at a time: bounded register use
      }
    } else {
      // chunk (channels CL ln .., tokens 4 lg ..)
      uint4 sw[CL / 8], zw[CL / 8];
      const uint4* sp = reinterpret_cast<const uint4*>(reg + 12 * D + 32 + 2 * CL * ln);
      const uint4* zp = reinterpret_cast<const uint4*>(reg + 14 * D + 32 + 2 * CL * ln);
#pragma unroll
      for (int i = 0; i < CL / 8; ++i) {
        sw[i] = sp[i];
        zw[i] = zp[i];
      }
      const _Float16* sc = reinterpret_cast<const _Float16*>(sw);
      const _Float16* ze = reinterpret_cast<const _Float16*>(zw);
      uint32_t o[4][CL / 2];
#pragma unroll
      for (int m = 0; m < CL; m += 2) {
        const uint32_t ca = quad_sel<NDW>(dw, m), cb = quad_sel<NDW>(dw, m + 1);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          o[u][m / 2] = bf16x2(fmaf((float)sc[m], (float)((ca >> (8 * u)) & 0xFFu), (float)ze[m]),
                               fmaf((float)sc[m + 1], (float)((cb >> (8 * u)) & 0xFFu), (float)ze[m + 1]));
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int t = 4 * lg + u;
        if (t >= t0 && t < t1) {
          u4* dst = reinterpret_cast<u4*>(rows + t * tb + 2 * CL * ln);
#pragma unroll
          for (int i = 0; i < CL / 8; ++i) dst[i] = u4{o[u][4 * i], o[u][4 * i + 1], o[u][4 * i + 2], o[u][4 * i + 3]};
        }
      }
    }
  }
  // entries that fall (and so all that leave [0, n_total]): the waves above see those that a slot leads to
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int r = threadIdx.x; r < a.n_req; r += 256)
      if (a.cu[r + 1] < a.cu[r]) atomicOr(&P.ctrl[CTRL_ERR], (int)MKV_DEVERR_RANGE);
}

// blockIdx.y: keys or values, where both are asked for
template <int D>
__global__ __launch_bounds__(256, 4) void read_tokens_kernel(ReadArgs a) {
  if (a.k && blockIdx.y == 0) read_rows<D, false>(a);
  else read_rows<D, true>(a);
}

// waves of a call, for keys or values each
int64_t read_tasks(const PoolView& P, int layer, int n_req, int n_total) {
  const int64_t slots = (int64_t)n_total / PAGE + 2 * (int64_t)n_req;
  return slots * (layer < 0 ? P.n_layers : 1) * P.n_kv_heads;
}

hipError_t launch_read_tokens(const PoolView& P, int layer, int n_req, const int32_t* bt, const uint8_t* tags, int max_pages,
                              const int32_t* from, const int32_t* cu, int n_total, uint16_t* k, int64_t kts, uint16_t* v,
                              int64_t vts, hipStream_t s) {
  ReadArgs a;
  a.P = P;
  a.layer = layer;
  a.n_lcall = layer < 0 ? P.n_layers : 1;
  a.n_req = n_req;
  a.max_pages = max_pages;
  a.n_total = n_total;
  a.bt = bt;
  a.tags = tags;
  a.from = from;
  a.cu = cu;
  a.k = k;
  a.v = v;
  a.kts = kts;
  a.vts = vts;
  const int64_t tasks = read_tasks(P, layer, n_req, n_total);
  a.n_tasks = (uint32_t)tasks;
  const int64_t wg = (tasks + 3) / 4;
  const dim3 grid((unsigned)(wg < 65536 ? wg : 65536), k && v ? 2 : 1);
  if (P.d == 256)
    hipLaunchKernelGGL(read_tokens_kernel<256>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(read_tokens_kernel<128>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace mkv
