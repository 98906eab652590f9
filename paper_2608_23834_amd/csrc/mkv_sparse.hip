// Pages for sparse decode attention: the channelwise bounds of a page's keys, and the
// selection of the pages whose bound on q.k is largest.
//
// For any query, q.k_t <= s sum_c max(q_c hi_c, q_c lo_c) for every token t of a page, hi
// and lo the channelwise extremes of the page's key codes and s its key scale.  The
// extremes of E4M3 codes are E4M3 codes: the bound loses nothing to storage and costs 2 d
// + 4 bytes a page-head, a sixteenth of an FP8 page and an eighth of a TQ3 page.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "mkv_attn.h"
#include "mkv_internal.h"
#include "../../include/minima_kv.h"

namespace mkv {

// ---------------------------------------------------------------------------
// Bounds.  One wave per (page, layer, KV head): K is 16 d bytes [token][channel], lane l
// loads 16 bytes of every 64-lane row of it, reduces its tokens and the wave folds the
// lanes of a channel group.  Codes are compared as bytes: with the magnitude of the
// negative ones inverted they order as signed integers, and a byte in the upper half of a
// 16-bit lane is compared by v_pk_max_i16 whatever lies below it (8 operations on four
// codes, fp16 values take 14).  Memory bound: d bytes a token in, 2 d + 4 a page out (33 K
// tokens, 4 heads, 4 layers: 154 MB in 38 us, of every 8 KB page-head the K half).
// The pages of all requests form one run (a scan of their counts by every workgroup), dealt
// to the waves of the grid in turn, so requests of uneven lengths level out and a workgroup
// without pages leaves at once: with a part of the grid for each request, the update after a
// decode step of 64 requests took 8.1 us, now 4.8.
// ---------------------------------------------------------------------------
typedef short s2 __attribute__((ext_vector_type(2)));
// E4M3 codes <-> bytes that order like their values (it is its own inverse)
__device__ __forceinline__ uint32_t code_order(uint32_t x) { return x ^ ((x >> 7) & 0x01010101u) * 0x7Fu; }
constexpr int BOUNDS_REQ = 1024;  // requests of a launch (their counts are scanned in LDS)
constexpr int BOUNDS_WG = 2048;  // workgroups: eight waves a SIMD

template <int D>
__global__ __launch_bounds__(256) void page_bounds_kernel(PoolView P, int layer_sel, int n_req, int req0, int n_here,
                                                          const int32_t* bt, const uint8_t* tags, int max_pages,
                                                          const int32_t* from, const int32_t* seq, uint8_t* codes,
                                                          float* scales) {
  constexpr int LR = D / 16, NI = D / 64;  // lanes of a token, loads of a lane
  __shared__ int s_first[BOUNDS_REQ + 1], s_p0[BOUNDS_REQ], s_seq[BOUNDS_REQ], s_scan[5];  // the requests' runs
  const int layer = layer_sel < 0 ? (int)blockIdx.y : layer_sel, tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int H = P.n_kv_heads;
  int total = 0;
  for (int r0 = 0; r0 < n_here; r0 += 256) {
    const int r = r0 + tid;
    int n = 0;
    if (r < n_here) {
      const int S = seq[req0 + r], f = from[req0 + r];
      if (S < 0 || f < 0 || (int64_t)S > (int64_t)max_pages * PAGE) {
        if (blockIdx.x == 0 && blockIdx.y == 0) atomicOr(&P.ctrl[CTRL_ERR], (int)MKV_DEVERR_RANGE);
      } else {
        n = max(0, (S + PAGE - 1) / PAGE - f / PAGE);
      }
      s_p0[r] = f / PAGE;
      s_seq[r] = S;
    }
    int sum;
    const int at = block_excl_scan(n, s_scan, &sum);
    if (r < n_here) s_first[r] = total + at;
    total += sum;
  }
  if (tid == 0) s_first[n_here] = total;
  __syncthreads();
  // wave w: page-heads w, w + step, ..; run position g and head h stepped without divisions
  const int w0 = blockIdx.x * 4 + wid, step = gridDim.x * 4, dg = step / H, dh = step - dg * H;
  int g = w0 / H, h = w0 - g * H;
  if (g >= total) return;
  int r = 0;
  {
    int hi = n_here - 1;  // the last request whose run begins at or before g
    while (r < hi) {
      const int mid = (r + hi + 1) >> 1;
      if (s_first[mid] <= g) r = mid;
      else hi = mid - 1;
    }
  }
  for (; g < total; g += dg, h += dh) {
    if (h >= H) {
      h -= H;
      if (++g >= total) break;
    }
    while (s_first[r + 1] <= g) ++r;
    const int rq = __builtin_amdgcn_readfirstlane(r);
    const int p = __builtin_amdgcn_readfirstlane(s_p0[r] + g - s_first[r]);
    const int64_t ti = (int64_t)(req0 + rq) * max_pages + p;
    const int tag = tags[ti], id = bt[ti];
    const bool fp8 = tag == TAG_R || tag == TAG_A;
    if (!fp8 || id < 0 || id >= P.n_fp8) {
      if (lane == 0) atomicOr(&P.ctrl[CTRL_ERR], fp8 ? (int)MKV_DEVERR_RANGE : (int)MKV_DEVERR_BAD_TAG);
      continue;
    }
    const int64_t ph = ((int64_t)layer * P.n_fp8 + id) * H + h;
    const uint4* k = reinterpret_cast<const uint4*>(P.fp8 + ph * fp8_region_bytes(D));
    uint4 x[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) x[i] = k[64 * i + lane];
    const float s = P.fp8_scales[ph * 2];
    const int held = s_seq[rq] - p * PAGE;  // tokens of the page (16 or more: all)
    // per dword of codes: bytes 1, 3 (odd) and 0, 2 (even)
    s2 mo[4], me[4], no[4], ne[4];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const uint32_t q[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      const bool in = held >= PAGE || (64 / LR) * i + lane / LR < held;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t y = code_order(q[w]);
        const uint32_t ym = held >= PAGE ? y : in ? y : 0x80808080u, yn = held >= PAGE ? y : in ? y : 0x7F7F7F7Fu;
        const s2 a = __builtin_bit_cast(s2, ym), b = __builtin_bit_cast(s2, ym << 8);
        const s2 c = __builtin_bit_cast(s2, yn), d = __builtin_bit_cast(s2, yn << 8);
        mo[w] = i ? __builtin_elementwise_max(mo[w], a) : a;
        me[w] = i ? __builtin_elementwise_max(me[w], b) : b;
        no[w] = i ? __builtin_elementwise_min(no[w], c) : c;
        ne[w] = i ? __builtin_elementwise_min(ne[w], d) : d;
      }
    }
    if constexpr (LR == 8) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        auto other = [&](s2 v) { return __builtin_bit_cast(s2, lane_xor<8>(__builtin_bit_cast(float, v), lane)); };
        mo[w] = __builtin_elementwise_max(mo[w], other(mo[w]));
        me[w] = __builtin_elementwise_max(me[w], other(me[w]));
        no[w] = __builtin_elementwise_min(no[w], other(no[w]));
        ne[w] = __builtin_elementwise_min(ne[w], other(ne[w]));
      }
    }
    // lanes [0, LR) store the largest, [LR, 2 LR) the smallest: 16 codes each
    uint32_t o[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      // (each swap returns a value and its partner's, in one order for both lanes)
      auto over = [&](s2 v, auto op) {
        uint2 t = swap16(__builtin_bit_cast(float, v));
        v = op(__builtin_bit_cast(s2, t.x), __builtin_bit_cast(s2, t.y));
        t = swap32(__builtin_bit_cast(float, v));
        return op(__builtin_bit_cast(s2, t.x), __builtin_bit_cast(s2, t.y));
      };
      auto mx = [](s2 a, s2 b) { return __builtin_elementwise_max(a, b); };
      auto mn = [](s2 a, s2 b) { return __builtin_elementwise_min(a, b); };
      auto merge = [](s2 odd, s2 even) {  // the upper bytes back in their places
        return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, odd), __builtin_bit_cast(uint32_t, even), 0x07030501u);
      };
      const uint32_t big = merge(over(mo[w], mx), over(me[w], mx)), small = merge(over(no[w], mn), over(ne[w], mn));
      o[w] = code_order(lane >= LR ? small : big);
    }
    if (lane < 2 * LR) {
      const int64_t row = (((int64_t)layer * n_req + req0 + rq) * H + h) * max_pages + p;
      *reinterpret_cast<uint4*>(codes + row * 2 * D + 16 * lane) = make_uint4(o[0], o[1], o[2], o[3]);
      if (lane == 0) scales[row] = s;
    }
  }
}

hipError_t launch_page_bounds(const PoolView& P, int layer, int n_req, const int32_t* bt, const uint8_t* tags,
                              int max_pages, const int32_t* from, const int32_t* seq, uint8_t* codes, float* scales,
                              hipStream_t s) {
  const int n_lcall = layer < 0 ? P.n_layers : 1;
  for (int r0 = 0; r0 < n_req; r0 += BOUNDS_REQ) {
    const int n_here = n_req - r0 < BOUNDS_REQ ? n_req - r0 : BOUNDS_REQ;
    int64_t nb = (BOUNDS_WG + n_lcall - 1) / n_lcall;
    const int64_t most = ((int64_t)n_here * max_pages * P.n_kv_heads + 3) / 4;
    if (nb > most) nb = most;
    auto go = [&](auto kern) {
      hipLaunchKernelGGL(kern, dim3((unsigned)nb, (unsigned)n_lcall), dim3(256), 0, s, P, layer, n_req, r0, n_here, bt,
                         tags, max_pages, from, seq, codes, scales);
    };
    P.d == 256 ? go(page_bounds_kernel<256>) : go(page_bounds_kernel<128>);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Selection.  b(p) = s_p max_g sum_c max(q_c hi_c, q_c lo_c) = s_p max_g (q+ . hi + q- . lo)
// with q+ and q- the positive and the negative part of q: a product of 2 d against the
// group's heads, on the bf16 MFMA (bf16 holds both the query and E4M3 exactly).  Which page
// is in must not hang on the order of sums, so the choice is made in fp64, but only where
// the MFMA's score leaves it open: step 1 writes fp32 scores, step 2 brackets the smallest
// score that is in and recomputes in fp64 the few pages within the scores' error of it.
// ---------------------------------------------------------------------------
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));

// Error of an fp32 score over s_p.  The matrix unit adds eight products at a time to a sum,
// each cut below 2^-24 of the largest of them and the sum, then rounds: at most 8.5 * 2^-24
// of the sum so far, which grows to sum |q b| <= 448 sum |q| over two sums of d / 8 such
// steps (d = 256: 32): 32 * 8.5 / 2 * 2^-24 = 2^-16.9 of it; 2^-16 here.  (Measured: 2^-25.)
constexpr float SCORE_ERR = 448.0f * 0x1p-16f;
// Where products are subnormal or a subnormal query entry counts as 0: at most 448 * 2^-126
// of each of 256 channels, 2^-109, over s_p; and 2^-126 for the product with s_p itself.
constexpr float SCORE_SUB = 0x1p-109f;
// Both hold as long as no sum leaves fp32's range: 448 sum |q| below 2^127.  Past that a head's
// score may be an infinity or a NaN, which the maximum over the heads hides, where its true
// score is neither.
constexpr float SCORE_TOP = 0x1p118f;

// Step 1: one wave per 16 pages and step of the grid.  A: lane (page l % 16, group l / 16)
// loads 16 bytes of every 64 of its page's row; B: the same channels of head l % 16, in
// registers for the whole wave.  Memory bound (2 d + 4 bytes a page-head); the next tile is
// loaded while this one is multiplied.
template <int D>
__global__ __launch_bounds__(64) void select_score_kernel(int n_req, int H, int G, const uint16_t* q,
                                                          const int32_t* seq, int max_pages, int n_select,
                                                          const uint8_t* codes, const float* scales, float* score) {
  constexpr int NL = 2 * D / 64;  // 16-byte loads of a lane per tile
  const int h = blockIdx.y, r = blockIdx.z, lane = threadIdx.x, ln = lane & 15, lg = lane >> 4;
  const int S = seq[r];
  if (S < 1 || (int64_t)S > (int64_t)max_pages * PAGE) return;
  const int n_pg = (S + PAGE - 1) / PAGE;
  if (n_pg <= n_select) return;  // every page is taken
  const int n_tile = (n_pg + 15) / 16;
  int t = blockIdx.x;
  if (t >= n_tile) return;
  const int64_t row0 = ((int64_t)r * H + h) * max_pages;
  const uint8_t* base = codes + row0 * 2 * D;
  uint4 x[NL];
  auto load = [&](int tile) {
    const int p = min(tile * 16 + ln, n_pg - 1);
    const uint4* src = reinterpret_cast<const uint4*>(base + (int64_t)p * 2 * D) + lg;
#pragma unroll
    for (int i = 0; i < NL; ++i) x[i] = src[4 * i];
  };
  load(t);
  uint4 qb[2 * NL];  // bf16 pairs of q+ (first half) and q-
  {
    const uint16_t* qh = q + (((int64_t)r * H + h) * G + min(ln, G - 1)) * D;
#pragma unroll
    for (int i = 0; i < NL / 2; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint4 w = reinterpret_cast<const uint4*>(qh + 64 * i + 16 * lg)[u];
        const uint32_t in[4] = {w.x, w.y, w.z, w.w};
        uint32_t pos[4], neg[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t m = ((in[k] >> 15) & 0x00010001u) * 0xFFFFu;  // the negative ones
          neg[k] = ln < G ? in[k] & m : 0u;
          pos[k] = ln < G ? in[k] & ~m : 0u;
        }
        qb[2 * i + u] = make_uint4(pos[0], pos[1], pos[2], pos[3]);
        qb[NL + 2 * i + u] = make_uint4(neg[0], neg[1], neg[2], neg[3]);
      }
  }
  auto widen = [](uint32_t lo, uint32_t hi) {
    const bf2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    const bf2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    const bf2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  };
  for (; t < n_tile; t += gridDim.x) {
    uint4 y[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) y[i] = x[i];
    const int p0 = t * 16, p = p0 + 4 * lg + (ln & 3);
    const float sp = p < n_pg ? scales[row0 + p] : 0.0f;
    if (t + gridDim.x < (unsigned)n_tile) load(t + gridDim.x);
    float4v acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(y[i].x, y[i].y), __builtin_bit_cast(bf8, qb[2 * i]), acc[0], 0, 0, 0);
      acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(y[i].z, y[i].w), __builtin_bit_cast(bf8, qb[2 * i + 1]), acc[1], 0, 0, 0);
    }
    const float4v sum = acc[0] + acc[1];
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = ln < G ? sum[i] : -INFINITY;
      v[i] = fmaxf(v[i], lane_xor<1>(v[i], lane));
      v[i] = fmaxf(v[i], lane_xor<2>(v[i], lane));
      v[i] = fmaxf(v[i], lane_xor<4>(v[i], lane));
      v[i] = fmaxf(v[i], lane_xor<8>(v[i], lane));
    }
    const float best = ln & 2 ? (ln & 1 ? v[3] : v[2]) : (ln & 1 ? v[1] : v[0]);
    if (ln < 4 && p < n_pg) score[row0 + p] = best * sp;
  }
}

// The exact score of a page as a key that orders like it (larger score, larger key; NaN 0),
// by one wave: lane l holds channels D/64 l ..
__device__ __forceinline__ uint64_t score_key(double x) {
  if (x != x) return 0;
  const int64_t b = __builtin_bit_cast(int64_t, x + 0.0);  // -0 orders as 0
  return b < 0 ? ~(uint64_t)b : (uint64_t)b | 0x8000000000000000ull;
}
template <int M>
__device__ __forceinline__ double lane_xor64(double x, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __float_as_uint(lane_xor<M>(__uint_as_float((uint32_t)u), lane));
  const uint32_t hi = __float_as_uint(lane_xor<M>(__uint_as_float((uint32_t)(u >> 32)), lane));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// qs: the group's query rows in LDS
template <int D>
__device__ __forceinline__ uint64_t exact_key(const uint16_t* qs, int G, const uint8_t* row, float scale, int lane) {
  constexpr int NC = D / 64;
  typedef typename std::conditional<NC == 4, uint32_t, uint16_t>::type codes_t;
  const uint32_t ch = *reinterpret_cast<const codes_t*>(row + NC * lane);
  const uint32_t cl = *reinterpret_cast<const codes_t*>(row + D + NC * lane);
  double hi[NC], lo[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    hi[i] = (double)e4m3_to_f32(ch >> (8 * i) & 0xFFu);
    lo[i] = (double)e4m3_to_f32(cl >> (8 * i) & 0xFFu);
  }
  double best = -INFINITY;
  bool nan = false;  // a NaN among the extremes is one whatever the query's signs
#pragma unroll
  for (int i = 0; i < NC; ++i) nan |= hi[i] != hi[i] || lo[i] != lo[i];
  nan = __any(nan);
#pragma unroll 2
  for (int g = 0; g < G; ++g) {
    double a = 0.0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const double x = (double)bf16_to_f32(qs[g * D + NC * lane + i]);
      a = __builtin_fma(x, x < 0.0 ? lo[i] : hi[i], a);
    }
    a += lane_xor64<1>(a, lane);
    a += lane_xor64<2>(a, lane);
    a += lane_xor64<4>(a, lane);
    a += lane_xor64<8>(a, lane);
    a += lane_xor64<16>(a, lane);
    a += lane_xor64<32>(a, lane);
    nan |= a != a;
    best = a > best ? a : best;
  }
  return nan ? 0 : score_key(best * (double)scale);
}

// Inclusive prefix sum over a wave on the VALU: within rows of 16 by DPP shifts, then the
// rows' last sums broadcast to the next row and the next two.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // row_bcast:31 into rows 2 and 3
  return x;
}
// Exclusive prefix sum over a workgroup of 16 waves; s_w: 16 words, free again after the
// next barrier.
__device__ __forceinline__ int block_scan16(int v, int* s_w, int lane, int wid) {
  const int incl = wave_scan(v);
  if (lane == 63) s_w[wid] = incl;
  __syncthreads();
  const int w = wave_scan(lane < 16 ? s_w[lane] : 0);
  const int before = wid ? __builtin_amdgcn_readlane(w, wid - 1) : 0;
  return before + incl - v;
}

// Step 2: the n_select pages of a (request, KV head), one workgroup each: the first and
// last ones, and of the others (the competing ones) the `need` with the largest scores, ties
// to the lower page.
//  1. the range of the competing fp32 scores and their error E;
//  2. a histogram over the range: the bin that holds the need-th largest score.  That score
//     lies between the bin's edges lo and hi, and its exact value within E of it: a page
//     above hi + 2 E is in, one below lo - 2 E is out;
//  3. the pages between (or with a NaN) get their fp64 score; up to SEL_NB of them are
//     ranked against each other in LDS, more (equal pages, a query of NaN) by a radix
//     selection over the keys, 8 bits a round from the top;
//  4. the chosen pages in ascending order, by ballots and one scan.
// Latency bound: the scores of up to SEL_LDS pages and the queries are read into LDS in one
// round trip, every later pass reads them there.
constexpr int SEL_NT = 1024, SEL_NW = SEL_NT / 64, SEL_BINS = 2048, SEL_NB = 256;
constexpr int SEL_MAX_PAGES = 1024 * 256, SEL_LDS = 8192;

template <int D>
__global__ __launch_bounds__(SEL_NT) void select_pick_kernel(int H, int G, const uint16_t* q, const int32_t* seq,
                                                             int max_pages, int n_select, int n_first, int n_last,
                                                             const uint8_t* codes, const float* scales,
                                                             const float* score, uint64_t* keys, int32_t* sel,
                                                             int32_t* counts, int32_t* ctrl) {
  __shared__ int s_cnt[SEL_MAX_PAGES / 64];          // histogram, then chosen pages per 64
  // border pages that are in, a bit each; with at most SEL_LDS pages the bits are in s_few
  // and the scores here
  __shared__ uint32_t s_mem[SEL_MAX_PAGES / 32];
  __shared__ uint32_t s_few[SEL_LDS / 32];
  __shared__ __align__(16) uint16_t s_q[16 * D];
  __shared__ uint64_t s_key[SEL_NB];
  static_assert(SEL_LDS <= SEL_MAX_PAGES / 32, "the scores fit");
  __shared__ int s_idx[SEL_NB], s_scan[SEL_NW + 1], s_sum[2][SEL_NW], s_digit, s_above, s_here, s_nb, s_in;
  __shared__ float s_min[SEL_NW], s_max[SEL_NW], s_smax[SEL_NW], s_l1[16];
  __shared__ int s_nan[SEL_NW];
  const int h = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = (int64_t)r * H + h;
  int32_t* out = sel + row * n_select;
  const int S = seq[r];
  const bool bad = S < 1 || (int64_t)S > (int64_t)max_pages * PAGE;
  const int n_pg = bad ? 0 : (S + PAGE - 1) / PAGE;
  if (bad && h == 0 && tid == 0) atomicOr(&ctrl[CTRL_ERR], (int)MKV_DEVERR_RANGE);
  if (n_pg <= n_select) {
    for (int i = tid; i < n_select; i += SEL_NT) out[i] = i < n_pg ? i : -1;
    if (tid == 0) counts[row] = n_pg;
    return;
  }
  const float* sg = score + row * max_pages;
  const bool few = n_pg <= SEL_LDS;
  float* s_sc = reinterpret_cast<float*>(s_mem);
  uint32_t* s_bit = few ? s_few : s_mem;
  auto sc = [&](int p) { return few ? s_sc[p] : sg[p]; };
  const uint8_t* bc = codes + row * max_pages * 2 * D;
  const float* bs = scales + row * max_pages;
  const uint16_t* qh = q + row * G * D;
  uint64_t* key = keys + row * max_pages;
  const int m0 = n_first, m1 = n_pg - n_last;  // the competing pages
  const int need = n_select - n_first - n_last;
  auto larger = [](float a, float b) { return b > a || b != b ? b : a; };  // NaN if either is
  for (int i = tid; i < (n_pg + 31) / 32; i += SEL_NT) s_bit[i] = 0;
  float hi = INFINITY;
  int lowest = 0;  // competing pages taken from the lowest on, whatever their score
  if (need > 0) {
    // ---- 1. range and error
    for (int i = tid; i < SEL_BINS; i += SEL_NT) s_cnt[i] = 0;
    float mn = INFINITY, mx = -INFINITY, sm = 0.0f, l1 = 0.0f;
    bool nan = false;
    for (int p = m0 + tid; p < m1; p += SEL_NT) {
      const float a = sg[p];
      if (few) s_sc[p] = a;
      mn = fminf(mn, a);
      mx = fmaxf(mx, a);
      nan |= a != a;
      sm = larger(sm, fabsf(bs[p]));
    }
    if (wid < G) {
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint16_t x = qh[wid * D + 64 * i + lane];
        s_q[wid * D + 64 * i + lane] = x;
        l1 += fabsf(bf16_to_f32(x));
      }
    }
    auto fold = [&](auto mc) {
      constexpr int m = decltype(mc)::value;
      mn = fminf(mn, lane_xor<m>(mn, lane));
      mx = fmaxf(mx, lane_xor<m>(mx, lane));
      sm = larger(sm, lane_xor<m>(sm, lane));
      l1 += lane_xor<m>(l1, lane);
    };
    fold(std::integral_constant<int, 1>{});
    fold(std::integral_constant<int, 2>{});
    fold(std::integral_constant<int, 4>{});
    fold(std::integral_constant<int, 8>{});
    fold(std::integral_constant<int, 16>{});
    fold(std::integral_constant<int, 32>{});
    const int any_nan = __any(nan);
    if (lane == 0) {
      s_nan[wid] = any_nan;
      s_min[wid] = mn;
      s_max[wid] = mx;
      s_smax[wid] = sm;
      s_l1[wid] = l1;
    }
    if (tid == 0) s_nb = s_in = 0;
    __syncthreads();
    l1 = 0.0f;
#pragma unroll
    for (int w = 0; w < SEL_NW; ++w) {
      mn = fminf(mn, s_min[w]);
      mx = fmaxf(mx, s_max[w]);
      sm = larger(sm, s_smax[w]);
      l1 = larger(l1, s_l1[w]);
      nan |= s_nan[w];
    }
    const float E2 = 2.0f * (SCORE_ERR * l1 + SCORE_SUB) * sm + 0x1p-125f;
    // ---- 2. the bin of the need-th largest.  A range without a finite width, or of one at
    // which bin() would lose its bits to the subnormals, an error without one, or a query whose
    // products may leave fp32's range leaves every page open
    const float width = mx - mn;
    const bool bins = width > 0x1p-100f && width < INFINITY && E2 < INFINITY && l1 < SCORE_TOP;
    const float inv = bins ? (float)(SEL_BINS - 1) / width : 0.0f;
    auto bin = [&](float a) { return bins ? min(max((int)((a - mn) * inv), 0), SEL_BINS - 1) : 0; };
    float lo = -INFINITY;
    // a query or scales of zeros: every score is 0
    if ((l1 == 0.0f || sm == 0.0f) && l1 < SCORE_TOP && mn == mx && !nan) {
      lowest = need;
      lo = INFINITY;
    }
    if (bins) {
      for (int p = m0 + tid; p < m1; p += SEL_NT) atomicAdd(&s_cnt[bin(sc(p))], 1);
      __syncthreads();
      // suffix sums: thread t holds bins 2 t, 2 t + 1 counted from the top
      const int c0 = s_cnt[SEL_BINS - 1 - 2 * tid], c1 = s_cnt[SEL_BINS - 2 - 2 * tid];
      const int above = block_scan16(c0 + c1, s_sum[0], lane, wid);
      if (above < need && above + c0 >= need) s_digit = SEL_BINS - 1 - 2 * tid;
      if (above + c0 < need && above + c0 + c1 >= need) s_digit = SEL_BINS - 2 - 2 * tid;
      __syncthreads();
      // the bin's edges, a hundredth of a bin wider on either side (bin() is off by 2^-12 of
      // one at most); the lowest bin also holds what is no number, and has no lower edge
      const float one = width / (float)(SEL_BINS - 1);
      hi = mn + ((float)s_digit + 1.01f) * one + E2;
      lo = s_digit ? mn + ((float)s_digit - 0.01f) * one - E2 : -INFINITY;
    }
    // ---- 3. pages that the fp32 scores leave open
    int n_in = 0;
    for (int p = m0 + tid; p < m1; p += SEL_NT) {
      const float a = sc(p);
      n_in += a > hi;
      if (!(a > hi) && !(a < lo)) {
        const int at = atomicAdd(&s_nb, 1);
        if (at < SEL_NB) s_idx[at] = p;
      }
    }
    n_in = wave_scan(n_in);
    if (lane == 63 && n_in) atomicAdd(&s_in, n_in);
    __syncthreads();
    int left = need - lowest - s_in;  // of the open pages
    const int nb = s_nb;
    if (nb <= SEL_NB) {
      if (nb > left) {
        for (int j = wid; j < nb; j += SEL_NW) {
          const int p = s_idx[j];
          const uint64_t k = exact_key<D>(s_q, G, bc + (int64_t)p * 2 * D, bs[p], lane);
          if (lane == 0) s_key[j] = k;
        }
        __syncthreads();
      }
      for (int j = wid; j < nb; j += SEL_NW) {  // a wave counts the pages before page j
        const int p = s_idx[j];
        int rank = 0;
        if (nb > left) {
          const uint64_t k = s_key[j];
          for (int i0 = 0; i0 < nb; i0 += 64) {
            const int i = min(i0 + lane, nb - 1);
            const uint64_t o = s_key[i];
            rank += __popcll(__ballot(i0 + lane < nb && (o > k || (o == k && s_idx[i] < p))));
          }
        }
        if (lane == 0 && rank < left) atomicOr(&s_bit[p >> 5], 1u << (p & 31));
      }
      __syncthreads();
    } else {
      auto open = [&](int p) {
        const float a = sc(p);
        return !(a > hi) && !(a < lo);
      };
      for (int p = m0 + wid; p < m1; p += SEL_NW) {
        if (!open(p)) continue;  // wave-uniform
        const uint64_t k = exact_key<D>(s_q, G, bc + (int64_t)p * 2 * D, bs[p], lane);
        if (lane == 0) key[p] = k;
      }
      __syncthreads();
      uint64_t prefix = 0;  // the digits found, the rest 0
      int shift = 64;       // bits below which nothing is found yet
      bool all = false;     // every open page at or above the prefix is in
      while (shift > 0 && !all) {
        for (int i = tid; i < 256; i += SEL_NT) s_cnt[i] = 0;
        __syncthreads();
        for (int p = m0 + tid; p < m1; p += SEL_NT) {
          if (!open(p)) continue;
          const uint64_t k = key[p];
          if (shift == 64 || (k >> shift) == (prefix >> shift)) atomicAdd(&s_cnt[(k >> (shift - 8)) & 255], 1);
        }
        __syncthreads();
        const int c = tid < 256 ? s_cnt[255 - tid] : 0;
        const int above = block_scan16(c, s_sum[0], lane, wid);
        if (above < left && above + c >= left) {
          s_digit = 255 - tid;
          s_above = above;
          s_here = c;
        }
        __syncthreads();
        shift -= 8;
        prefix |= (uint64_t)s_digit << shift;
        left -= s_above;
        all = left == s_here;
        __syncthreads();
      }
      int tied = 0;
      for (int b0 = m0; b0 < m1; b0 += SEL_NT) {
        const int p = b0 + tid;
        bool in = false, tie = false;
        if (p < m1 && open(p)) {
          const uint64_t k = key[p] >> shift, t = prefix >> shift;
          in = k > t;
          tie = k == t;
        }
        int n_tie;
        const int before = block_excl_scan(tie ? 1 : 0, s_scan, &n_tie);
        if (in || (tie && tied + before < left)) atomicOr(&s_bit[p >> 5], 1u << (p & 31));
        tied += n_tie;
      }
      __syncthreads();
    }
  } else {
    __syncthreads();
  }
  // ---- 4. list
  const int n64 = (n_pg + 63) / 64;
  auto chosen = [&](int p) {
    return p < n_pg && (p < m0 + lowest || p >= m1 || sc(p) > hi || ((s_bit[p >> 5] >> (p & 31)) & 1u));
  };
  for (int c = wid; c < n64; c += SEL_NW) {
    const uint64_t m = __ballot(chosen(64 * c + lane));
    if (lane == 0) s_cnt[c] = __popcll(m);
  }
  __syncthreads();
  {
    constexpr int PER = SEL_MAX_PAGES / 64 / SEL_NT;
    int v[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      v[i] = PER * tid + i < n64 ? s_cnt[PER * tid + i] : 0;
      sum += v[i];
    }
    int at = block_scan16(sum, s_sum[1], lane, wid);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (PER * tid + i < n64) s_cnt[PER * tid + i] = at;
      at += v[i];
    }
  }
  __syncthreads();
  const uint64_t below = (1ull << lane) - 1ull;
  for (int c = wid; c < n64; c += SEL_NW) {
    const bool in = chosen(64 * c + lane);
    const uint64_t m = __ballot(in);
    const int at = s_cnt[c] + __popcll(m & below);
    if (in && at < n_select) out[at] = 64 * c + lane;
  }
  if (tid == 0) counts[row] = n_select;
}

// workspace: a key, then a score, per (request, KV head, page)
size_t select_ws_bytes(int n_req, int max_pages, int H) {
  return (size_t)n_req * H * max_pages * (sizeof(uint64_t) + sizeof(float));
}

hipError_t launch_select(const PoolView& P, int layer, int n_req, const uint16_t* q, const int32_t* seq,
                         int max_pages, const uint8_t* codes, const float* scales, int n_select, int n_first,
                         int n_last, int32_t* sel, int32_t* counts, void* ws, hipStream_t s) {
  const int H = P.n_kv_heads, G = P.group;
  const int64_t rows = (int64_t)n_req * H * max_pages;
  codes += layer * rows * 2 * P.d;
  scales += layer * rows;
  uint64_t* keys = reinterpret_cast<uint64_t*>(ws);
  float* score = reinterpret_cast<float*>(keys + rows);
  if (max_pages > n_select) {
    // waves: three a SIMD, not more than there are tiles
    const int64_t pairs = (int64_t)n_req * H, tiles = (max_pages + 15) / 16;
    int64_t nb = (3 * 1024 + pairs - 1) / pairs;
    if (nb > tiles) nb = tiles;
    const dim3 grid((unsigned)nb, (unsigned)H, (unsigned)n_req);
    auto go = [&](auto kern) {
      hipLaunchKernelGGL(kern, grid, dim3(64), 0, s, n_req, H, G, q, seq, max_pages, n_select, codes, scales, score);
    };
    P.d == 256 ? go(select_score_kernel<256>) : go(select_score_kernel<128>);
  }
  auto pick = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3((unsigned)H, (unsigned)n_req), dim3(SEL_NT), 0, s, H, G, q, seq, max_pages, n_select,
                       n_first, n_last, codes, scales, score, keys, sel, counts, P.ctrl);
  };
  P.d == 256 ? pick(select_pick_kernel<256>) : pick(select_pick_kernel<128>);
  return hipGetLastError();
}

}  // namespace mkv
