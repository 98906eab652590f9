// Pages for sparse decode attention: the channelwise bounds of a page's keys, and the
// selection of the pages whose bound on q.k is largest.
//
// For any query, q.k_t <= s sum_c max(q_c hi_c, q_c lo_c) for every token t of a page, hi
// and lo the channelwise extremes of the page's key codes and s its key scale.  The
// extremes of E4M3 codes are E4M3 codes: the bound loses nothing to storage and costs 2 d
// + 4 bytes a page-head, a sixteenth of an FP8 page and an eighth of a TQ3 page.
#include <hip/hip_runtime.h>

#include "mkv_attn.h"
#include "mkv_internal.h"
#include "../../include/minima_kv.h"

namespace mkv {

// ---------------------------------------------------------------------------
// Bounds.  One wave per (page, layer, KV head): K is 16 d bytes [token][channel], lane l
// loads 16 bytes of every 64-lane row of it, reduces its tokens as packed fp16 (E4M3 in
// fp16 is exact) and the wave folds the lanes of a channel group.  Memory bound: d bytes
// a token in, 2 d + 4 a page out.
// ---------------------------------------------------------------------------
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

template <int D>
__global__ __launch_bounds__(256) void page_bounds_kernel(PoolView P, int layer_sel, int n_lcall, int n_req,
                                                          const int32_t* bt, const uint8_t* tags, int max_pages,
                                                          const int32_t* from, const int32_t* seq, uint8_t* codes,
                                                          float* scales) {
  constexpr int LR = D / 16, NI = D / 64;  // lanes of a token, loads of a lane
  const int r = blockIdx.y, lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int H = P.n_kv_heads, S = seq[r], f = from[r];
  if (S < 0 || f < 0 || (int64_t)S > (int64_t)max_pages * PAGE) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(&P.ctrl[CTRL_ERR], (int)MKV_DEVERR_RANGE);
    return;
  }
  const int p0 = f / PAGE, n_pg = max(0, (S + PAGE - 1) / PAGE - p0), LH = n_lcall * H;
  const int64_t n_tasks = (int64_t)n_pg * LH;
  for (int64_t task = (int64_t)blockIdx.x * 4 + wid; task < n_tasks; task += (int64_t)gridDim.x * 4) {
    const int pl = (int)(task / LH), lh = (int)(task - (int64_t)pl * LH), p = p0 + pl;
    const int li = lh / H, h = lh - li * H, layer = layer_sel < 0 ? li : layer_sel;
    const int64_t ti = (int64_t)r * max_pages + p;
    const int tag = tags[ti], id = bt[ti];
    if ((tag != TAG_R && tag != TAG_A) || id < 0 || id >= P.n_fp8) {
      if (lane == 0)
        atomicOr(&P.ctrl[CTRL_ERR], tag != TAG_R && tag != TAG_A ? (int)MKV_DEVERR_BAD_TAG : (int)MKV_DEVERR_RANGE);
      continue;
    }
    const int64_t ph = ((int64_t)layer * P.n_fp8 + id) * H + h;
    const uint4* k = reinterpret_cast<const uint4*>(P.fp8 + ph * fp8_region_bytes(D));
    uint4 x[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) x[i] = k[64 * i + lane];
    const float s = P.fp8_scales[ph * 2];
    const int held = S - p * PAGE;  // tokens of the page (16 or more: all)
    const h2 big = {(_Float16)INFINITY, (_Float16)INFINITY};
    h2 hi[8], lo[8];
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      hi[w] = -big;
      lo[w] = big;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if ((64 / LR) * i + lane / LR < held) {
        const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const h2 a = cvt_lo(u[w]), b = cvt_hi(u[w]);
          hi[2 * w] = __builtin_elementwise_max(hi[2 * w], a);
          hi[2 * w + 1] = __builtin_elementwise_max(hi[2 * w + 1], b);
          lo[2 * w] = __builtin_elementwise_min(lo[2 * w], a);
          lo[2 * w + 1] = __builtin_elementwise_min(lo[2 * w + 1], b);
        }
      }
    }
#pragma unroll
    for (int o = 32; o >= LR; o >>= 1)
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        hi[w] = __builtin_elementwise_max(hi[w], __builtin_bit_cast(h2, __shfl_xor(__builtin_bit_cast(int, hi[w]), o, 64)));
        lo[w] = __builtin_elementwise_min(lo[w], __builtin_bit_cast(h2, __shfl_xor(__builtin_bit_cast(int, lo[w]), o, 64)));
      }
    // lanes [0, LR) store hi, [LR, 2 LR) lo: 16 codes each
    const bool low = lane >= LR;
    if (lane < 2 * LR) {
      uint32_t o[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const h2 a = low ? lo[2 * w] : hi[2 * w], b = low ? lo[2 * w + 1] : hi[2 * w + 1];
        const int c = __builtin_amdgcn_cvt_pk_fp8_f32((float)a[0], (float)a[1], 0, false);
        o[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32((float)b[0], (float)b[1], c, true);
      }
      const int64_t row = (((int64_t)layer * n_req + r) * H + h) * max_pages + p;
      *reinterpret_cast<uint4*>(codes + row * 2 * D + 16 * lane) = make_uint4(o[0], o[1], o[2], o[3]);
      if (lane == 0) scales[row] = s;
    }
  }
}

hipError_t launch_page_bounds(const PoolView& P, int layer, int n_req, const int32_t* bt, const uint8_t* tags,
                              int max_pages, const int32_t* from, const int32_t* seq, uint8_t* codes, float* scales,
                              hipStream_t s) {
  const int n_lcall = layer < 0 ? P.n_layers : 1;
  // workgroups of four waves: enough for every SIMD to hold eight waves, not more than the
  // table has page-heads
  int64_t nb = (2048 + n_req - 1) / n_req;
  const int64_t most = ((int64_t)max_pages * n_lcall * P.n_kv_heads + 3) / 4;
  if (nb > most) nb = most;
  const dim3 grid((unsigned)nb, (unsigned)n_req);
  if (P.d == 256)
    hipLaunchKernelGGL(page_bounds_kernel<256>, grid, dim3(256), 0, s, P, layer, n_lcall, n_req, bt, tags, max_pages,
                       from, seq, codes, scales);
  else
    hipLaunchKernelGGL(page_bounds_kernel<128>, grid, dim3(256), 0, s, P, layer, n_lcall, n_req, bt, tags, max_pages,
                       from, seq, codes, scales);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Selection, step 1: scores.  One wave per page-head, lane l holds channels D/64 l ..; per
// head of the group sum_c max(q_c hi_c, q_c lo_c) in fp64 (a choice between two pages has
// to come out the same whatever the order of the sums), the largest over the group times
// the page's scale, as a key that orders like the score: larger score, larger key; NaN 0.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint64_t score_key(double x) {
  if (x != x) return 0;
  const int64_t b = __builtin_bit_cast(int64_t, x + 0.0);  // -0 orders as 0
  return b < 0 ? ~(uint64_t)b : (uint64_t)b | 0x8000000000000000ull;
}

template <int D>
__global__ __launch_bounds__(256) void select_score_kernel(int n_req, int H, int G, const uint16_t* q,
                                                           const int32_t* seq, int max_pages, int n_select,
                                                           const uint8_t* codes, const float* scales, uint64_t* keys) {
  constexpr int NC = D / 64;
  const int h = blockIdx.y, r = blockIdx.z, lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int S = seq[r];
  if (S < 1 || (int64_t)S > (int64_t)max_pages * PAGE) return;
  const int n_pg = (S + PAGE - 1) / PAGE;
  if (n_pg <= n_select) return;  // every page is taken
  const int64_t row0 = ((int64_t)r * H + h) * max_pages;
  const uint16_t* qh = q + ((int64_t)r * H + h) * G * D;
  for (int p = blockIdx.x * 4 + wid; p < n_pg; p += gridDim.x * 4) {
    const uint8_t* c = codes + (row0 + p) * 2 * D + NC * lane;
    double hi[NC], lo[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      hi[i] = (double)e4m3_to_f32(c[i]);
      lo[i] = (double)e4m3_to_f32(c[D + i]);
    }
    double best = -INFINITY;
    bool nan = false;
    for (int g = 0; g < G; ++g) {
      double a = 0.0;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const double x = (double)bf16_to_f32(qh[g * D + NC * lane + i]);
        a = __builtin_fma(x, x < 0.0 ? lo[i] : hi[i], a);
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) a += __shfl_xor(a, o, 64);
      nan |= a != a;
      best = a > best ? a : best;
    }
    if (lane == 0) keys[row0 + p] = nan ? 0 : score_key(best * (double)scales[row0 + p]);
  }
}

// Step 2: the n_select pages of a (request, KV head), one workgroup each: the first and
// last ones, and of the others the largest keys, ties to the lower page.  The smallest key
// that is in (radix selection, 8 bits a round, from the top; it ends as soon as a digit's
// pages are all in) and how many pages of that key, then the pages in ascending order.
constexpr int SEL_NT = 1024;
__global__ __launch_bounds__(SEL_NT) void select_pick_kernel(int H, const int32_t* seq, int max_pages, int n_select,
                                                             int n_first, int n_last, const uint64_t* keys,
                                                             int32_t* sel, int32_t* counts, int32_t* ctrl) {
  __shared__ int s_hist[256], s_scan[SEL_NT / 64 + 1], s_digit, s_above, s_here;
  const int h = blockIdx.x, r = blockIdx.y, tid = threadIdx.x;
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
  const uint64_t* key = keys + row * max_pages;
  const int m0 = n_first, m1 = n_pg - n_last;  // the pages that compete
  int need = n_select - n_first - n_last;
  uint64_t prefix = 0;  // the digits found, the rest 0
  int shift = 64;       // bits below which nothing is found yet
  const bool none = need == 0;  // no page but the first and last ones
  bool all = none;              // every page at or above the prefix is in
  while (shift > 0 && !all) {
    for (int i = tid; i < 256; i += SEL_NT) s_hist[i] = 0;
    __syncthreads();
    for (int p = m0 + tid; p < m1; p += SEL_NT) {
      const uint64_t k = key[p];
      if (shift == 64 || (k >> shift) == (prefix >> shift)) atomicAdd(&s_hist[(k >> (shift - 8)) & 255], 1);
    }
    __syncthreads();
    if (tid < 64) {  // suffix sums of the digits, four a lane from the top
      int v[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += v[i] = s_hist[255 - (4 * tid + i)];
      int incl = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(incl, o, 64);
        if (tid >= o) incl += y;
      }
      int above = incl - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < need && above + v[i] >= need) {
          s_digit = 255 - (4 * tid + i);
          s_above = above;
          s_here = v[i];
        }
        above += v[i];
      }
    }
    __syncthreads();
    shift -= 8;
    prefix |= (uint64_t)s_digit << shift;
    need -= s_above;
    all = need == s_here;
    __syncthreads();
  }
  // above the prefix's digits: in; equal to them: the lowest `need` (all of them when `all`)
  int base = 0, tied = 0;
  for (int b0 = 0; b0 < n_pg; b0 += SEL_NT) {
    const int p = b0 + tid;
    bool in = p < n_pg && (p < m0 || p >= m1), tie = false;
    if (p >= m0 && p < m1 && !none) {
      const uint64_t k = key[p] >> shift, t = prefix >> shift;
      in = k > t;
      tie = k == t;
    }
    int n_tie, total;
    const int before = block_excl_scan(tie ? 1 : 0, s_scan, &n_tie);
    if (tie) in = tied + before < need;
    const int at = block_excl_scan(in ? 1 : 0, s_scan, &total);
    if (in) out[base + at] = p;
    tied += n_tie;
    base += total;
  }
  if (tid == 0) counts[row] = n_select;
}

size_t select_ws_bytes(int n_req, int max_pages, int H) { return (size_t)n_req * H * max_pages * sizeof(uint64_t); }

hipError_t launch_select(const PoolView& P, int layer, int n_req, const uint16_t* q, const int32_t* seq,
                         int max_pages, const uint8_t* codes, const float* scales, int n_select, int n_first,
                         int n_last, int32_t* sel, int32_t* counts, void* ws, hipStream_t s) {
  const int H = P.n_kv_heads, G = P.group;
  const int64_t off = (int64_t)layer * n_req * H * max_pages;
  codes += off * 2 * P.d;
  scales += off;
  uint64_t* keys = reinterpret_cast<uint64_t*>(ws);
  if (max_pages > n_select) {
    int64_t nb = (4096 + (int64_t)n_req * H - 1) / ((int64_t)n_req * H);
    if (nb > (max_pages + 3) / 4) nb = (max_pages + 3) / 4;
    const dim3 grid((unsigned)nb, (unsigned)H, (unsigned)n_req);
    if (P.d == 256)
      hipLaunchKernelGGL(select_score_kernel<256>, grid, dim3(256), 0, s, n_req, H, G, q, seq, max_pages, n_select,
                         codes, scales, keys);
    else
      hipLaunchKernelGGL(select_score_kernel<128>, grid, dim3(256), 0, s, n_req, H, G, q, seq, max_pages, n_select,
                         codes, scales, keys);
  }
  hipLaunchKernelGGL(select_pick_kernel, dim3((unsigned)H, (unsigned)n_req), dim3(SEL_NT), 0, s, H, seq, max_pages,
                     n_select, n_first, n_last, keys, sel, counts, P.ctrl);
  return hipGetLastError();
}

}  // namespace mkv
