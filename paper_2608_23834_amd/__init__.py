"""Python binding of libminimakv (MI355X / gfx950 Minima-KV hot path).

Argument marshalling only: every step of the path runs in the HIP kernels of
``libminimakv.so``.  torch supplies device memory and streams.  The functions
keep the C ABI's names (include/minima_kv.h).  There is no CPU fallback: if the
built library is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import math
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libminimakv.so")

MKV_ALL_LAYERS = -1
PAGE = 16
TAG_R, TAG_A, TAG_S, TAG_NONE = 0, 1, 2, 0xFF
STATUS = {0: "MKV_OK", 1: "MKV_EINVAL", 2: "MKV_EUNSUP", 3: "MKV_ENOMEM", 4: "MKV_ERANGE",
          5: "MKV_ESTATE", 6: "MKV_EHIP"}
DEVERR = {"FP8_EXHAUSTED": 0x1, "TQ3_EXHAUSTED": 0x2, "NOT_RECENT": 0x4, "RANGE": 0x8,
          "BAD_TAG": 0x10, "REFCOUNT": 0x20}
EXPORTS = ["kv_pool_bytes", "kv_pool_create", "kv_pool_destroy", "kv_append_fp8",
           "kv_migrate_to_tq3", "kv_promote_to_fp8", "kv_pages_acquire", "kv_pages_release",
           "kv_request_finish", "kv_pool_read_refcounts", "paged_attn_workspace_bytes", "paged_attn_workspace_init",
           "paged_attn_decode", "paged_attn_decode_append", "paged_attn_chunk",
           "kv_partition_pages", "kv_pool_free_counts",
           "kv_pool_read_free_lists", "kv_pool_counters", "kv_pool_check_errors",
           "paged_attn_set_timing", "paged_attn_set_deterministic", "paged_attn_last_times",
           "mkv_stream_read",
           "paged_attn_decode_noalloc", "mkv_fp64_probe", "mkv_control_bf16_write",
           "mkv_control_bf16_workspace_bytes", "mkv_control_bf16_decode",
           "paged_attn_decode_cohort_key", "paged_attn_decode_scores", "kv_page_scores_update",
           "kv_rope_bytes", "kv_rope_create", "kv_rope_destroy", "kv_rope_apply", "kv_append_fp8_rope",
           "paged_attn_decode_append_rope", "kv_page_bounds_bytes", "kv_page_bounds_update",
           "paged_attn_select_workspace_bytes", "paged_attn_select_pages", "paged_attn_decode_sparse",
           "kv_read_tokens", "kv_norm_rope_apply", "kv_append_fp8_norm_rope",
           "paged_attn_decode_shaped", "paged_attn_decode_append_shaped", "paged_attn_chunk_shaped",
           "mkv_status_string"]

_lib = None


class MkvError(RuntimeError):
    def __init__(self, fn, code):
        super().__init__(f"{fn} failed: {STATUS.get(code, code)}")
        self.code = code


class PoolDesc(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_fp8_pages", ctypes.c_int32),
                ("n_tq3_pages", ctypes.c_int32), ("recent_tokens", ctypes.c_int32),
                ("rot_signs", ctypes.c_void_p), ("fp8_order", ctypes.c_void_p),
                ("tq3_order", ctypes.c_void_p),
                ("fp8_data", ctypes.c_void_p), ("fp8_data_bytes", ctypes.c_size_t),
                ("fp8_scales", ctypes.c_void_p), ("fp8_scales_bytes", ctypes.c_size_t),
                ("tq3_data", ctypes.c_void_p), ("tq3_data_bytes", ctypes.c_size_t),
                ("ctrl", ctypes.c_void_p), ("ctrl_bytes", ctypes.c_size_t)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("scale", ctypes.c_double), ("inv_freq", ctypes.c_void_p),
                ("axis", ctypes.c_void_p), ("table", ctypes.c_void_p), ("table_bytes", ctypes.c_size_t)]


class HeadNormDesc(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("eps", ctypes.c_double), ("add", ctypes.c_double),
                ("weight", ctypes.c_void_p), ("head_stride", ctypes.c_int64), ("layer_stride", ctypes.c_int64)]


class ShapingDesc(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("cap", ctypes.c_float), ("window", ctypes.c_int32),
                ("slopes", ctypes.c_void_p), ("sinks", ctypes.c_void_p), ("first_keys", ctypes.c_void_p),
                ("prefix_lens", ctypes.c_void_p)]


class Counters(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in (
        "decode_routes", "chunk_routes", "fallbacks", "dense_shadow_bytes", "fp8_pages_live",
        "tq3_pages_live", "fp8_bytes_live", "tq3_bytes_live")]


def lib() -> ctypes.CDLL:
    """Load the built library (build it with ``python -m paper_2608_23834_amd.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libminimakv.so is not built ({LIB_PATH}); run "
                               "`python -m paper_2608_23834_amd.build` first")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        for name in EXPORTS:
            getattr(L, name).restype = ctypes.c_int
        L.mkv_status_string.restype = ctypes.c_char_p
        L.kv_pool_bytes.argtypes = [vp, vp, vp, vp, vp]
        L.kv_pool_create.argtypes = [vp, vp]
        L.kv_pool_destroy.argtypes = [vp]
        L.kv_append_fp8.argtypes = [vp, i32, i32, vp, vp, i32, vp, vp, i32, vp, vp, vp]
        L.kv_migrate_to_tq3.argtypes = [vp, i32, vp, vp, i32, vp, vp, vp]
        L.kv_promote_to_fp8.argtypes = [vp, i32, vp, vp, i32, vp, vp, vp]
        L.kv_pages_acquire.argtypes = [vp, i32, vp, vp, vp]
        L.kv_pages_release.argtypes = [vp, i32, vp, vp, vp]
        L.kv_request_finish.argtypes = [vp, i32, vp, i32, vp, vp, i32, vp]
        L.kv_pool_read_refcounts.argtypes = [vp, vp, vp]
        L.paged_attn_workspace_bytes.argtypes = [vp, i32, i32, i32, vp]
        L.paged_attn_workspace_init.argtypes = [vp, sz, vp]
        L.paged_attn_decode.argtypes = [vp, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.paged_attn_decode_noalloc.argtypes = [vp, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp]
        L.paged_attn_decode_append.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp,
                                               vp, sz, vp]
        L.paged_attn_chunk.argtypes = [vp, i32, i32, vp, vp, i32, vp, vp, i32, vp, vp, vp, sz, vp]
        L.kv_partition_pages.argtypes = [i32, vp, vp, i32, vp, vp, vp, vp, vp]
        L.kv_pool_free_counts.argtypes = [vp, vp, vp]
        L.kv_pool_read_free_lists.argtypes = [vp, vp, vp, vp, vp]
        L.kv_pool_counters.argtypes = [vp, vp]
        L.kv_pool_check_errors.argtypes = [vp, vp, i32]
        L.paged_attn_set_timing.argtypes = [vp, i32]
        L.paged_attn_set_deterministic.argtypes = [vp, i32]
        L.paged_attn_last_times.argtypes = [vp, vp, vp]
        L.mkv_stream_read.argtypes = [vp, sz, vp, vp]
        L.mkv_fp64_probe.argtypes = [vp, vp, ctypes.c_int64, vp, vp, vp, vp]
        L.paged_attn_decode_cohort_key.argtypes = [vp, i32, i32, i32, i32, vp]
        L.paged_attn_decode_scores.argtypes = [vp, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, sz,
                                               vp, vp]
        L.kv_page_scores_update.argtypes = [vp, i32, i32, vp, vp, vp, vp, ctypes.c_float, vp, vp,
                                            vp, vp]
        i64 = ctypes.c_int64
        L.kv_rope_bytes.argtypes = [i32, vp]
        L.kv_rope_create.argtypes = [vp, vp]
        L.kv_rope_destroy.argtypes = [vp]
        L.kv_rope_apply.argtypes = [vp, i32, i32, vp, i64, vp, vp, i64, vp]
        L.kv_append_fp8_rope.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp, vp, i32, vp, vp, i64, vp, i64, vp]
        L.paged_attn_decode_append_rope.argtypes = [vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp,
                                                    vp, sz, vp]
        L.kv_page_bounds_bytes.argtypes = [vp, i32, i32, vp, vp]
        L.kv_page_bounds_update.argtypes = [vp, i32, i32, vp, vp, i32, vp, vp, vp, sz, vp, sz, vp]
        L.paged_attn_select_workspace_bytes.argtypes = [vp, i32, i32, vp]
        L.paged_attn_select_pages.argtypes = [vp, i32, i32, vp, vp, i32, vp, sz, vp, sz, i32, i32, i32, vp, vp,
                                              vp, sz, vp]
        L.paged_attn_decode_sparse.argtypes = [vp, i32, i32, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.kv_norm_rope_apply.argtypes = [vp, vp, i32, i32, vp, i64, vp, vp, i64, vp]
        L.kv_append_fp8_norm_rope.argtypes = [vp, vp, vp, i32, i32, vp, vp, i32, vp, vp, i32, vp, vp, i64, vp, i64, vp]
        L.paged_attn_decode_shaped.argtypes = [vp, vp, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.paged_attn_decode_append_shaped.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp,
                                                      vp, vp, sz, vp]
        L.paged_attn_chunk_shaped.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp, vp, i32, vp, vp, vp, sz, vp]
        L.kv_read_tokens.argtypes = [vp, i32, i32, vp, vp, i32, vp, vp, i32, vp, i64, vp, i64, vp]
        L.mkv_control_bf16_write.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp, i32, vp, vp, i32,
                                             vp, vp, vp]
        L.mkv_control_bf16_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, vp]
        L.mkv_control_bf16_decode.argtypes = [vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, i32,
                                              vp, vp, vp, vp, sz, vp]
        L.mkv_status_string.argtypes = [ctypes.c_int]
        _lib = L
    return _lib


def _check(fn, code):
    if code != 0:
        raise MkvError(fn, code)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _current():
    """(current device, its current stream's handle): without the Stream object around it 0.2 us
    of a call instead of 3."""
    global _current
    import torch
    device, raw = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream

    def _current():
        d = device()
        return d, raw(d)
    return _current()


def _stream(stream=None):
    return _current()[1] if stream is None else stream.cuda_stream


def _types():
    """Types that (rows of bf16 bits, int32, float32) may come as; the first call loads torch."""
    global _types
    import torch
    t = (torch.int16, torch.bfloat16, torch.uint16), (torch.int32,), (torch.float32,)

    def _types():
        return t
    return t


def _here(dev, *tensors):
    """Every tensor (None aside) lies on device dev, without gaps."""
    for t in tensors:
        if t is not None and (t.get_device() != dev or not t.is_contiguous()):
            raise ValueError("tensors are contiguous and on the current device")


_WRONG_TYPE = "rows are bf16 (or its bits in int16), lengths and pages int32, out and lse float32"


def _sizes(*pairs):
    """(tensor, shape): of the shape, for more requests, or as many elements or more in fewer axes."""
    for t, want in pairs:
        s = t.shape
        if s != want and (t.numel() < math.prod(want) or len(s) >= len(want) and s[-len(want) + 1:] != want[1:]):
            raise ValueError(f"{want} is wanted, not {tuple(s)}")


def _table(dev, pool, block_table, tags, i32):
    n_req, max_pages = block_table.shape
    if (block_table.dtype not in i32 or tags.element_size() != 1 or tags.numel() < n_req * max_pages
            or not block_table.is_contiguous() or not tags.is_contiguous() or block_table.get_device() != dev
            or tags.get_device() != dev or pool.device != dev):
        raise ValueError("block_table int32 and tags uint8 are [n_req][max_pages], contiguous and with the pool on the "
                         "current device")
    return n_req, max_pages


def pool_bytes(n_layers, n_q_heads, n_kv_heads, head_dim, n_fp8_pages, n_tq3_pages, recent_tokens):
    d = PoolDesc(n_layers, n_q_heads, n_kv_heads, head_dim, PAGE, n_fp8_pages, n_tq3_pages,
                 recent_tokens)
    out = (ctypes.c_size_t * 4)()
    _check("kv_pool_bytes", lib().kv_pool_bytes(ctypes.byref(d), ctypes.byref(out, 0),
                                                ctypes.byref(out, 8), ctypes.byref(out, 16),
                                                ctypes.byref(out, 24)))
    return tuple(out)


class Pool:
    """A pool over torch-allocated device buffers (the caller owns memory)."""

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, n_fp8_pages, n_tq3_pages,
                 recent_tokens, rot_signs, fp8_order=None, tq3_order=None, device="cuda"):
        import torch
        self.n_layers, self.n_q_heads, self.n_kv_heads, self.d = n_layers, n_q_heads, n_kv_heads, head_dim
        self.n_fp8, self.n_tq3, self.recent = n_fp8_pages, n_tq3_pages, recent_tokens
        b8, bs, b3, bc = pool_bytes(n_layers, n_q_heads, n_kv_heads, head_dim, n_fp8_pages,
                                    n_tq3_pages, recent_tokens)
        self.fp8 = torch.zeros(b8, dtype=torch.uint8, device=device)
        self.fp8_scales = torch.zeros(bs // 4, dtype=torch.float32, device=device)
        self.tq3 = torch.zeros(max(b3, 16), dtype=torch.uint8, device=device)
        self.ctrl = torch.zeros(bc // 4, dtype=torch.int32, device=device)
        self.device = self.ctrl.get_device()
        sig = np.ascontiguousarray(rot_signs, dtype=np.int8)
        o8 = None if fp8_order is None else np.ascontiguousarray(fp8_order, dtype=np.int32)
        o3 = None if tq3_order is None else np.ascontiguousarray(tq3_order, dtype=np.int32)
        desc = PoolDesc(n_layers, n_q_heads, n_kv_heads, head_dim, PAGE, n_fp8_pages, n_tq3_pages,
                        recent_tokens, sig.ctypes.data,
                        None if o8 is None else o8.ctypes.data,
                        None if o3 is None else o3.ctypes.data,
                        self.fp8.data_ptr(), b8, self.fp8_scales.data_ptr(), bs,
                        self.tq3.data_ptr(), b3, self.ctrl.data_ptr(), bc)
        h = ctypes.c_void_p()
        torch.cuda.synchronize()
        _check("kv_pool_create", lib().kv_pool_create(ctypes.byref(desc), ctypes.byref(h)))
        self.handle = h

    # views in the documented layouts
    def fp8_view(self):
        return self.fp8.view(self.n_layers, self.n_fp8, self.n_kv_heads, 2 * PAGE * self.d)

    def fp8_scales_view(self):
        return self.fp8_scales.view(self.n_layers, self.n_fp8, self.n_kv_heads, 2)

    def tq3_view(self):
        return self.tq3[: self.n_layers * self.n_tq3 * self.n_kv_heads * (16 * self.d + 32)].view(
            self.n_layers, self.n_tq3, self.n_kv_heads, 16 * self.d + 32)

    def close(self):
        if getattr(self, "handle", None):
            lib().kv_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def kv_append_fp8(pool: Pool, layer, block_table, tags, seq_lens_before, cu_new_tokens, k, v,
                  stream=None):
    n_req, max_pages = block_table.shape
    n_new = int(k.shape[-3]) if k is not None else 0
    _check("kv_append_fp8", lib().kv_append_fp8(
        pool.handle, layer, n_req, _ptr(block_table), _ptr(tags), max_pages, _ptr(seq_lens_before),
        _ptr(cu_new_tokens), n_new, _ptr(k), _ptr(v), _stream(stream)))


def kv_migrate_to_tq3(pool: Pool, block_table, tags, anchor_mask, seq_lens, stream=None):
    n_req, max_pages = block_table.shape
    _check("kv_migrate_to_tq3", lib().kv_migrate_to_tq3(
        pool.handle, n_req, _ptr(block_table), _ptr(tags), max_pages, _ptr(anchor_mask),
        _ptr(seq_lens), _stream(stream)))


def kv_promote_to_fp8(pool: Pool, block_table, tags, promote_mask, seq_lens, stream=None):
    n_req, max_pages = block_table.shape
    _check("kv_promote_to_fp8", lib().kv_promote_to_fp8(
        pool.handle, n_req, _ptr(block_table), _ptr(tags), max_pages, _ptr(promote_mask),
        _ptr(seq_lens), _stream(stream)))


def kv_pages_acquire(pool: Pool, ids, tags, stream=None):
    """SealPrefix / prefix attach: one more reference per listed page (device tensors)."""
    _check("kv_pages_acquire", lib().kv_pages_acquire(pool.handle, int(ids.numel()), _ptr(ids),
                                                      _ptr(tags), _stream(stream)))


def kv_pages_release(pool: Pool, ids, tags, stream=None):
    """Prefix eviction: one reference fewer per listed page (device tensors)."""
    _check("kv_pages_release", lib().kv_pages_release(pool.handle, int(ids.numel()), _ptr(ids),
                                                      _ptr(tags), _stream(stream)))


def kv_request_finish(pool: Pool, reqs, block_table, tags, stream=None):
    """Finish(q) of the requests in `reqs` (device int32, ascending)."""
    n_req, max_pages = block_table.shape
    _check("kv_request_finish", lib().kv_request_finish(
        pool.handle, int(reqs.numel()), _ptr(reqs), n_req, _ptr(block_table), _ptr(tags),
        max_pages, _stream(stream)))


def kv_pool_read_refcounts(pool: Pool):
    r8 = np.zeros(pool.n_fp8, np.int32)
    r3 = np.zeros(max(pool.n_tq3, 1), np.int32)
    _check("kv_pool_read_refcounts", lib().kv_pool_read_refcounts(pool.handle, r8.ctypes.data,
                                                                  r3.ctypes.data))
    return r8, r3[: pool.n_tq3]


def paged_attn_workspace_bytes(pool: Pool, n_req, max_pages, n_q_total=0):
    out = ctypes.c_size_t()
    _check("paged_attn_workspace_bytes", lib().paged_attn_workspace_bytes(
        pool.handle, n_req, max_pages, n_q_total, ctypes.byref(out)))
    return out.value


def workspace(pool: Pool, n_req, max_pages, n_q_total=0, device="cuda"):
    import torch
    return torch.zeros(paged_attn_workspace_bytes(pool, n_req, max_pages, n_q_total),
                       dtype=torch.uint8, device=device)


def paged_attn_workspace_init(ws, stream=None):
    _check("paged_attn_workspace_init", lib().paged_attn_workspace_init(
        _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def paged_attn_decode(pool: Pool, layer, q, block_table, tags, seq_lens, out, lse, ws,
                      stream=None):
    n_req, max_pages = block_table.shape
    _check("paged_attn_decode", lib().paged_attn_decode(
        pool.handle, layer, n_req, _ptr(q), _ptr(block_table), _ptr(tags), max_pages,
        _ptr(seq_lens), _ptr(out), _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)))


def paged_attn_decode_scores(pool: Pool, layer, q, block_table, tags, seq_lens, out, lse, ws,
                             page_mass, stream=None):
    """paged_attn_decode that also writes each page's local mass and reference
    exponent (page_mass: device float32 [n_req][max_pages][n_q_heads][2])."""
    n_req, max_pages = block_table.shape
    _check("paged_attn_decode_scores", lib().paged_attn_decode_scores(
        pool.handle, layer, n_req, _ptr(q), _ptr(block_table), _ptr(tags), max_pages,
        _ptr(seq_lens), _ptr(out), _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(),
        _ptr(page_mass), _stream(stream)))


def kv_page_scores_update(pool: Pool, seq_lens, lse, page_mass, head_mask, beta, scores,
                          r_out=None, qn_out=None, stream=None):
    n_req, max_pages = scores.shape
    _check("kv_page_scores_update", lib().kv_page_scores_update(
        pool.handle, n_req, max_pages, _ptr(seq_lens), _ptr(lse), _ptr(page_mass),
        _ptr(head_mask), float(beta), _ptr(scores), _ptr(r_out), _ptr(qn_out), _stream(stream)))


DECODE_SCRATCH_BYTES = 32 * 1024 * 1024


def paged_attn_decode_noalloc(pool: Pool, layer, q, block_table, tags, seq_lens, out, lse,
                              stream=None):
    """paged_attn_decode with the split partials in the library's fixed device
    scratch (no workspace argument; the call allocates nothing)."""
    n_req, max_pages = block_table.shape
    _check("paged_attn_decode_noalloc", lib().paged_attn_decode_noalloc(
        pool.handle, layer, n_req, _ptr(q), _ptr(block_table), _ptr(tags), max_pages,
        _ptr(seq_lens), _ptr(out), _ptr(lse), _stream(stream)))


def paged_attn_decode_append(pool: Pool, layer, q, k_new, v_new, block_table, tags,
                             seq_lens_before, out, lse, ws, stream=None):
    n_req, max_pages = block_table.shape
    _check("paged_attn_decode_append", lib().paged_attn_decode_append(
        pool.handle, layer, n_req, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(block_table),
        _ptr(tags), max_pages, _ptr(seq_lens_before), _ptr(out), _ptr(lse), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))


class Rope:
    """Rotary positions (kv_rope): pair i of a head turns by positions[axis[i]] *
    inv_freq[i].  2 * len(inv_freq) channels are rotated, pairs (i, i + half) or,
    interleaved, (2i, 2i + 1).  The table lives in a torch tensor of this object."""

    def __init__(self, head_dim, inv_freq, axis=None, n_axes=1, interleaved=False, scale=1.0, device="cuda"):
        import torch
        f = np.ascontiguousarray(inv_freq, dtype=np.float64)
        ax = None if axis is None else np.ascontiguousarray(axis, dtype=np.uint8)
        if f.ndim != 1 or (ax is not None and ax.shape != f.shape):
            raise ValueError("inv_freq is a vector and axis, if given, one of the same length")
        self.head_dim, self.rot_dim, self.n_axes = head_dim, 2 * f.size, n_axes
        b = ctypes.c_size_t()
        _check("kv_rope_bytes", lib().kv_rope_bytes(self.rot_dim, ctypes.byref(b)))
        self.table = torch.zeros(b.value, dtype=torch.uint8, device=device)
        self.device = self.table.get_device()
        desc = RopeDesc(head_dim, self.rot_dim, n_axes, int(bool(interleaved)), float(scale), f.ctypes.data,
                        None if ax is None else ax.ctypes.data, self.table.data_ptr(), b.value)
        h = ctypes.c_void_p()
        torch.cuda.synchronize(self.table.device)
        _check("kv_rope_create", lib().kv_rope_create(ctypes.byref(desc), ctypes.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            lib().kv_rope_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _rows(dev, t, shape):
    """Elements from one row [heads][d] of t, of this shape, to the next; the heads lie together."""
    if t.get_device() != dev or t.dtype not in _types()[0]:
        raise ValueError("rows are bf16 (or its bits in int16) on the current device")
    if t.is_contiguous():
        return shape[-2] * shape[-1]
    n, heads, d = shape[-3:]
    st = t.stride()
    if st[-1] != 1 or (heads > 1 and st[-2] != d):
        raise ValueError("rows are [heads][head_dim] without gaps")
    layers = shape[0] if len(shape) == 4 else 1
    stride = st[-3] if n > 1 else st[0] if layers > 1 else heads * d
    if layers > 1 and st[0] != n * stride:
        raise ValueError("one layer's rows follow the other's")
    return stride


def _positions(dev, rope, positions, n):
    if rope.device != dev:
        raise ValueError("the rope's table is on another device")
    if positions is None:
        return None
    if (positions.shape != (rope.n_axes, n) or positions.get_device() != dev or positions.dtype not in _types()[1]
            or not positions.is_contiguous()):
        raise ValueError(f"positions are contiguous int32 [{rope.n_axes}][{n}] on the current device")
    return positions.data_ptr()


def kv_rope_apply(rope: Rope, x, positions, out, stream=None):
    """Rotate bf16 rows x [n][heads][head_dim] (int16 bits, tokens may be strided) into out;
    positions: int32 [n_axes][n]."""
    dev, cur = _current()
    shape = x.shape
    n, heads, d = shape
    if out.shape != shape or d != rope.head_dim:
        raise ValueError("x and out are [n][heads][head_dim]")
    _check("kv_rope_apply", lib().kv_rope_apply(
        rope.handle, n, heads, x.data_ptr(), _rows(dev, x, shape), _positions(dev, rope, positions, n), out.data_ptr(),
        _rows(dev, out, shape), cur if stream is None else stream.cuda_stream))


class HeadNorm:
    """Norm of query or key heads (kv_head_norm): rows times 1 / sqrt(mean x^2 + eps) and the weights,
    bf16 (or its bits in int16) [head_dim], [heads][head_dim] or [layers][heads][head_dim]; None: ones.
    unit_offset: the weights are kept as differences from one.  The object holds the tensor, whose
    values may change and whose memory may be replaced (as moving a module's parameters does), and is
    otherwise fixed."""

    def __init__(self, head_dim, weight=None, eps=1e-6, unit_offset=False):
        self.head_dim = head_dim
        self._weight, self._shape, self._dev = weight, (), None
        self._desc = HeadNormDesc(head_dim, float(eps), 1.0 if unit_offset else 0.0, None, 0, 0)
        self._ref = ctypes.byref(self._desc)
        if weight is not None:
            self._take()

    def _take(self):
        """The weights as they lie now, into the description."""
        w, d = self._weight, self.head_dim
        s = tuple(w.shape)
        if w.dtype not in _types()[0] or not w.is_contiguous() or not 1 <= len(s) <= 3 or s[-1] != d:
            raise ValueError("weights are contiguous bf16 (or its bits in int16), [..][head_dim]")
        self._shape, self._dev = s, w.get_device()
        desc = self._desc
        desc.head_stride, desc.layer_stride = d if len(s) > 1 else 0, s[-2] * d if len(s) > 2 else 0
        desc.weight = w.data_ptr()

    @property
    def weight(self):
        return self._weight

    def _for(self, dev, heads, layers=1):
        """The description, for rows of `heads` heads and `layers` layers on device dev."""
        w = self._weight
        if w is not None and w.data_ptr() != self._desc.weight:
            self._take()
        s = self._shape
        if s and (self._dev != dev or len(s) > 1 and s[-2] != heads or len(s) > 2 and s[0] != layers):
            raise ValueError(f"weights are [head_dim], [{heads}][head_dim] or [{layers}][{heads}][head_dim] on the "
                             "current device")
        return self._ref


def kv_norm_rope_apply(rope, norm: HeadNorm, x, positions, out, stream=None):
    """Every head of bf16 rows x [n][heads][head_dim] normed and rotated into out; rope None: normed
    only (positions are not read).  positions: int32 [n_axes][n]."""
    dev, cur = _current()
    shape = x.shape
    n, heads, d = shape
    if out.shape != shape or d != norm.head_dim or (rope is not None and d != rope.head_dim):
        raise ValueError("x and out are [n][heads][head_dim]")
    _check("kv_norm_rope_apply", lib().kv_norm_rope_apply(
        None if rope is None else rope.handle, norm._for(dev, heads), n, heads, x.data_ptr(), _rows(dev, x, shape),
        None if rope is None else _positions(dev, rope, positions, n), out.data_ptr(), _rows(dev, out, shape),
        cur if stream is None else stream.cuda_stream))


def _append_rows(dev, pool, layer, block_table, tags, seq_lens_before, cu_new_tokens, k, v):
    """(n_req, max_pages, shape of k and v) of an append of strided rows."""
    i32 = _types()[1]
    n_req, max_pages = _table(dev, pool, block_table, tags, i32)
    shape = k.shape
    ok = v.shape == shape
    if layer >= 0:
        ok = ok and len(shape) == 3
    else:
        ok = ok and len(shape) == 4 and shape[0] == pool.n_layers
    if not ok or shape[-2] != pool.n_kv_heads or shape[-1] != pool.d:
        raise ValueError("k and v are [n][H][head_dim], with all layers [n_layers][n][H][head_dim]")
    _here(dev, seq_lens_before, cu_new_tokens)
    if not (seq_lens_before.dtype in i32 and cu_new_tokens.dtype in i32):
        raise ValueError(_WRONG_TYPE)
    if seq_lens_before.numel() < n_req or cu_new_tokens.numel() <= n_req:
        raise ValueError("seq_lens_before is [n_req], cu_new_tokens [n_req + 1]")
    return n_req, max_pages, shape


def kv_append_fp8_rope(pool: Pool, rope: Rope, layer, block_table, tags, seq_lens_before, cu_new_tokens,
                       positions, k, v, stream=None):
    """kv_append_fp8 with the keys rotated on the way; k, v: [n][H][d] of one layer or
    [n_layers][n][H][d], tokens may be strided; positions: int32 [n_axes][n] or None."""
    dev, cur = _current()
    n_req, max_pages, shape = _append_rows(dev, pool, layer, block_table, tags, seq_lens_before, cu_new_tokens, k, v)
    n = shape[-3]
    _check("kv_append_fp8_rope", lib().kv_append_fp8_rope(
        pool.handle, rope.handle, layer, n_req, block_table.data_ptr(), tags.data_ptr(), max_pages,
        seq_lens_before.data_ptr(), cu_new_tokens.data_ptr(), n, _positions(dev, rope, positions, n), k.data_ptr(),
        _rows(dev, k, shape), v.data_ptr(), _rows(dev, v, shape), cur if stream is None else stream.cuda_stream))


def kv_append_fp8_norm_rope(pool: Pool, rope, norm: HeadNorm, layer, block_table, tags, seq_lens_before, cu_new_tokens,
                            positions, k, v, stream=None):
    """kv_append_fp8_rope with every key head normed before its rotation; rope None: normed only."""
    dev, cur = _current()
    n_req, max_pages, shape = _append_rows(dev, pool, layer, block_table, tags, seq_lens_before, cu_new_tokens, k, v)
    n = shape[-3]
    _check("kv_append_fp8_norm_rope", lib().kv_append_fp8_norm_rope(
        pool.handle, None if rope is None else rope.handle,
        norm._for(dev, pool.n_kv_heads, shape[0] if layer < 0 else 1), layer, n_req, block_table.data_ptr(),
        tags.data_ptr(), max_pages, seq_lens_before.data_ptr(), cu_new_tokens.data_ptr(), n,
        None if rope is None else _positions(dev, rope, positions, n), k.data_ptr(), _rows(dev, k, shape), v.data_ptr(),
        _rows(dev, v, shape), cur if stream is None else stream.cuda_stream))


def paged_attn_decode_append_rope(pool: Pool, rope: Rope, layer, q, k_new, v_new, positions, block_table, tags,
                                  seq_lens_before, out, lse, ws, stream=None):
    """paged_attn_decode_append with q and k_new rotated in the launch; positions: int32
    [n_axes][n_req] or None (the token's place in the cache)."""
    dev, cur = _current()
    rows, i32, f32 = _types()
    n_req, max_pages = _table(dev, pool, block_table, tags, i32)
    _here(dev, q, k_new, v_new, seq_lens_before, out, lse, ws)
    if not (q.dtype in rows and k_new.dtype in rows and v_new.dtype in rows and seq_lens_before.dtype in i32
            and out.dtype in f32 and (lse is None or lse.dtype in f32)):
        raise ValueError(_WRONG_TYPE)
    qs, ks = (n_req, pool.n_q_heads, pool.d), (n_req, pool.n_kv_heads, pool.d)
    if q.shape != qs or out.shape != qs or k_new.shape != ks or v_new.shape != ks:
        _sizes((q, qs), (out, qs), (k_new, ks), (v_new, ks))
    if seq_lens_before.numel() < n_req or (lse is not None and lse.numel() < qs[0] * qs[1]):
        raise ValueError("seq_lens_before is [n_req], lse [n_req][n_q_heads]")
    _check("paged_attn_decode_append_rope", lib().paged_attn_decode_append_rope(
        pool.handle, rope.handle, layer, n_req, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(),
        _positions(dev, rope, positions, n_req), block_table.data_ptr(), tags.data_ptr(), max_pages,
        seq_lens_before.data_ptr(), out.data_ptr(), _ptr(lse), ws.data_ptr(), ws.nbytes,
        cur if stream is None else stream.cuda_stream))


class PageBounds:
    """Channelwise extremes of the keys of every logical page, for page selection:
    codes uint8 (E4M3) [n_layers][n_req][H][max_pages][2][d] (largest, smallest) and
    scales float32 [n_layers][n_req][H][max_pages]."""

    def __init__(self, pool: Pool, n_req, max_pages, device="cuda"):
        import torch
        c, s = ctypes.c_size_t(), ctypes.c_size_t()
        _check("kv_page_bounds_bytes", lib().kv_page_bounds_bytes(pool.handle, n_req, max_pages,
                                                                  ctypes.byref(c), ctypes.byref(s)))
        shape = (pool.n_layers, n_req, pool.n_kv_heads, max_pages)
        self.n_req, self.max_pages = n_req, max_pages
        self.codes = torch.zeros((*shape, 2, pool.d), dtype=torch.uint8, device=device)
        self.scales = torch.zeros(shape, dtype=torch.float32, device=device)
        assert self.codes.numel() == c.value and self.scales.numel() * 4 == s.value


def _bounds(dev, b):
    """The tensors that b holds now, as the library takes them (it checks their sizes)."""
    codes, scales = b.codes, b.scales
    if (codes.get_device() != dev or scales.get_device() != dev or not codes.is_contiguous() or not scales.is_contiguous()
            or codes.element_size() != 1 or scales.dtype not in _types()[2]):
        raise ValueError("bounds are contiguous codes of a byte and float32 scales on the current device")
    return codes.data_ptr(), codes.numel(), scales.data_ptr(), 4 * scales.numel()


def kv_page_bounds_update(pool: Pool, layer, block_table, tags, seq_lens_from, seq_lens, bounds: PageBounds,
                          stream=None):
    """Recompute the bounds of the pages that hold tokens [seq_lens_from, seq_lens)."""
    dev, cur = _current()
    i32 = _types()[1]
    n_req, max_pages = _table(dev, pool, block_table, tags, i32)
    if n_req != bounds.n_req or max_pages != bounds.max_pages:
        raise ValueError("the bounds are those of another table shape")
    _here(dev, seq_lens_from, seq_lens)
    if not (seq_lens_from.dtype in i32 and seq_lens.dtype in i32):
        raise ValueError(_WRONG_TYPE)
    if seq_lens_from.numel() < n_req or seq_lens.numel() < n_req:
        raise ValueError("seq_lens_from and seq_lens are [n_req]")
    _check("kv_page_bounds_update", lib().kv_page_bounds_update(
        pool.handle, layer, n_req, block_table.data_ptr(), tags.data_ptr(), max_pages, seq_lens_from.data_ptr(),
        seq_lens.data_ptr(), *_bounds(dev, bounds), cur if stream is None else stream.cuda_stream))


def select_workspace(pool: Pool, n_req, max_pages, device="cuda"):
    import torch
    b = ctypes.c_size_t()
    _check("paged_attn_select_workspace_bytes", lib().paged_attn_select_workspace_bytes(
        pool.handle, n_req, max_pages, ctypes.byref(b)))
    return torch.empty(b.value, dtype=torch.uint8, device=device)


def paged_attn_select_pages(pool: Pool, layer, q, seq_lens, bounds: PageBounds, n_first, n_last, pages, counts, ws,
                            stream=None):
    """Per request and KV head the pages to attend to: pages int32 [n_req][H][n_select]
    (ascending, -1 behind), counts int32 [n_req][H]; q is the rotated query."""
    dev, cur = _current()
    n_req, H, n_select = pages.shape
    if n_req != bounds.n_req or H != pool.n_kv_heads or counts.shape != (n_req, H):
        raise ValueError("pages are [n_req][H][n_select], counts [n_req][H]")
    rows, i32, _ = _types()
    _here(dev, q, seq_lens, pages, counts, ws)
    if not (q.dtype in rows and seq_lens.dtype in i32 and pages.dtype in i32 and counts.dtype in i32):
        raise ValueError(_WRONG_TYPE)
    qs = (n_req, pool.n_q_heads, pool.d)
    if q.shape != qs:
        _sizes((q, qs))
    if seq_lens.numel() < n_req or pool.device != dev:
        raise ValueError("seq_lens is [n_req], the pool on the current device")
    _check("paged_attn_select_pages", lib().paged_attn_select_pages(
        pool.handle, layer, n_req, q.data_ptr(), seq_lens.data_ptr(), bounds.max_pages, *_bounds(dev, bounds), n_select,
        n_first, n_last, pages.data_ptr(), counts.data_ptr(), ws.data_ptr(), ws.nbytes,
        cur if stream is None else stream.cuda_stream))


def paged_attn_decode_sparse(pool: Pool, layer, q, block_table, tags, seq_lens, pages, counts, out, lse, ws,
                             stream=None):
    """paged_attn_decode over the listed logical pages of each request and KV head."""
    dev, cur = _current()
    rows, i32, f32 = _types()
    n_req, max_pages = _table(dev, pool, block_table, tags, i32)
    if pages.dim() != 3 or counts.shape != (n_req, pool.n_kv_heads) or pages.shape[:2] != counts.shape:
        raise ValueError("pages are [n_req][H][n_select], counts [n_req][H]")
    _here(dev, q, seq_lens, pages, counts, out, lse, ws)
    if not (q.dtype in rows and seq_lens.dtype in i32 and pages.dtype in i32 and counts.dtype in i32
            and out.dtype in f32 and (lse is None or lse.dtype in f32)):
        raise ValueError(_WRONG_TYPE)
    qs = (n_req, pool.n_q_heads, pool.d)
    if q.shape != qs or out.shape != qs:
        _sizes((q, qs), (out, qs))
    if seq_lens.numel() < n_req or (lse is not None and lse.numel() < qs[0] * qs[1]):
        raise ValueError("seq_lens is [n_req], lse [n_req][n_q_heads]")
    _check("paged_attn_decode_sparse", lib().paged_attn_decode_sparse(
        pool.handle, layer, n_req, q.data_ptr(), block_table.data_ptr(), tags.data_ptr(), max_pages,
        seq_lens.data_ptr(), pages.shape[2], pages.data_ptr(), counts.data_ptr(), out.data_ptr(), _ptr(lse),
        ws.data_ptr(), ws.nbytes, cur if stream is None else stream.cuda_stream))


class Shaping:
    """Scores and masks of shaped attention (paged_attn_shaping): softmax scale (0: 1 / sqrt(head_dim)),
    cap of the scores by a tanh (0: none), window of visible tokens (0: all), and device tensors or None:
    slopes float32 [n_q_heads] (bias -slope * distance), sinks float32 [n_q_heads], first_keys int32 [rows]
    (first token each query row sees), prefix_lens int32 [n_req] (tokens seen from both sides; chunks).
    The object holds the tensors, whose values may change and whose memory may be replaced, and is
    otherwise fixed."""

    def __init__(self, scale=0.0, cap=0.0, window=0, slopes=None, sinks=None, first_keys=None, prefix_lens=None):
        self._tensors = slopes, sinks, first_keys, prefix_lens
        self._where = [t.data_ptr for t in self._tensors if t is not None]
        self._desc = ShapingDesc(scale, cap, window)
        self._ref = ctypes.byref(self._desc)
        self._take()

    def _take(self):
        """The tensors as they lie now, into the description."""
        _, i32, f32 = _types()
        dev, most = None, []  # most: heads, heads, rows, requests that the tensors serve
        for t, types in zip(self._tensors, (f32, f32, i32, i32)):
            if t is None:
                most.append(1 << 62)
                continue
            if t.dtype not in types or not t.is_contiguous() or dev not in (None, t.get_device()):
                raise ValueError("slopes and sinks are float32, first_keys and prefix_lens int32, contiguous and on "
                                 "one device")
            dev = t.get_device()
            most.append(t.numel())
        self._dev, self._heads, self._rows, self._reqs = dev, min(most[:2]), most[2], most[3]
        d = self._desc
        d.slopes, d.sinks, d.first_keys, d.prefix_lens = map(_ptr, self._tensors)
        self._at = [p() for p in self._where]

    slopes = property(lambda self: self._tensors[0])
    sinks = property(lambda self: self._tensors[1])
    first_keys = property(lambda self: self._tensors[2])
    prefix_lens = property(lambda self: self._tensors[3])

    def _for(self, dev, heads, rows, n_req):
        """The description, for so many query heads, rows and requests on device dev."""
        if self._at != [p() for p in self._where]:
            self._take()
        if self._heads < heads or self._rows < rows or self._reqs < n_req or self._dev not in (None, dev):
            raise ValueError("slopes and sinks are [n_q_heads], first_keys [rows], prefix_lens [n_req], on the "
                             "current device")
        return self._ref


def paged_attn_decode_shaped(pool: Pool, shaping: Shaping, layer, q, block_table, tags, seq_lens, out, lse, ws,
                             stream=None):
    """paged_attn_decode with shaped scores and masks."""
    dev, cur = _current()
    rows, i32, f32 = _types()
    n_req, max_pages = _table(dev, pool, block_table, tags, i32)
    _here(dev, q, seq_lens, out, lse, ws)
    if not (q.dtype in rows and seq_lens.dtype in i32 and out.dtype in f32 and (lse is None or lse.dtype in f32)):
        raise ValueError(_WRONG_TYPE)
    qs = (n_req, pool.n_q_heads, pool.d)
    if q.shape != qs or out.shape != qs:
        _sizes((q, qs), (out, qs))
    if seq_lens.numel() < n_req or (lse is not None and lse.numel() < qs[0] * qs[1]):
        raise ValueError("seq_lens is [n_req], lse [n_req][n_q_heads]")
    desc = shaping._for(dev, pool.n_q_heads, n_req, n_req)
    _check("paged_attn_decode_shaped", lib().paged_attn_decode_shaped(
        pool.handle, desc, layer, n_req, q.data_ptr(), block_table.data_ptr(), tags.data_ptr(), max_pages,
        seq_lens.data_ptr(), out.data_ptr(), _ptr(lse), ws.data_ptr(), ws.nbytes,
        cur if stream is None else stream.cuda_stream))


def paged_attn_decode_append_shaped(pool: Pool, shaping: Shaping, rope, q_norm, k_norm, layer, q, k_new, v_new,
                                    positions, block_table, tags, seq_lens_before, out, lse, ws, stream=None):
    """A decode step of one layer: query and key heads normed (q_norm, k_norm: HeadNorm or None) and rotated
    (rope or None), the token appended, attention with shaped scores; positions as in
    paged_attn_decode_append_rope."""
    dev, cur = _current()
    rows, i32, f32 = _types()
    n_req, max_pages = _table(dev, pool, block_table, tags, i32)
    _here(dev, q, k_new, v_new, seq_lens_before, out, lse, ws)
    if not (q.dtype in rows and k_new.dtype in rows and v_new.dtype in rows and seq_lens_before.dtype in i32
            and out.dtype in f32 and (lse is None or lse.dtype in f32)):
        raise ValueError(_WRONG_TYPE)
    qs, ks = (n_req, pool.n_q_heads, pool.d), (n_req, pool.n_kv_heads, pool.d)
    if q.shape != qs or out.shape != qs or k_new.shape != ks or v_new.shape != ks:
        _sizes((q, qs), (out, qs), (k_new, ks), (v_new, ks))
    if seq_lens_before.numel() < n_req or (lse is not None and lse.numel() < qs[0] * qs[1]):
        raise ValueError("seq_lens_before is [n_req], lse [n_req][n_q_heads]")
    desc = shaping._for(dev, pool.n_q_heads, n_req, n_req)
    qd = None if q_norm is None else q_norm._for(dev, pool.n_q_heads)
    kd = None if k_norm is None else k_norm._for(dev, pool.n_kv_heads)
    _check("paged_attn_decode_append_shaped", lib().paged_attn_decode_append_shaped(
        pool.handle, desc, None if rope is None else rope.handle, qd, kd, layer, n_req, q.data_ptr(), k_new.data_ptr(),
        v_new.data_ptr(),
        None if rope is None else _positions(dev, rope, positions, n_req), block_table.data_ptr(), tags.data_ptr(),
        max_pages, seq_lens_before.data_ptr(), out.data_ptr(), _ptr(lse), ws.data_ptr(), ws.nbytes,
        cur if stream is None else stream.cuda_stream))


def kv_read_tokens(pool: Pool, layer, block_table, tags, seq_from, cu_tokens, k, v, stream=None):
    """bf16 K and V rows of positions seq_from[r] .. of every request (cu_tokens[r+1] - cu_tokens[r]
    of them); k, v: [n][H][d] of one layer or [n_layers][n][H][d], tokens may be strided, either None."""
    dev, cur = _current()
    i32 = _types()[1]
    n_req, max_pages = _table(dev, pool, block_table, tags, i32)
    one = k if v is None else v
    if one is None:
        raise ValueError("k or v is wanted")
    shape = one.shape
    ok = k is None or k.shape == shape
    if layer >= 0:
        ok = ok and len(shape) == 3
    else:
        ok = ok and len(shape) == 4 and shape[0] == pool.n_layers
    if not ok or shape[-2] != pool.n_kv_heads or shape[-1] != pool.d:
        raise ValueError("k and v are [n][H][head_dim], with all layers [n_layers][n][H][head_dim]")
    n = shape[-3]
    _here(dev, seq_from, cu_tokens)
    if not (seq_from.dtype in i32 and cu_tokens.dtype in i32):
        raise ValueError(_WRONG_TYPE)
    if seq_from.numel() < n_req or cu_tokens.numel() <= n_req:
        raise ValueError("seq_from is [n_req], cu_tokens [n_req + 1]")
    ks, vs = [0 if t is None else _rows(dev, t, shape) for t in (k, v)]
    _check("kv_read_tokens", lib().kv_read_tokens(
        pool.handle, layer, n_req, block_table.data_ptr(), tags.data_ptr(), max_pages, seq_from.data_ptr(),
        cu_tokens.data_ptr(), n, _ptr(k), ks, _ptr(v), vs, cur if stream is None else stream.cuda_stream))


def paged_attn_chunk(pool: Pool, layer, q, cu_q, block_table, tags, seq_lens, out, ws,
                     stream=None):
    n_req, max_pages = block_table.shape
    _check("paged_attn_chunk", lib().paged_attn_chunk(
        pool.handle, layer, n_req, _ptr(q), _ptr(cu_q), int(q.shape[0]), _ptr(block_table),
        _ptr(tags), max_pages, _ptr(seq_lens), _ptr(out), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)))


def paged_attn_chunk_shaped(pool: Pool, shaping: Shaping, layer, q, cu_q, block_table, tags, seq_lens, out, ws,
                            stream=None):
    """paged_attn_chunk with shaped scores and masks; out: bf16 (or its bits in int16) [n][n_q_heads][head_dim]."""
    dev, cur = _current()
    rows, i32, _ = _types()
    n_req, max_pages = _table(dev, pool, block_table, tags, i32)
    _here(dev, q, cu_q, seq_lens, out, ws)
    if not (q.dtype in rows and out.dtype in rows and cu_q.dtype in i32 and seq_lens.dtype in i32):
        raise ValueError("q and out are bf16 (or its bits in int16), lengths int32")
    if q.shape != (q.shape[0], pool.n_q_heads, pool.d) or out.shape != q.shape:
        raise ValueError("q and out are [n][n_q_heads][head_dim]")
    if cu_q.numel() <= n_req or seq_lens.numel() < n_req:
        raise ValueError("cu_q is [n_req + 1], seq_lens [n_req]")
    desc = shaping._for(dev, pool.n_q_heads, q.shape[0], n_req)
    _check("paged_attn_chunk_shaped", lib().paged_attn_chunk_shaped(
        pool.handle, desc, layer, n_req, q.data_ptr(), cu_q.data_ptr(), q.shape[0], block_table.data_ptr(),
        tags.data_ptr(), max_pages, seq_lens.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.nbytes,
        cur if stream is None else stream.cuda_stream))


def kv_partition_pages(block_table, tags, seq_lens, list8, list3, counts, stream=None):
    n_req, max_pages = block_table.shape
    _check("kv_partition_pages", lib().kv_partition_pages(
        n_req, _ptr(block_table), _ptr(tags), max_pages, _ptr(seq_lens), _ptr(list8), _ptr(list3),
        _ptr(counts), _stream(stream)))


def kv_pool_free_counts(pool: Pool):
    a, b = ctypes.c_int32(), ctypes.c_int32()
    _check("kv_pool_free_counts", lib().kv_pool_free_counts(pool.handle, ctypes.byref(a),
                                                             ctypes.byref(b)))
    return a.value, b.value


def kv_pool_read_free_lists(pool: Pool):
    f8 = np.zeros(pool.n_fp8, np.int32)
    f3 = np.zeros(max(pool.n_tq3, 1), np.int32)
    n8, n3 = ctypes.c_int32(), ctypes.c_int32()
    _check("kv_pool_read_free_lists", lib().kv_pool_read_free_lists(
        pool.handle, f8.ctypes.data, ctypes.byref(n8), f3.ctypes.data, ctypes.byref(n3)))
    return f8[: n8.value].copy(), f3[: n3.value].copy()


def kv_pool_counters(pool: Pool) -> dict:
    c = Counters()
    _check("kv_pool_counters", lib().kv_pool_counters(pool.handle, ctypes.byref(c)))
    return {n: getattr(c, n) for n, _ in Counters._fields_}


def paged_attn_set_deterministic(pool: Pool, enable: bool) -> None:
    _check("paged_attn_set_deterministic",
           lib().paged_attn_set_deterministic(pool.handle, int(bool(enable))))


def paged_attn_set_timing(pool: Pool, enable: bool) -> None:
    _check("paged_attn_set_timing", lib().paged_attn_set_timing(pool.handle, int(bool(enable))))


def paged_attn_last_times(pool: Pool) -> tuple:
    """(scan_us, merge_us) of the last timed paged_attn_decode call (waits for it)."""
    a, b = ctypes.c_float(), ctypes.c_float()
    _check("paged_attn_last_times", lib().paged_attn_last_times(pool.handle, ctypes.byref(a),
                                                                ctypes.byref(b)))
    return a.value, b.value


STREAM_PROBE_WORKGROUPS = 2048


def mkv_stream_read(buf, sink, stream=None):
    """Streaming-read probe (measurement only): reads the device tensor `buf`
    once; `sink` is a device int32 tensor of STREAM_PROBE_WORKGROUPS words."""
    assert sink.numel() >= STREAM_PROBE_WORKGROUPS
    _check("mkv_stream_read", lib().mkv_stream_read(
        _ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), _stream(stream)))


def mkv_fp64_probe(a, b, quot, root, half, stream=None):
    """Conformance probe (tests only): quot = a / b, root = sqrt(a), half =
    binary16(a), by the library's own compiled fp64 code (device tensors)."""
    n = a.numel()
    assert b.numel() == n and quot.numel() == n and root.numel() == n and half.numel() == n
    _check("mkv_fp64_probe", lib().mkv_fp64_probe(_ptr(a), _ptr(b), n, _ptr(quot), _ptr(root),
                                                  _ptr(half), _stream(stream)))


def paged_attn_decode_cohort_key(pool: Pool, n_req, max_pages, fused_append=True, scoring=False):
    key = ctypes.c_uint64()
    _check("paged_attn_decode_cohort_key", lib().paged_attn_decode_cohort_key(
        pool.handle, n_req, max_pages, int(bool(fused_append)), int(bool(scoring)),
        ctypes.byref(key)))
    return key.value


class DecodeStepGraph:
    """A decode step (per layer paged_attn_decode_append, then
    kv_migrate_to_tq3) captured once into a HIP graph and replayed for later
    steps of the same cohort (Sec. 4.1 graph path gated on a homogeneous
    cohort).  The step reads its inputs from fixed device buffers -- q
    [n_layers][n_req][Hq][d], k_new / v_new [n_layers][n_req][Hkv][d],
    seq_lens_before [n_req], seq_lens_after [n_req], anchor mask -- which the
    caller refills before each run.  run(key) replays only when `key` (the
    cohort key of the step about to run) equals the key captured; otherwise it
    fails closed to launching the same calls directly.  Host orchestration
    only: the work is the library's kernels either way."""

    def __init__(self, pool: Pool, block_table, tags, bufs: dict, out, lse, ws):
        self.pool, self.bt, self.tags, self.b, self.out, self.lse, self.ws = (
            pool, block_table, tags, bufs, out, lse, ws)
        n_req, max_pages = block_table.shape
        self.key = paged_attn_decode_cohort_key(pool, n_req, max_pages, True, False)
        self.graph = None
        self.replays = 0
        self.direct = 0

    def _step(self):
        b = self.b
        for layer in range(self.pool.n_layers):
            paged_attn_decode_append(self.pool, layer, b["q"][layer], b["k_new"][layer],
                                     b["v_new"][layer], self.bt, self.tags, b["seq_before"],
                                     self.out[layer], self.lse[layer], self.ws)
        kv_migrate_to_tq3(self.pool, self.bt, self.tags, b["anchor"], b["seq_after"])

    def capture(self):
        """Capture one step (every kernel instance it uses must have run once
        on this device before, so that no launch attribute is set inside)."""
        import torch
        g = torch.cuda.CUDAGraph()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=s):
            self._step()
        torch.cuda.current_stream().wait_stream(s)
        self.graph = g

    def run(self, key):
        if self.graph is not None and key == self.key:
            self.graph.replay()
            self.replays += 1
        else:
            self._step()
            self.direct += 1


class ControlBf16:
    """Dense bf16 control pages (measurement only): the same KV as the mixed
    pool held as bf16, for timing the mixed path against an uncompressed
    cache.  Page ids come from the caller's block table."""

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, n_pages, device="cuda"):
        import torch
        self.n_layers, self.n_q_heads, self.n_kv_heads, self.d = n_layers, n_q_heads, n_kv_heads, head_dim
        self.n_pages = n_pages
        self.pages = torch.zeros((n_layers, n_pages, n_kv_heads, 2 * PAGE * head_dim),
                                 dtype=torch.int16, device=device)

    def write(self, layer, block_table, seq_lens_before, cu_new_tokens, k, v, stream=None):
        n_req, max_pages = block_table.shape
        _check("mkv_control_bf16_write", lib().mkv_control_bf16_write(
            _ptr(self.pages), self.n_pages, self.n_layers, self.n_kv_heads, self.d, layer, n_req,
            _ptr(block_table), max_pages, _ptr(seq_lens_before), _ptr(cu_new_tokens),
            int(k.shape[0]), _ptr(k), _ptr(v), _stream(stream)))

    def workspace(self, n_req, max_pages, device="cuda"):
        import torch
        b = ctypes.c_size_t()
        _check("mkv_control_bf16_workspace_bytes", lib().mkv_control_bf16_workspace_bytes(
            n_req, max_pages, self.n_kv_heads, self.n_q_heads, self.d, ctypes.byref(b)))
        return torch.empty(b.value, dtype=torch.uint8, device=device)

    def decode(self, layer, q, block_table, seq_lens, out, lse, ws, stream=None):
        n_req, max_pages = block_table.shape
        _check("mkv_control_bf16_decode", lib().mkv_control_bf16_decode(
            _ptr(self.pages), self.n_pages, self.n_layers, self.n_kv_heads, self.n_q_heads, self.d,
            layer, n_req, _ptr(q), _ptr(block_table), max_pages, _ptr(seq_lens), _ptr(out),
            _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def kv_pool_check_errors(pool: Pool, clear=False) -> int:
    e = ctypes.c_uint32()
    _check("kv_pool_check_errors", lib().kv_pool_check_errors(pool.handle, ctypes.byref(e),
                                                               int(bool(clear))))
    return e.value
