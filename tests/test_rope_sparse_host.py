"""Refusals of the rotation, rotated-append, page-selection and sparse-attention calls: every
bad argument is refused on the host, before the device is touched."""
import ctypes

import numpy as np
import pytest

import _rope_ref as ref

P = ctypes.c_void_p
A = P(1 << 20)  # aligned placeholder, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def mk():
    import paper_2608_23834_amd as mk
    mk.lib()
    return mk


def _desc(mk, **kw):
    f = np.ones(64)
    d = mk.RopeDesc(128, 128, 1, 0, 1.0, f.ctypes.data, None, 1 << 20, 1024)
    d._keep = f
    for k, v in kw.items():
        if isinstance(v, np.ndarray):
            d.__dict__["_" + k] = v
            v = v.ctypes.data
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("rot,code", [(0, 1), (1, 1), (3, 1), (258, 1), (-2, 1), (2, 0), (256, 0)])
def test_rope_bytes(mk, rot, code):
    b = ctypes.c_size_t()
    assert mk.lib().kv_rope_bytes(rot, ctypes.byref(b)) == code
    if code == 0:
        assert b.value == rot // 2 * 16
    assert mk.lib().kv_rope_bytes(2, None) == 1


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=64), 2), (dict(rot_dim=130), 1), (dict(rot_dim=7), 1), (dict(rot_dim=0), 1),
    (dict(n_axes=0), 2), (dict(n_axes=5), 2), (dict(scale=0.0), 4), (dict(scale=float("nan")), 4),
    (dict(scale=-1.0), 4), (dict(inv_freq=None), 1), (dict(table=None), 1), (dict(table=(1 << 20) + 8), 1),
    (dict(table_bytes=1023), 3), (dict(inv_freq=np.full(64, 4.5)), 4), (dict(inv_freq=np.full(64, np.nan)), 4),
    (dict(inv_freq=np.full(64, -np.inf)), 4), (dict(axis=np.ones(64, np.uint8)), 4),
])
def test_rope_create_refuses(mk, kw, code):
    h = P()
    d = _desc(mk, **kw)
    assert mk.lib().kv_rope_create(ctypes.byref(d), ctypes.byref(h)) == code
    assert h.value is None


def test_null_handles_are_refused(mk):
    L = mk.lib()
    assert L.kv_rope_create(None, None) == 1
    assert L.kv_rope_destroy(None) == 1
    assert L.kv_rope_apply(None, 1, 1, A, 128, A, A, 128, None) == 1
    assert L.kv_append_fp8_rope(None, None, 0, 1, A, A, 1, A, A, 1, None, A, 128, A, 128, None) == 1
    assert L.paged_attn_decode_append_rope(None, None, 0, 1, A, A, A, None, A, A, 1, A, A, None, A, 0, None) == 1
    assert L.kv_page_bounds_bytes(None, 1, 1, None, None) == 1
    assert L.kv_page_bounds_update(None, 0, 1, A, A, 1, A, A, A, 0, A, 0, None) == 1
    assert L.paged_attn_select_workspace_bytes(None, 1, 1, None) == 1
    assert L.paged_attn_select_pages(None, 0, 1, A, A, 1, A, 0, A, 0, 1, 0, 0, A, A, A, 0, None) == 1
    assert L.paged_attn_decode_sparse(None, 0, 1, A, A, A, 1, A, 1, A, A, A, None, A, 0, None) == 1


def test_reference_rounds_once():
    # halfway between two bf16 values, and just past it by less than fp32 can hold
    x = np.array([1 + 2.0 ** -8, 1 + 2.0 ** -8 + 2.0 ** -40, 1 + 3 * 2.0 ** -8, -(1 + 2.0 ** -8) - 2.0 ** -45])
    assert ref.bf16_f64(ref.bf16_bits(x)).tolist() == [1.0, 1 + 2.0 ** -7, 1 + 2.0 ** -6, -(1 + 2.0 ** -7)]


def test_reference_selection_ties_and_nan():
    s = np.array([[[1.0, 3.0, 3.0, np.nan, 3.0, -np.inf, 0.0]]])
    pages, counts = ref.select(s, [7 * 16], 4, 0, 0)
    assert pages[0, 0].tolist() == [0, 1, 2, 4] and counts[0, 0] == 4
    pages, _ = ref.select(s, [7 * 16 - 3], 6, 1, 1)
    assert pages[0, 0].tolist() == [0, 1, 2, 4, 5, 6]  # NaN is below -inf


def test_e4m3_values():
    import oracle
    t = oracle.lib()
    got = ref.e4m3(np.arange(256, dtype=np.uint8))
    for c in range(256):
        if c & 127 != 127:
            assert got[c] == t.orc_e4m3_to_f64(c)
