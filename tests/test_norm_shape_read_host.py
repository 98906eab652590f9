"""Refusals of the normed rotation and append, shaped attention and the reading back of the cache: every
bad argument is refused on the host, before the device is touched."""
import ctypes

import pytest

P = ctypes.c_void_p
A, B = P(1 << 20), P(1 << 30)  # aligned placeholders, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def mk():
    import paper_2608_23834_amd as mk
    mk.lib()
    return mk


def _norm(mk, **kw):
    d = mk.HeadNormDesc(128, 1e-6, 0.0, 1 << 20, 128, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return ctypes.byref(d)


def _rows(mk, norm, n=4, heads=2, x=A, xs=256, pos=A, out=B, os=256, rope=None):
    return mk.lib().kv_norm_rope_apply(rope, norm, n, heads, x, xs, pos, out, os, None)


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=64), 2), (dict(head_dim=0), 2), (dict(eps=0.0), 4), (dict(eps=-1.0), 4), (dict(eps=1.5), 4),
    (dict(eps=float("nan")), 4), (dict(add=float("nan")), 4), (dict(add=float("inf")), 4), (dict(add=-2e6), 4),
    (dict(weight=(1 << 20) + 2), 1), (dict(weight=(1 << 20) + 4), 1), (dict(head_stride=-4), 1), (dict(head_stride=2), 1),
    (dict(layer_stride=-4), 1), (dict(layer_stride=7), 1), (dict(head_stride=(1 << 31) + 4), 4),
    (dict(layer_stride=1 << 40), 4),
])
def test_norms(mk, kw, code):
    assert _rows(mk, _norm(mk, **kw)) == code
    assert _rows(mk, _norm(mk, **kw), n=0) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), 1), (dict(heads=0), 1), (dict(x=None), 1), (dict(out=None), 1), (dict(xs=252), 1), (dict(xs=258), 1),
    (dict(os=128), 1), (dict(x=P((1 << 20) + 2)), 1), (dict(out=P((1 << 30) + 4)), 1), (dict(xs=(1 << 31) + 4), 4),
    (dict(heads=1 << 24, xs=1 << 31, os=1 << 31), 4), (dict(out=P((1 << 20) + 512)), 1), (dict(out=A, os=512), 1),
])
def test_rows(mk, kw, code):
    assert _rows(mk, _norm(mk), **kw) == code


def test_no_rows_and_no_norm(mk):
    assert _rows(mk, _norm(mk), n=0, x=None, out=None) == 0
    assert _rows(mk, None) == 1


def test_null_handles(mk):
    L, sh, n = mk.lib(), ctypes.byref(mk.ShapingDesc()), _norm(mk)
    assert L.kv_append_fp8_norm_rope(None, None, n, 0, 1, A, A, 1, A, A, 1, None, A, 256, B, 256, None) == 1
    assert L.paged_attn_decode_shaped(None, sh, 0, 1, A, A, A, 1, A, A, None, A, 1 << 30, None) == 1
    assert L.paged_attn_decode_append_shaped(None, sh, None, n, n, 0, 1, A, A, A, None, A, A, 1, A, A, None, A, 1 << 30,
                                             None) == 1
    assert L.paged_attn_chunk_shaped(None, sh, 0, 1, A, A, 1, A, A, 1, A, A, A, 1 << 30, None) == 1
    assert L.kv_read_tokens(None, 0, 1, A, A, 1, A, A, 1, A, 256, B, 256, None) == 1


@pytest.mark.parametrize("kw,code", [
    (dict(window=-1), 1), (dict(cap=-1.0), 4), (dict(cap=float("nan")), 4), (dict(cap=float("inf")), 4), (dict(cap=2e6), 4),
    (dict(cap=1e-7), 4), (dict(scale=-0.5), 4), (dict(scale=float("nan")), 4), (dict(scale=1e7), 4), (dict(slopes=2), 1),
    (dict(sinks=(1 << 20) + 1), 1), (dict(first_keys=3), 1), (dict(prefix_lens=(1 << 20) + 2), 1),
])
def test_shapings(mk, kw, code):
    """(the chunk call looks at the shaping before the pool)"""
    sh = mk.ShapingDesc(**kw)
    assert mk.lib().paged_attn_chunk_shaped(None, ctypes.byref(sh), 0, 1, A, A, 1, A, A, 1, A, A, A, 1 << 30, None) == code
    assert mk.lib().paged_attn_chunk_shaped(None, None, 0, 1, A, A, 1, A, A, 1, A, A, A, 1 << 30, None) == 1
