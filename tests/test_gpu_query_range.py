"""Queries far outside fp16's numbers.  A power of two on the queries, and its inverse on the softmax scale or on the
keys, changes no significand anywhere, so the rows have to be the same bits."""
import numpy as np
import pytest

import mkv_workloads as wl
import _rope_ref as ref
import _shape_ref as sref
from test_gpu_shaped import _decode, _i16, _i32, _slopes, _twin, _w
from test_gpu_shaped_chunk import _chunk, _near

pytestmark = pytest.mark.gpu
BASE = float(np.float32(0.08))


def _scaled(q, k):
    """bf16 rows times 2^k (none of these leaves bf16's normal numbers)."""
    return wl.bf16_round((wl.bf16_to_f32(q) * np.float32(2.0 ** k)).astype(np.float32))


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("kw", [{}, dict(cap=5.0), dict(cap=200.0), dict(slopes=_slopes(8))])
def test_shaped(d, kw):
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(d)
    lens, nq = [700, 333, 40], [60, 1, 40]
    t = _twin(_w(d, 8, 2, 3), lens, recent=128)
    assert (t.otags == 2).any() and (t.otags != 2).any()
    cu = np.r_[0, np.cumsum(nq)]
    q = wl.bf16_round((2 * rng.standard_normal((cu[-1], 8, d))).astype(np.float32))
    mk.paged_attn_set_deterministic(t.gpu, True)
    rows, (out, lse) = _chunk(t, q, cu, dict(kw, scale=BASE)), _decode(t, q[:3], dict(kw, scale=BASE))
    _near(rows, sref.chunk(t.orc, 0, ref.bf16_f64(q), cu, t.obt, t.otags, t.cur, dict(kw, scale=BASE)))
    for k in (-19, -9, 8, 15):
        far = dict(kw, scale=BASE * 2.0 ** -k)
        assert np.array_equal(_chunk(t, _scaled(q, k), cu, far), rows), k
        o, l = _decode(t, _scaled(q[:3], k), far)
        assert np.array_equal(o, out) and np.array_equal(l, lse), k
    assert mk.kv_pool_check_errors(t.gpu) == 0


@pytest.mark.parametrize("d", [128, 256])
def test_plain_chunk(d):
    import paper_2608_23834_amd as mk
    from _harness import Twin, _torch
    torch = _torch()
    rng = np.random.default_rng(d)
    n, nq = 300, 40
    w = _w(d, 8, 2, 1)
    q = wl.bf16_round((2 * rng.standard_normal((nq, 8, d))).astype(np.float32))
    kv = wl.bf16_round(rng.standard_normal((2, n, 2, d)).astype(np.float32))
    got = []
    for k in (0, 15, -30):
        t = Twin(w, n_layers=1, lens=[n], recent=1 << 20, with_oracle=False)
        t.append([n], layer_kv=(_scaled(kv[0], -k)[None], kv[1][None]))
        out = torch.zeros((nq, 8, d), device="cuda")
        mk.paged_attn_chunk(t.gpu, 0, _i16(_scaled(q, k)), _i32([0, nq]), t.bt, t.tags, _i32([n]), out,
                            mk.workspace(t.gpu, 1, t.max_pages, nq))
        assert mk.kv_pool_check_errors(t.gpu) == 0
        got.append(out.cpu().numpy())
    assert np.isfinite(got[0]).all() and got[0].any()
    assert np.array_equal(got[1], got[0]) and np.array_equal(got[2], got[0])
