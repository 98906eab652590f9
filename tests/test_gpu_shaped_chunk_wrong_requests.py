"""Shaped chunks whose last round is cut into parts, beside requests that have nothing to read: these get zeros
and their error, every other row is what it is without them."""
import numpy as np
import pytest

import _rope_ref as ref
import _shape_ref as sref
import mkv_workloads as wl
from test_gpu_shaped import _twin, _w
from test_gpu_shaped_chunk import _chunk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,hkv,lens,nq", [
    (128, 16, 1, [1556, 1581, 1556, 1646, 1669], [639] * 5),   # 400 row blocks for 256 compute units
    (256, 24, 4, [1932, 1932, 1932, 1932, 1932, 2110], [432] * 6),  # 126 for 64
])
def test_requests_with_nothing_to_read(d, hq, hkv, lens, nq):
    """One request with fewer tokens than queries, without queries, or without a readable page, in every place: a
    row block of no pages is a work item like the others.  The workspace holds NaN before each call."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(hq)
    t = _twin(_w(d, hq, hkv, len(lens)), lens, recent=256)
    cu = np.r_[0, np.cumsum(nq)]
    q = wl.bf16_round((2 * rng.standard_normal((cu[-1], hq, d))).astype(np.float32))
    kw = dict(cap=6.0, sinks=np.ones(hq))
    out, tol = sref.chunk(t.orc, 0, ref.bf16_f64(q), cu, t.obt, t.otags, t.cur, kw)
    for j in range(len(lens)):
        own = np.arange(cu[j], cu[j + 1])
        others = np.setdiff1d(np.arange(cu[-1]), own)

        def valid(got, what):
            err = np.linalg.norm(got - out[others], axis=2)
            assert np.all(err <= tol[others]), (j, what, np.argwhere(~(err <= tol[others]))[:4])

        wrong = list(t.cur)
        wrong[j] = nq[j] - 1
        got = _chunk(t, q, cu, kw, lens=wrong)
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]
        assert np.all(got[own] == 0)
        valid(got[others], "fewer tokens than queries")

        counts = list(nq)
        counts[j] = 0
        valid(_chunk(t, q[others], np.r_[0, np.cumsum(counts)], kw), "no queries")
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]

        tags = t.tags.clone()
        t.tags[j] = 0xFF
        got = _chunk(t, q, cu, kw)
        t.tags.copy_(tags)
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["BAD_TAG"]
        assert np.all(got[own] == 0)
        valid(got[others], "no readable page")
    valid_all = np.linalg.norm(_chunk(t, q, cu, kw) - out, axis=2)
    assert np.all(valid_all <= tol) and mk.kv_pool_check_errors(t.gpu) == 0
