"""Shaped chunks over tables whose first pages no row sees: these may be unmapped, or hold what is no number."""
import numpy as np
import pytest

import _rope_ref as ref
import _shape_ref as sref
import mkv_workloads as wl
from test_gpu_shaped import _slopes, _twin, _w
from test_gpu_shaped_chunk import _chunk, _near

pytestmark = pytest.mark.gpu
PAGE = 16


def _made(d, lens, nq, recent):
    rng = np.random.default_rng(d + lens[0])
    t = _twin(_w(d, 8, 2, len(lens)), lens, recent=recent)
    cu = np.r_[0, np.cumsum(nq)]
    return t, cu, wl.bf16_round((2 * rng.standard_normal((cu[-1], 8, d))).astype(np.float32))


def _first_pages(t, cu, kw):
    """Of every request, the first page that any of its rows sees (at most that of its first query)."""
    pages = []
    for r, n in enumerate(t.cur):
        p0 = n - (cu[r + 1] - cu[r])
        f = 0 if kw.get("first_keys") is None else int(np.min(kw["first_keys"][cu[r]:cu[r + 1]]))
        if kw.get("window"):
            f = max(f, p0 - kw["window"] + 1)
        pages.append(min(max(f, 0), p0) // PAGE)
    return pages


@pytest.mark.parametrize("d", [128, 256])
def test_pages_that_are_gone(d):
    import paper_2608_23834_amd as mk
    lens, nq = [1203, 40, 700, 2003], [40, 33, 300, 1]
    t, cu, q = _made(d, lens, nq, 256)
    bt, tags = t.bt.clone(), t.tags.clone()
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, nq)])
    none = pos + 5  # rows that see nothing
    for kw in (dict(window=1), dict(window=300, cap=5.0), dict(window=17, sinks=np.ones(8), slopes=_slopes(8)),
               dict(first_keys=pos // 130 * 130, prefix_lens=[1200, 3, 700, 0]), dict(first_keys=none, sinks=np.ones(8)),
               dict(first_keys=pos - 60, window=40)):
        want = sref.chunk(t.orc, 0, ref.bf16_f64(q), cu, t.obt, t.otags, t.cur, kw)
        first = _first_pages(t, cu, kw)
        assert any(first)
        for gone in ((0xFF, -1), (2, 10 ** 6), (1, -7)):
            for r, p in enumerate(first):
                t.tags[r, :p], t.bt[r, :p] = gone
            for det in (False, True):
                mk.paged_attn_set_deterministic(t.gpu, det)
                _near(_chunk(t, q, cu, kw), want)
            assert mk.kv_pool_check_errors(t.gpu) == 0
            t.tags.copy_(tags)
            t.bt.copy_(bt)
        t.tags[3, first[3]] = 0xFF  # the first page that is seen is checked
        _chunk(t, q, cu, kw)
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["BAD_TAG"]
        t.tags.copy_(tags)


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("recent", [64, 1 << 20])
def test_page_before_the_first_holds_no_numbers(d, recent):
    """In front of an odd and of an even page, of either format."""
    import paper_2608_23834_amd as mk
    t, cu, q = _made(d, [1203], [40], recent)
    scales = t.gpu.fp8_scales_view()
    for window in (100, 116, 132, 148):
        kw = dict(window=window)
        p = _first_pages(t, cu, kw)[0]
        stale = t.otags[0, p - 1] == 2
        page = int(t.bt[0, p - 1])
        held = (t.gpu.tq3_view() if stale else t.gpu.fp8_view())[0, page]
        was, ws = held.clone(), scales[0, page].clone()
        held.fill_(0x7F)
        if not stale:
            scales[0, page] = float("nan")
        _near(_chunk(t, q, cu, kw), sref.chunk(t.orc, 0, ref.bf16_f64(q), cu, t.obt, t.otags, t.cur, kw))
        held.copy_(was)
        if not stale:
            scales[0, page] = ws
    assert mk.kv_pool_check_errors(t.gpu) == 0
