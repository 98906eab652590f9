"""Page bounds, page selection and attention over the selected pages, against numpy in 64
bits and the CPU oracle's reconstructed pages; then a whole run of them with the rotated
appends, as a serving loop makes it."""
import ctypes
import dataclasses

import numpy as np
import pytest

import _rope_ref as ref
import mkv_workloads as wl

pytestmark = pytest.mark.gpu
PAGE = 16


def _torch():
    import torch
    return torch


def _gpu(a):
    return _torch().from_numpy(np.ascontiguousarray(a)).cuda()


def _i16(bits):
    return _gpu(np.asarray(bits).view(np.int16))


def _w(d, hq, hkv, n_req, layers=1):
    return dataclasses.replace(wl.scaled(wl.workload(2), (16,) * n_req, layers), head_dim=d, n_q_heads=hq, n_kv_heads=hkv)


def _twin(w, lens, layers=1, recent=64, headroom=0):
    from _harness import Twin
    return Twin(w, n_layers=layers, lens=lens, recent=recent, headroom=headroom)


def _values(b):
    """The bounds' (largest, smallest) as float64, and the scales."""
    return ref.e4m3(b.codes.cpu().numpy()), b.scales.cpu().numpy()


# ---------------------------------------------------------------- bounds

@pytest.mark.parametrize("d,hq,hkv", [(256, 24, 4), (128, 8, 1), (128, 32, 8)])
def test_bounds_match(d, hq, hkv):
    import paper_2608_23834_amd as mk
    t = _twin(_w(d, hq, hkv, 5, 2), [1, 16, 17, 700, 2003], 2)
    t.fill()
    b = mk.PageBounds(t.gpu, t.n_req, t.max_pages)
    zero = _gpu(np.zeros(5, np.int32))
    for layer in (0, -1):
        mk.kv_page_bounds_update(t.gpu, layer, t.bt, t.tags, zero, _gpu(np.array(t.cur, np.int32)), b)
        want, sc = ref.bounds(t.orc.fp8, t.orc.fp8_scale, t.obt, t.cur, d)
        if layer == 0:
            want[1:], sc[1:] = 0, 0
        got, gs = _values(b)
        assert np.array_equal(got, want) and np.array_equal(gs, sc)
    # only the pages from seq_lens_from on are written
    b.codes.fill_(0x11)
    b.scales.fill_(5.0)
    frm = np.array([0, 16, 16, 690, 1999], np.int32)
    mk.kv_page_bounds_update(t.gpu, -1, t.bt, t.tags, _gpu(frm), _gpu(np.array(t.cur, np.int32)), b)
    got, gs = _values(b)
    for r in range(5):
        a, e = frm[r] // PAGE, (t.cur[r] + PAGE - 1) // PAGE
        assert np.array_equal(got[:, r, :, a:e], want[:, r, :, a:e]) and np.array_equal(gs[:, r, :, a:e], sc[:, r, :, a:e])
        for rest in (slice(0, a), slice(e, None)):
            assert np.all(b.codes.cpu().numpy()[:, r, :, rest] == 0x11) and np.all(gs[:, r, :, rest] == 5.0)
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_bounds_of_many_requests():
    """More requests than one launch takes, most of them a page or none."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 40, 2100)]
    lens[1023], lens[1024], lens[2099] = 300, 0, 129
    t = _twin(_w(128, 8, 1, len(lens)), lens)
    t.fill()
    b = mk.PageBounds(t.gpu, t.n_req, t.max_pages)
    mk.kv_page_bounds_update(t.gpu, 0, t.bt, t.tags, _gpu(np.zeros(t.n_req, np.int32)), _gpu(np.array(t.cur, np.int32)), b)
    want, sc = ref.bounds(t.orc.fp8, t.orc.fp8_scale, t.obt, t.cur, 128)
    got, gs = _values(b)
    assert np.array_equal(got, want) and np.array_equal(gs, sc)
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_bounds_of_wrong_pages():
    import paper_2608_23834_amd as mk
    t = _twin(_w(128, 8, 2, 4), [400, 400, 400, 400], recent=64)
    t.fill()
    t.migrate()  # pages outside the window and not anchors are Stale now
    b = mk.PageBounds(t.gpu, 4, t.max_pages)
    b.codes.fill_(0x22)
    lens = np.array([400, -1, 401 * 16, 0], np.int32)
    mk.kv_page_bounds_update(t.gpu, 0, t.bt, t.tags, _gpu(np.zeros(4, np.int32)), _gpu(lens), b)
    assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["BAD_TAG"] | mk.DEVERR["RANGE"]
    codes = b.codes.cpu().numpy()
    assert np.all(codes[:, 1:] == 0x22)
    stale = t.otags[0] == 2
    assert stale.any() and np.all(codes[0, 0][:, stale] == 0x22) and not np.any(np.all(codes[0, 0][:, ~stale] == 0x22, axis=(2, 3)))
    bt = t.bt.clone()
    bt[0, t.max_pages - 1] = 1 << 20  # an id outside the pool
    mk.kv_page_bounds_update(t.gpu, 0, bt, t.tags, _gpu(np.array([395] * 4, np.int32)), _gpu(np.array([400, 0, 0, 0], np.int32)), b)
    assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]


# ---------------------------------------------------------------- selection

def _select(pool, b, q, lens, n_select, n_first, n_last, fill=7):
    import paper_2608_23834_amd as mk
    torch = _torch()
    pages = torch.full((b.n_req, pool.n_kv_heads, n_select), fill, dtype=torch.int32, device="cuda")
    counts = torch.full((b.n_req, pool.n_kv_heads), fill, dtype=torch.int32, device="cuda")
    ws = mk.select_workspace(pool, b.n_req, b.max_pages)
    ws.fill_(0xA5)
    mk.paged_attn_select_pages(pool, 0, _i16(q), _gpu(np.asarray(lens, np.int32)), b, n_first, n_last, pages, counts, ws)
    torch.cuda.synchronize()
    return pages.cpu().numpy(), counts.cpu().numpy()


def _random_bounds(rng, pool, n_req, mp):
    import paper_2608_23834_amd as mk
    b = mk.PageBounds(pool, n_req, mp)
    a = rng.integers(0, 256, b.codes.shape).astype(np.uint8)
    a[(a & 127) == 127] = 0
    v = ref.e4m3(a)
    a = np.where((v[..., :1, :] >= v[..., 1:, :]), a, a[..., ::-1, :])  # larger one first
    b.codes.copy_(_gpu(a))
    b.scales.copy_(_gpu(rng.uniform(0.001, 0.01, b.scales.shape).astype(np.float32)))
    return b


@pytest.mark.parametrize("d,hq,hkv,lens,mp,k,first,last", [
    (256, 24, 4, [1, 16, 33, 700, 2047, 2048], 128, 32, 2, 4),
    (128, 8, 1, [4000, 16384], 1024, 128, 4, 16),
    (128, 32, 2, [5000, 77, 60000], 4096, 1, 0, 0),
    (256, 16, 2, [3000], 200, 5, 0, 5),       # the last pages alone
    (256, 16, 2, [3000, 100], 200, 7, 7, 0),  # the first pages alone
    (128, 16, 4, [20000], 1250, 1249, 3, 64),  # all but one
    (256, 12, 4, [2000, 1999], 125, 300, 4, 4),  # more than there are
    (128, 16, 4, [60000], 4000, 1500, 1, 1),
])
def test_selection(d, hq, hkv, lens, mp, k, first, last):
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(d + k + mp)
    pool = mk.Pool(1, hq, hkv, d, 1, 1, 64, np.ones(d, np.int8))
    b = _random_bounds(rng, pool, len(lens), mp)
    q = wl.bf16_round(rng.standard_normal((len(lens), hq, d)).astype(np.float32))
    vals, sc = _values(b)
    want, cnt = ref.select(ref.scores(q, vals[0], sc[0]), lens, k, first, last)
    got, gc = _select(pool, b, q, lens, k, first, last)
    assert np.array_equal(gc, cnt) and np.array_equal(got, want)
    assert mk.kv_pool_check_errors(pool) == 0


def test_selection_near_and_equal_scores():
    """Scores that fp32 cannot tell apart, equal ones, -0 and 0, NaN and infinities."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(6)
    pool = mk.Pool(1, 8, 2, 128, 1, 1, 64, np.ones(128, np.int8))
    n, mp = 3, 600
    b = _random_bounds(rng, pool, n, mp)
    codes = b.codes.cpu().numpy()
    codes[:] = codes[:, :, :, :1]       # every page alike,
    codes[0, 0, :, :, :, 0] = rng.integers(0, 8, codes[0, 0, :, :, :, 0].shape)  # but for 2^-9's in a small channel
    codes[0, 0, :, :, 1, 0] = 0
    b.codes.copy_(_gpu(codes))
    b.scales.fill_(0.01)
    q = wl.bf16_round(rng.standard_normal((n, 8, 128)).astype(np.float32))
    q[0, :, 0] = 0x3280  # 2^-26: the pages' scores differ by 2^-35 steps
    q[1] = 0             # all scores 0
    q[2, 0, 3], q[2, 5, 4] = 0x7F80, 0x7FC0  # infinity for one KV head, NaN for the other
    vals, sc = _values(b)
    s = ref.scores(q, vals[0], sc[0])
    for k, first, last in ((64, 0, 0), (100, 3, 5), (599, 0, 1)):
        want, cnt = ref.select(s, [mp * PAGE] * n, k, first, last)
        got, gc = _select(pool, b, q, [mp * PAGE] * n, k, first, last)
        assert np.array_equal(gc, cnt)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])


def test_selection_scales_that_overflow():
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(16)
    pool = mk.Pool(1, 6, 1, 128, 1, 1, 64, np.ones(128, np.int8))
    b = _random_bounds(rng, pool, 1, 300)
    sc = b.scales.cpu().numpy()
    sc[..., 5], sc[..., 17], sc[..., 30], sc[..., 31] = np.inf, 0.0, 3e38, 1e-40
    b.scales.copy_(_gpu(sc))
    q = wl.bf16_round((1e20 * rng.standard_normal((1, 6, 128))).astype(np.float32))
    vals, sc = _values(b)
    want, _ = ref.select(ref.scores(q, vals[0], sc[0]), [4800], 20, 0, 0)
    got, _ = _select(pool, b, q, [4800], 20, 0, 0)
    assert np.array_equal(got, want) and 5 in got[0, 0] and 30 in got[0, 0]


@pytest.mark.parametrize("qe,se", [(-60, -75), (-126, -3), (-133, -10), (-20, -126), (-140, -126), (-100, 20)])
def test_selection_of_tiny_scores(qe, se):
    """Queries and scales whose products fall below fp32's numbers: the choice is fp64's."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(8)
    pool = mk.Pool(1, 16, 2, 256, 1, 1, 64, np.ones(256, np.int8))
    b = _random_bounds(rng, pool, 2, 500)
    b.scales.copy_(_gpu((2.0 ** se * rng.uniform(1, 2, b.scales.shape)).astype(np.float32)))
    q = wl.bf16_round((2.0 ** qe * rng.standard_normal((2, 16, 256))).astype(np.float32))
    vals, sc = _values(b)
    want, cnt = ref.select(ref.scores(q, vals[0], sc[0]), [8000, 7991], 40, 2, 3)
    got, gc = _select(pool, b, q, [8000, 7991], 40, 2, 3)
    assert np.array_equal(gc, cnt) and np.array_equal(got, want)


def test_selection_zero_query_and_nan_keys():
    """0 * NaN is NaN: pages whose extremes hold one come last even where all other scores are 0."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(9)
    pool = mk.Pool(1, 8, 2, 128, 1, 1, 64, np.ones(128, np.int8))
    b = _random_bounds(rng, pool, 2, 300)
    codes = b.codes.cpu().numpy()
    codes[0, :, :, [3, 17, 40], 0, 5] = 0x7F
    b.codes.copy_(_gpu(codes))
    vals, sc = _values(b)
    q = wl.bf16_round(rng.standard_normal((2, 8, 128)).astype(np.float32))
    q[0] = 0
    want, _ = ref.select(ref.scores(q, vals[0], sc[0]), [4800, 4800], 30, 0, 1)
    got, _ = _select(pool, b, q, [4800, 4800], 30, 0, 1)
    assert np.array_equal(got, want) and not np.isin(got[0], [3, 17]).any()


def test_selection_bad_lengths_and_refusals():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(7)
    pool = mk.Pool(1, 8, 2, 128, 1, 1, 64, np.ones(128, np.int8))
    b = _random_bounds(rng, pool, 3, 20)
    q = wl.bf16_round(rng.standard_normal((3, 8, 128)).astype(np.float32))
    got, cnt = _select(pool, b, q, [0, 321, 320], 4, 1, 1)
    assert mk.kv_pool_check_errors(pool, clear=True) == mk.DEVERR["RANGE"]
    assert np.all(cnt[:2] == 0) and np.all(got[:2] == -1) and np.all(cnt[2] == 4)
    ws = mk.select_workspace(pool, 3, 20)
    pages, counts = torch.zeros((3, 2, 4), dtype=torch.int32, device="cuda"), torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    L = mk.lib()
    ok = dict(q=_i16(q), seq=_gpu(np.array([1, 2, 3], np.int32)), mp=20, k=4, first=1, last=1, ws=ws, wsb=ws.numel(), layer=0, cb=b.codes.numel())

    def call(**kw):
        a = {**ok, **kw}
        p = lambda x: ctypes.c_void_p(x.data_ptr()) if hasattr(x, "data_ptr") else x  # noqa: E731
        return L.paged_attn_select_pages(pool.handle, a["layer"], 3, p(a["q"]), p(a["seq"]), a["mp"], p(b.codes), a["cb"],
                                         p(b.scales), 4 * b.scales.numel(), a["k"], a["first"], a["last"], p(pages), p(counts),
                                         p(a["ws"]), a["wsb"], None)
    assert call() == 0
    assert call(q=None) == 1 and call(k=0) == 1 and call(first=-1) == 1 and call(first=3, last=2) == 1
    assert call(layer=1) == 4 and call(mp=0) == 1 and call(k=1 << 19) == 4
    assert call(wsb=ws.numel() - 1) == 3 and call(cb=b.codes.numel() - 1) == 3 and call(mp=21) == 3
    assert call(ws=ctypes.c_void_p(ws.data_ptr() + 8)) == 1
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        mk.paged_attn_select_pages(pool, 0, _i16(q), ok["seq"], b, 1, 1, pages[:2], counts, ws)


# ---------------------------------------------------------------- attention

def _sparse(t, q, pages, counts, lens=None, layer=0, bt=None, tags=None, ws=None, stream=None):
    import paper_2608_23834_amd as mk
    torch = _torch()
    w = t.w
    out = torch.full((t.n_req, w.n_q_heads, w.head_dim), float("nan"), device="cuda")
    lse = torch.full((t.n_req, w.n_q_heads), float("nan"), device="cuda")
    if ws is None:
        ws = mk.workspace(t.gpu, t.n_req, pages.shape[2])
        ws.view(torch.float32)[: ws.numel() // 4].fill_(float("nan"))
    mk.paged_attn_decode_sparse(t.gpu, layer, _i16(q), t.bt if bt is None else bt, t.tags if tags is None else tags,
                                _gpu(np.asarray(t.cur if lens is None else lens, np.int32)), _gpu(pages.astype(np.int32)),
                                _gpu(counts.astype(np.int32)), out, lse, ws, stream=stream)
    torch.cuda.synchronize()
    return out.cpu().numpy(), lse.cpu().numpy()


def _close(got, want):
    (go, gl), (o, l, tol) = got, want
    assert np.all(np.abs(go - o) <= tol[..., None])
    fin = np.isfinite(l)
    assert np.array_equal(fin, np.isfinite(gl)) and np.all(gl[~fin] == -np.inf)
    assert np.all(np.abs(gl[fin] - l[fin]) <= tol[fin] + 2.0 ** -22 * np.abs(l[fin]))


def _choose(rng, lens, H, k, some=1.0):
    pages, counts = np.full((len(lens), H, k), -1, np.int64), np.zeros((len(lens), H), np.int64)
    for r, n in enumerate(lens):
        npg = (n + PAGE - 1) // PAGE
        for h in range(H):
            c = min(npg, int(rng.integers(0, k + 1)) if some < 1 else k)
            pages[r, h, :c] = np.sort(rng.choice(npg, c, replace=False))
            counts[r, h] = c
    return pages, counts


@pytest.mark.parametrize("d,hq,hkv", [(256, 24, 4), (256, 16, 2), (256, 32, 2), (128, 32, 8), (128, 24, 4), (128, 16, 1)])
def test_sparse_attention(d, hq, hkv):
    import paper_2608_23834_amd as mk
    w = _w(d, hq, hkv, 5)
    t = _twin(w, [2500, 333, 64, 17, 1])
    t.fill()
    t.migrate()
    t.check_tables()
    rng = np.random.default_rng(d + hq)
    q = wl.bf16_round(rng.standard_normal((5, hq, d)).astype(np.float32))
    for k, some in ((20, 1.0), (40, 0.5), (1, 1.0), (157, 1.0), (400, 1.0)):
        pages, counts = _choose(rng, t.cur, hkv, k, some)
        want = ref.attend(t.orc, 0, q, t.obt, t.otags, t.cur, pages, counts)
        got = _sparse(t, q, pages, counts)
        print(f"  d={d} {hq}/{hkv} k={k}: max|dO| {np.abs(got[0] - want[0]).max():.2e}", flush=True)
        _close(got, want)
        assert mk.kv_pool_check_errors(t.gpu) == 0
    # every page listed: the outputs of the dense decode, up to its own query precision
    res = t.decode(0, q=q)
    assert np.abs(got[0] - res["out"]).max() <= 1e-3


def test_sparse_deterministic_and_timed():
    import paper_2608_23834_amd as mk
    w = _w(256, 24, 4, 2)
    t = _twin(w, [4000, 3000])
    t.fill()
    t.migrate()
    rng = np.random.default_rng(1)
    q = wl.bf16_round(rng.standard_normal((2, 24, 256)).astype(np.float32))
    pages, counts = _choose(rng, t.cur, 4, 100)
    mk.paged_attn_set_deterministic(t.gpu, True)
    a = _sparse(t, q, pages, counts)
    mk.paged_attn_set_timing(t.gpu, True)
    b = _sparse(t, q, pages, counts)
    scan, merge = mk.paged_attn_last_times(t.gpu)
    assert scan > 0 and merge > 0
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_sparse_bad_lists():
    """Entries out of order, twice, past the end, unmapped or out of range are left out and set the
    error word; a count out of range gives zeros; none of it touches other rows."""
    import paper_2608_23834_amd as mk
    w = _w(128, 16, 2, 3)
    t = _twin(w, [500, 400, 300])
    t.fill()
    t.migrate()
    rng = np.random.default_rng(2)
    q = wl.bf16_round(rng.standard_normal((3, 16, 128)).astype(np.float32))
    good, cnt = _choose(rng, t.cur, 2, 8)

    def run(r, h, entries, count=None, err="RANGE", bt=None, tags=None):
        pages, counts = good.copy(), cnt.copy()
        pages[r, h] = -1
        pages[r, h, :len(entries)] = entries
        counts[r, h] = len(entries) if count is None else count
        keep, last = [], -1
        for e in entries:  # what stays in: above the entry before it, below the end
            if e > last and 0 <= e < (t.cur[r] + PAGE - 1) // PAGE:
                keep.append(e)
            last = e
        if count is not None:
            keep = []
        kp, kc = good.copy(), cnt.copy()
        kp[r, h], kc[r, h] = -1, len(keep)
        kp[r, h, :len(keep)] = keep
        got = _sparse(t, q, pages, counts, bt=bt, tags=tags)
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR[err]
        if bt is None and tags is None:
            _close(got, ref.attend(t.orc, 0, q, t.obt, t.otags, t.cur, kp, kc))
        return got
    run(0, 1, [3, 3, 5])
    run(0, 0, [9, 3, 5])
    run(1, 1, [-1, 2, 4])
    run(2, 0, [2, 19, 4000])
    run(2, 1, [2 ** 31 - 1])
    run(1, 0, [1, 2], count=-1)
    run(1, 0, [1, 2], count=9)
    tags = t.tags.clone()
    tags[0, 3] = 0xFF
    run(0, 0, [1, 3, 4], err="BAD_TAG", tags=tags)
    bt = t.bt.clone()
    bt[0, 3] = 1 << 20
    run(0, 0, [1, 3, 4], bt=bt)
    got = _sparse(t, q, good, cnt, lens=[0, 400, 300])
    assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]
    assert not got[0][0].any()
    none = np.zeros_like(cnt)
    got = _sparse(t, q, good, none)
    assert not got[0].any() and np.all(got[1] == -np.inf) and mk.kv_pool_check_errors(t.gpu) == 0


def test_sparse_refusals():
    import paper_2608_23834_amd as mk
    torch = _torch()
    t = _twin(_w(128, 8, 2, 1), [64])
    t.fill()
    L = mk.lib()
    ws = mk.workspace(t.gpu, 1, 4)
    bufs = dict(q=torch.zeros(8 * 128, dtype=torch.int16, device="cuda"), out=torch.zeros(8 * 128, device="cuda"),
                pages=torch.zeros(8, dtype=torch.int32, device="cuda"), counts=torch.zeros(2, dtype=torch.int32, device="cuda"),
                seq=_gpu(np.array([64], np.int32)), ws=ws)

    def call(layer=0, n=1, k=4, mp=t.max_pages, wsb=ws.numel(), **kw):
        a = {**bufs, **kw}
        p = lambda x: ctypes.c_void_p(x.data_ptr()) if hasattr(x, "data_ptr") else x  # noqa: E731
        return L.paged_attn_decode_sparse(t.gpu.handle, layer, n, p(a["q"]), p(t.bt), p(t.tags), mp, p(a["seq"]), k,
                                          p(a["pages"]), p(a["counts"]), p(a["out"]), None, p(a["ws"]), wsb, None)
    assert call() == 0
    for name in bufs:
        assert call(**{name: None}) == 1, name
    assert call(k=0) == 1 and call(n=0) == 1 and call(mp=0) == 1
    assert call(layer=1) == 4 and call(layer=-1) == 4 and call(k=(1 << 18) + 1) == 4 and call(n=65536) == 4
    assert call(wsb=16) == 3
    assert call(q=ctypes.c_void_p(bufs["q"].data_ptr() + 2)) == 1
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        mk.paged_attn_decode_sparse(t.gpu, 0, bufs["q"], t.bt, t.tags, bufs["seq"], bufs["pages"].view(1, 1, 8),
                                    bufs["counts"].view(1, 2), bufs["out"], None, ws)


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("d,hq,hkv,captured", [(256, 24, 4, False), (128, 32, 8, False), (256, 16, 2, True)])
def test_serving_run(d, hq, hkv, captured):
    """A prompt appended rotated, its chunk attention on rotated queries, its bounds, Retier; then steps
    of rotated append, bounds of the new token's page, selection and sparse attention, on a stream of
    their own (captured: each step replays a graph, eager work between), all against the oracle."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    w = _w(d, hq, hkv, 3)
    lens = [900, 400, 37]
    rng = np.random.default_rng(d)
    t = _twin(w, lens, headroom=32)
    freq = 1e6 ** (-np.arange(d // 4) / (d // 4))
    axis = (np.arange(d // 4) % 3).astype(np.uint8)
    rope = mk.Rope(d, freq, axis, 3)
    n = sum(lens)
    pos = np.concatenate([np.stack([np.arange(x), np.arange(x) // 7, np.arange(x) % 7]) for x in lens], 1).astype(np.int32)
    rows = wl.bf16_round(rng.standard_normal((n, hq + 2 * hkv, d)).astype(np.float32))  # packed q, k, v
    q, K, V = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    cu = np.r_[0, np.cumsum(lens)].astype(np.int32)
    g, zero, cug, pg = _i16(rows), _gpu(np.zeros(3, np.int32)), _gpu(cu), _gpu(pos)
    mk.kv_append_fp8_rope(t.gpu, rope, 0, t.bt, t.tags, zero, cug, pg, g[:, hq:hq + hkv], g[:, hq + hkv:])
    qr = torch.zeros((n, hq, d), dtype=torch.int16, device="cuda")
    mk.kv_rope_apply(rope, g[:, :hq], pg, qr)
    out = torch.zeros((n, hq, d), device="cuda")
    after = _gpu(np.array(lens, np.int32))
    mk.paged_attn_chunk(t.gpu, 0, qr, cug, t.bt, t.tags, after, out, mk.workspace(t.gpu, 3, t.max_pages, n))
    b = mk.PageBounds(t.gpu, 3, t.max_pages)
    mk.kv_page_bounds_update(t.gpu, 0, t.bt, t.tags, zero, after, b)
    assert t.orc.append(0, t.obt, t.otags, np.zeros(3, np.int32), cu, ref.rotate(K, pos, freq, axis, False)[None], V[None]) == 0
    t.cur = list(lens)
    t.check_tables()
    t.check_pages()
    qo = ref.rotate(q, pos, freq, axis, False)
    assert ref.same_bits(qr.cpu().numpy(), qo)
    co = t.orc.chunk(0, qo, cu, t.obt, t.otags, np.array(lens, np.int32), 97)
    ok = ~np.isnan(co)
    assert ok.any() and np.abs(out.cpu().numpy()[ok] - co[ok]).max() <= 1e-3
    vals, scl = ref.bounds(t.orc.fp8, t.orc.fp8_scale, t.obt, t.cur, d)
    t.migrate()
    k = 12
    pages, counts = torch.zeros((3, hkv, k), dtype=torch.int32, device="cuda"), torch.zeros((3, hkv), dtype=torch.int32, device="cuda")
    wsel, watt = mk.select_workspace(t.gpu, 3, t.max_pages), mk.workspace(t.gpu, 3, k)
    rowb = torch.zeros((3, hq + 2 * hkv, d), dtype=torch.int16, device="cuda")
    posb, sb, sa = torch.zeros((3, 3), dtype=torch.int32, device="cuda"), zero.clone(), zero.clone()
    one = _gpu(np.arange(4, dtype=np.int32))
    qb = torch.zeros((3, hq, d), dtype=torch.int16, device="cuda")
    so, sl = torch.zeros((3, hq, d), device="cuda"), torch.zeros((3, hq), device="cuda")
    side = torch.cuda.Stream()

    def step(stream=None):
        mk.kv_append_fp8_rope(t.gpu, rope, 0, t.bt, t.tags, sb, one, posb, rowb[:, hq:hq + hkv], rowb[:, hq + hkv:], stream=stream)
        mk.kv_rope_apply(rope, rowb[:, :hq], posb, qb, stream=stream)
        mk.kv_page_bounds_update(t.gpu, 0, t.bt, t.tags, sb, sa, b, stream=stream)
        mk.paged_attn_select_pages(t.gpu, 0, qb, sa, b, 1, 2, pages, counts, wsel, stream=stream)
        mk.paged_attn_decode_sparse(t.gpu, 0, qb, t.bt, t.tags, sa, pages, counts, so, sl, watt, stream=stream)
    graph = None
    for i in range(6):
        r = wl.bf16_round(rng.standard_normal((3, hq + 2 * hkv, d)).astype(np.float32))
        ps = rng.integers(0, 3000, (3, 3)).astype(np.int32)
        before = np.array(t.cur, np.int32)
        rowb.copy_(_i16(r))
        posb.copy_(_gpu(ps))
        sb.copy_(_gpu(before))
        sa.copy_(_gpu(before + 1))
        torch.cuda.synchronize()
        if captured and i == 1:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        if graph is not None:
            graph.replay()
        else:
            side.wait_stream(torch.cuda.current_stream())
            step(stream=side)
        torch.cuda.synchronize()
        Kr, qo = ref.rotate(r[:, hq:hq + hkv], ps, freq, axis, False), ref.rotate(r[:, :hq], ps, freq, axis, False)
        assert t.orc.append(0, t.obt, t.otags, before, np.arange(4, dtype=np.int32), Kr[None], r[None, :, hq + hkv:]) == 0
        t.cur = [c + 1 for c in t.cur]
        t.check_tables()
        t.check_pages()
        for rr, c in enumerate(t.cur):  # the new token's page
            p = (c - 1) // PAGE
            kk = ref.e4m3(t.orc.fp8[:, t.obt[rr, p], :, : PAGE * d]).reshape(1, hkv, PAGE, d)[:, :, : c - p * PAGE]
            vals[:, rr, :, p, 0], vals[:, rr, :, p, 1] = kk.max(2), kk.min(2)
            scl[:, rr, :, p] = t.orc.fp8_scale[:, t.obt[rr, p], :, 0]
        gv, gs = _values(b)
        assert np.array_equal(gv, vals) and np.array_equal(gs, scl)
        wp, wc = ref.select(ref.scores(qo, vals[0], scl[0]), t.cur, k, 1, 2)
        assert np.array_equal(pages.cpu().numpy(), wp) and np.array_equal(counts.cpu().numpy(), wc), i
        _close((so.cpu().numpy(), sl.cpu().numpy()), ref.attend(t.orc, 0, qo, t.obt, t.otags, t.cur, wp, wc))
        if i == 3:
            t.migrate()
            t.check_tables()
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_far_pages():
    """Page ids whose bytes lie past 2^32: the same answers, bit for bit, as from a small pool."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    d, hq, hkv, lens = 256, 24, 4, [900, 33, 17]
    rng = np.random.default_rng(12)
    n = sum(lens)
    rows, new = (_i16(wl.bf16_round(rng.standard_normal((c, hq + 2 * hkv, d)).astype(np.float32))) for c in (n, 3))
    q = _i16(wl.bf16_round(rng.standard_normal((3, hq, d)).astype(np.float32)))
    rope = mk.Rope(d, 1e6 ** (-np.arange(32) / 32))
    cu, zero, one = _gpu(np.r_[0, np.cumsum(lens)].astype(np.int32)), _gpu(np.zeros(3, np.int32)), _gpu(np.arange(4, dtype=np.int32))
    held, after = _gpu(np.array(lens, np.int32)), _gpu(np.array(lens, np.int32) + 1)

    def answers(n8, order):
        pool = mk.Pool(1, hq, hkv, d, n8, 1, 4096, np.ones(d, np.int8), order)
        mk.paged_attn_set_deterministic(pool, True)
        bt = torch.full((3, 60), -1, dtype=torch.int32, device="cuda")
        tags = torch.full((3, 60), 0xFF, dtype=torch.uint8, device="cuda")
        mk.kv_append_fp8_rope(pool, rope, 0, bt, tags, zero, cu, None, rows[:, hq:hq + hkv], rows[:, hq + hkv:])
        mk.kv_append_fp8_rope(pool, rope, 0, bt, tags, held, one, None, new[:, hq:hq + hkv], new[:, hq + hkv:])
        b = mk.PageBounds(pool, 3, 60)
        mk.kv_page_bounds_update(pool, 0, bt, tags, zero, after, b)
        pages, counts = torch.zeros((3, hkv, 20), dtype=torch.int32, device="cuda"), torch.zeros((3, hkv), dtype=torch.int32, device="cuda")
        mk.paged_attn_select_pages(pool, 0, q, after, b, 1, 2, pages, counts, mk.select_workspace(pool, 3, 60))
        out, lse = torch.zeros((3, hq, d), device="cuda"), torch.zeros((3, hq), device="cuda")
        mk.paged_attn_decode_sparse(pool, 0, q, bt, tags, after, pages, counts, out, lse, mk.workspace(pool, 3, 20))
        step, slse = torch.zeros((3, hq, d), device="cuda"), torch.zeros((3, hq), device="cuda")
        mk.paged_attn_decode_append_rope(pool, rope, 0, q, new[:, hq:hq + hkv].contiguous(), new[:, hq + hkv:].contiguous(),
                                         None, bt, tags, after, step, slse, mk.workspace(pool, 3, 60))
        torch.cuda.synchronize()
        assert mk.kv_pool_check_errors(pool) == 0
        return bt.max().item(), [x.clone() for x in (b.codes, b.scales, pages, counts, out, lse, step, slse)]
    n8 = 140000  # 32 KB a page
    small = answers(80, None)[1]
    tops = []
    for order in (np.arange(n8, dtype=np.int32), np.arange(n8, dtype=np.int32)[::-1]):
        top, far = answers(n8, order)
        tops.append(top)
        for k, (x, y) in enumerate(zip(small, far)):
            assert torch.equal(x, y), k
    assert max(tops) * 32768 > 2 ** 32


def test_far_bounds():
    """Bounds of more than 2^32 bytes, the request in question at their end and its sequence the
    table's whole width."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    n_req, mp, k = 130, 65536, 100
    rng = np.random.default_rng(14)
    pool = mk.Pool(1, 4, 2, 128, 64, 1, 64, np.ones(128, np.int8))
    b = mk.PageBounds(pool, n_req, mp)
    assert b.codes.numel() > 2 ** 32
    some = _random_bounds(rng, pool, 1, 400)
    at = np.sort(rng.choice(mp, 400, replace=False))
    for h in range(2):
        b.codes[0, -1, h, torch.from_numpy(at).cuda()] = some.codes[0, 0, h]
        b.scales[0, -1, h, torch.from_numpy(at).cuda()] = some.scales[0, 0, h]
    q = wl.bf16_round(rng.standard_normal((n_req, 4, 128)).astype(np.float32))
    lens = np.full(n_req, 16, np.int32)
    lens[-1] = mp * PAGE
    got, cnt = _select(pool, b, q, lens, k, 3, 5)
    vals, sc = _values(some)
    score = np.zeros((1, 2, mp))
    score[:, :, at] = ref.scores(q[-1:], vals[0], sc[0])
    want, _ = ref.select(score, [mp * PAGE], k, 3, 5)
    assert np.array_equal(got[-1], want[0]) and np.all(cnt[-1] == k)
    assert np.all(cnt[:-1] == 1) and np.all(got[:-1, :, 0] == 0) and np.all(got[:-1, :, 1:] == -1)
    # its last page, updated from a pool
    bt = torch.full((n_req, mp), -1, dtype=torch.int32, device="cuda")
    tags = torch.full((n_req, mp), 0xFF, dtype=torch.uint8, device="cuda")
    bt[-1, -1], tags[-1, -1] = 63, 0
    pool.fp8_view()[0, 63] = 0x22
    pool.fp8_scales_view()[0, 63] = 0.5
    frm, seq = np.zeros(n_req, np.int32), np.zeros(n_req, np.int32)
    frm[-1], seq[-1] = mp * PAGE - 1, mp * PAGE
    mk.kv_page_bounds_update(pool, 0, bt, tags, _gpu(frm), _gpu(seq), b)
    torch.cuda.synchronize()
    assert mk.kv_pool_check_errors(pool) == 0
    assert torch.all(b.codes[0, -1, :, -1] == 0x22) and torch.all(b.scales[0, -1, :, -1] == 0.5)
    assert not b.codes[0, :-1].any()


def test_two_streams_and_two_graphs():
    """Calls on two streams at once, each with its buffers, and two graphs over one workspace replayed
    in turn: the answers of separate calls."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    w = _w(256, 24, 4, 2)
    lens = [1900, 700]
    t = _twin(w, lens)
    rng = np.random.default_rng(31)
    K, V = (wl.bf16_round(rng.standard_normal((sum(lens), 4, 256)).astype(np.float32)) for _ in range(2))
    cu, zero, seq = (_gpu(np.array(x, np.int32)) for x in ([0, 1900, 2600], [0, 0], lens))
    mk.kv_append_fp8(t.gpu, 0, t.bt, t.tags, zero, cu, _i16(K), _i16(V))
    b = mk.PageBounds(t.gpu, 2, t.max_pages)
    mk.kv_page_bounds_update(t.gpu, 0, t.bt, t.tags, zero, seq, b)
    mk.paged_attn_set_deterministic(t.gpu, True)
    q = [_i16(wl.bf16_round(rng.standard_normal((2, 24, 256)).astype(np.float32))) for _ in range(2)]

    def buffers():
        return (torch.zeros((2, 4, 16), dtype=torch.int32, device="cuda"), torch.zeros((2, 4), dtype=torch.int32, device="cuda"),
                torch.zeros((2, 24, 256), device="cuda"), torch.zeros((2, 24), device="cuda"))

    def spaces():
        return mk.select_workspace(t.gpu, 2, t.max_pages), mk.workspace(t.gpu, 2, 16)

    def call(x, to, ws, stream=None):
        mk.paged_attn_select_pages(t.gpu, 0, x, seq, b, 1, 3, to[0], to[1], ws[0], stream=stream)
        mk.paged_attn_decode_sparse(t.gpu, 0, x, t.bt, t.tags, seq, to[0], to[1], to[2], to[3], ws[1], stream=stream)
    want, got = [buffers() for _ in q], [buffers() for _ in q]
    for x, to in zip(q, want):
        call(x, to, spaces())
    assert not torch.equal(want[0][2], want[1][2])
    own, side = [spaces() for _ in q], [torch.cuda.Stream() for _ in q]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            call(q[i], got[i], own[i], stream=side[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, y) for x, y in zip(want[i], got[i])), i
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side[0]):
            call(q[i], got[i], own[0])
        graphs.append(g)
    for _ in range(3):
        for to in got:
            for x in to:
                x.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(x, y) for x, y in zip(want[i], got[i])), i
    assert mk.kv_pool_check_errors(t.gpu) == 0
