"""Decode attention with shaped scores, alone and as a whole step (norms, rotation, append), against
64-bit numpy over the CPU oracle's reconstructed pages."""
import dataclasses

import numpy as np
import pytest

import _norm_ref as nref
import _rope_ref as ref
import _shape_ref as sref
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


def _i32(v):
    return _gpu(np.asarray(v, np.int32))


def _bits(rng, *shape):
    return wl.bf16_round(rng.standard_normal(shape).astype(np.float32))


def _w(d, hq, hkv, n_req, layers=1):
    return dataclasses.replace(wl.scaled(wl.workload(2), (16,) * n_req, layers), head_dim=d, n_q_heads=hq, n_kv_heads=hkv)


def _twin(w, lens, layers=1, recent=64, headroom=0):
    from _harness import Twin
    t = Twin(w, n_layers=layers, lens=lens, recent=recent, headroom=headroom)
    t.fill()
    t.migrate()
    return t


def _shaping(kw):
    import paper_2608_23834_amd as mk
    kw = dict(kw)
    for n in ("slopes", "sinks"):
        if kw.get(n) is not None:
            kw[n] = _gpu(np.asarray(kw[n], np.float32))
    for n in ("first_keys", "prefix_lens"):
        if kw.get(n) is not None:
            kw[n] = _i32(kw[n])
    return mk.Shaping(**kw)


def _slopes(hq):
    return (2.0 ** (-8.0 * np.arange(1, hq + 1) / hq)).astype(np.float32)


def _near(out, lse, want):
    o, l, to, tl = want
    err = np.abs(out - o).max(2)
    assert np.all(err <= to), (np.argwhere(err > to)[:4], (err / np.maximum(to, 1e-30)).max())
    both = np.isfinite(l) & np.isfinite(lse)
    same = (lse == l) | (both & (np.abs(np.where(both, lse, 0.0) - np.where(both, l, 0.0)) <= tl))
    assert same.all(), (np.argwhere(~same)[:4], lse[~same][:4], l[~same][:4])


def _decode(t, q, kw, lens=None, bt=None, tags=None, ws=None, out=None, lse=None):
    import paper_2608_23834_amd as mk
    torch = _torch()
    n_req = t.n_req
    out = torch.full((n_req, t.w.n_q_heads, t.w.head_dim), float("nan"), device="cuda")
    lse = torch.full((n_req, t.w.n_q_heads), float("nan"), device="cuda")
    ws = mk.workspace(t.gpu, n_req, t.max_pages) if ws is None else ws
    ws.fill_(0xFF)
    mk.paged_attn_decode_shaped(t.gpu, _shaping(kw), 0, _i16(q), t.bt if bt is None else bt, t.tags if tags is None else tags,
                                _i32(t.cur if lens is None else lens), out, lse, ws)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)


LENS = [1, 16, 17, 700, 2003, 333]


def _kinds(hq, n):
    sinks = np.random.default_rng(hq).standard_normal(hq).astype(np.float32)
    sinks[0] = -np.inf
    return [
        {}, dict(cap=5.0), dict(cap=1e-6), dict(cap=50.0, scale=0.3), dict(slopes=_slopes(hq)), dict(sinks=sinks + 3),
        dict(window=1), dict(window=15, sinks=sinks), dict(window=16), dict(window=17, cap=2.0), dict(window=100, slopes=_slopes(hq)),
        dict(window=1024, cap=30.0, slopes=_slopes(hq), sinks=sinks, scale=0.05), dict(window=1 << 30),
        dict(first_keys=[0, 3, 17, 333, -5, 332][:n]),                      # behind the end, at it, negative
        dict(first_keys=[9, 0, 1, 700, 1999, 1 << 30][:n], sinks=sinks), dict(first_keys=[0, 0, 16, 650, 5, 100][:n], window=60),
    ]


@pytest.mark.parametrize("d,hq,hkv", [(256, 24, 4), (256, 16, 2), (256, 16, 1), (128, 8, 1), (128, 32, 8), (128, 12, 1),
                                      (128, 3, 3)])
def test_decode(d, hq, hkv):
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(d + hq)
    t = _twin(_w(d, hq, hkv, len(LENS)), LENS)
    assert (t.otags == 2).any() and (t.otags == 1).any() and (t.otags == 0).any()
    q = wl.bf16_round((3 * rng.standard_normal((len(LENS), hq, d))).astype(np.float32))
    for kw in _kinds(hq, len(LENS)):
        want = sref.decode(t.orc, 0, ref.bf16_f64(q), t.obt, t.otags, t.cur, kw)
        _near(*_decode(t, q, kw), want)
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_scores_at_the_cap_and_past_it():
    """Scores of many times the cap, and of a small fraction of it."""
    rng = np.random.default_rng(7)
    t = _twin(_w(128, 8, 1, 2), [300, 77])
    for gain in (1e-3, 1e2, 1e4):
        q = wl.bf16_round((gain * rng.standard_normal((2, 8, 128))).astype(np.float32))
        for kw in (dict(cap=20.0), dict(cap=20.0, slopes=_slopes(8))):
            _near(*_decode(t, q, kw), sref.decode(t.orc, 0, ref.bf16_f64(q), t.obt, t.otags, t.cur, kw))


def test_pages_outside_the_window_are_not_read():
    """They need not be mapped, nor lie in the pool; those inside are checked as ever."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(9)
    t = _twin(_w(256, 24, 4, 3), [700, 701, 703])
    q = _bits(rng, 3, 24, 256)
    bt, tags = t.bt.clone(), t.tags.clone()
    kw = dict(window=100)
    for r, n in enumerate(t.cur):
        bt[r, : (n - 100) // PAGE] = 1 << 28
        tags[r, : (n - 100) // PAGE] = 0xFF
    _near(*_decode(t, q, kw, bt=bt, tags=tags), sref.decode(t.orc, 0, ref.bf16_f64(q), t.obt, t.otags, t.cur, kw))
    assert mk.kv_pool_check_errors(t.gpu) == 0
    bt[1, 690 // PAGE] = -3
    out, lse = _decode(t, q, kw, bt=bt, tags=tags)
    assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"] and np.isfinite(out).all()


def test_wrong_lengths_give_zeros():
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(4)
    t = _twin(_w(128, 8, 2, 4), [100, 100, 100, 100])
    q = _bits(rng, 4, 8, 128)
    for kw in ({}, dict(window=16), dict(first_keys=[0, 50, 0, 7], cap=3.0)):
        out, lse = _decode(t, q, kw, lens=[100, 0, 16 * t.max_pages + 1, -2 ** 31])
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]
        assert np.all(out[1:] == 0) and np.all(lse[1:] == -np.inf) and np.isfinite(out[0]).all()


def test_long_tables():
    """A window far down a long table, chunks of many pages; workspaces of the table's size serve every window."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(12)
    lens = [20000, 9001]
    t = _twin(_w(128, 16, 2, 2), lens, recent=256)
    q = wl.bf16_round((2 * rng.standard_normal((2, 16, 128))).astype(np.float32))
    ws = mk.workspace(t.gpu, 2, t.max_pages)
    for kw in (dict(cap=10.0), dict(window=8000, cap=4.0), dict(window=300), dict(first_keys=[19990, 40], slopes=_slopes(16))):
        _near(*_decode(t, q, kw, ws=ws), sref.decode(t.orc, 0, ref.bf16_f64(q), t.obt, t.otags, lens, kw))
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_deterministic_and_streams():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(1)
    t = _twin(_w(256, 24, 4, 2), [4000, 2777], recent=512)
    q = _bits(rng, 2, 24, 256)
    kw = dict(cap=7.0, window=3500, slopes=_slopes(24))
    mk.paged_attn_set_deterministic(t.gpu, True)
    a = _decode(t, q, kw)
    for _ in range(3):
        b = _decode(t, q, kw)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    mk.paged_attn_set_deterministic(t.gpu, False)
    # two streams, a workspace each
    sh, bt, tags, sl = _shaping(kw), t.bt, t.tags, _i32(t.cur)
    qs = [_i16(q), _i16(_bits(rng, 2, 24, 256))]
    outs = [torch.zeros((2, 24, 256), device="cuda") for _ in range(2)]
    ws = [mk.workspace(t.gpu, 2, t.max_pages) for _ in range(2)]
    ss = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            mk.paged_attn_decode_shaped(t.gpu, sh, 0, qs[i], bt, tags, sl, outs[i], None, ws[i], stream=ss[i])
    torch.cuda.synchronize()
    for i in range(2):
        want = sref.decode(t.orc, 0, ref.bf16_f64(qs[i].cpu().numpy()), t.obt, t.otags, t.cur, kw)
        assert np.all(np.abs(outs[i].cpu().numpy() - want[0]).max(2) <= want[2])


# ---------------------------------------------------------------- the step

def _rope(d, rot, axes=1, interleaved=False):
    import paper_2608_23834_amd as mk
    m = rot // 2
    freq = 1e4 ** (-np.arange(m) / max(m, 1))
    axis = (np.arange(m) % axes).astype(np.uint8)
    return mk.Rope(d, freq, axis, axes, interleaved=interleaved) if m else None, freq, axis


def _norm(rng, d, heads, kind):
    import paper_2608_23834_amd as mk
    if kind is None:
        return None, None
    shape = (d,) if kind == "one" else (heads, d)
    w = wl.bf16_round((1 + 0.3 * rng.standard_normal(shape)).astype(np.float32))
    return mk.HeadNorm(d, _i16(w), eps=1e-5, unit_offset=kind == "heads"), w


def _made(x, w, kind, pos, freq, axis, inter):
    """Rows as the step makes them."""
    if kind is None:
        return ref.rotate(x, pos, freq, axis, inter) if len(freq) else x
    return nref.norm_rotate(x, w, 1e-5, 1.0 if kind == "heads" else 0.0, pos, freq, axis, inter)


STEPS = [  # d, hq, hkv, rot, axes, interleaved, q norm, k norm
    (256, 24, 4, 64, 3, False, "one", "one"), (256, 16, 2, 256, 1, True, "heads", "heads"), (256, 16, 1, 20, 1, False, "one", None),
    (128, 8, 1, 128, 1, False, "one", "heads"), (128, 32, 8, 96, 2, True, None, "one"), (128, 6, 2, 0, 1, False, "heads", "one"),
    (256, 24, 4, 0, 1, False, None, None), (128, 16, 1, 10, 1, True, None, None), (256, 6, 1, 250, 4, False, "one", "one"),
]


@pytest.mark.parametrize("d,hq,hkv,rot,axes,inter,kq,kk", STEPS)
def test_step(d, hq, hkv, rot, axes, inter, kq, kk):
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(rot + d + hq)
    lens = [0, 15, 16, 700, 2003, 333]
    t = _twin(_w(d, hq, hkv, 6, 2), lens, 2, headroom=64)
    rope, freq, axis = _rope(d, rot, axes, inter)
    qn, wq = _norm(rng, d, hq, kq)
    kn, wk = _norm(rng, d, hkv, kk)
    ws = mk.workspace(t.gpu, 6, t.max_pages)
    kinds = [{}, dict(cap=5.0, sinks=rng.standard_normal(hq)), dict(window=16, slopes=_slopes(hq)),
             dict(window=300, cap=9.0), dict(first_keys=[0, 30, 17, 100, 5000, 333]), dict(scale=0.2, window=1)]
    for step, kw in enumerate(kinds):
        q, k, v = _bits(rng, 6, hq, d), _bits(rng, 6, hkv, d), _bits(rng, 6, hkv, d)
        sb = np.array(t.cur, np.int32)
        pos = rng.integers(0, 100000, (axes, 6)).astype(np.int32) if step % 2 else np.tile(sb, (axes, 1))
        layer = step % 2
        out = torch.full((6, hq, d), float("nan"), device="cuda")
        lse = torch.full((6, hq), float("nan"), device="cuda")
        ws.fill_(0xFF)
        mk.paged_attn_decode_append_shaped(t.gpu, _shaping(kw), rope, qn, kn, layer, _i16(q), _i16(k), _i16(v),
                                           _gpu(pos) if step % 2 and rope else None, t.bt, t.tags, _gpu(sb), out, lse, ws)
        torch.cuda.synchronize()
        qr = _made(q, wq, kq, pos, freq, axis, inter)
        kr = _made(k, wk, kk, pos, freq, axis, inter)
        assert t.orc.append(layer, t.obt, t.otags, sb, np.arange(7, dtype=np.int32), kr[None], v[None]) == 0
        t.check_tables()
        t.check_pages()
        want = sref.decode(t.orc, layer, ref.bf16_f64(qr), t.obt, t.otags, sb + 1, kw)
        _near(out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64), want)
        if layer:
            t.advance()


def test_step_that_fails_gives_zeros():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(6)
    t = _twin(_w(256, 8, 2, 3), [100, 64, 33], headroom=32)
    rope, _, _ = _rope(256, 64)
    kn, _ = _norm(rng, 256, 2, "one")
    q, k = _i16(_bits(rng, 3, 8, 256)), _i16(_bits(rng, 3, 2, 256))
    before = t.gpu.fp8_view().clone(), t.bt.clone(), t.tags.clone()
    for bad in ([100, -1, 33], [100, 16 * t.max_pages, 33], [100, 64, 2 ** 31 - 1]):
        for kw in ({}, dict(window=20, sinks=np.ones(8)), dict(first_keys=[50, 60, 2 ** 31 - 1])):
            out = torch.full((3, 8, 256), float("nan"), device="cuda")
            mk.paged_attn_decode_append_shaped(t.gpu, _shaping(kw), rope, None, kn, 0, q, k, k, None, t.bt, t.tags, _i32(bad),
                                               out, None, mk.workspace(t.gpu, 3, t.max_pages))
            assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]
            assert bool((out == 0).all())
    assert torch.equal(before[0], t.gpu.fp8_view()) and torch.equal(before[1], t.bt) and torch.equal(before[2], t.tags)
    t.check_tables()


def test_steps_in_two_graphs_over_one_workspace():
    """A step with a window and one without, captured and replayed in turn."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(14)
    t = _twin(_w(256, 24, 4, 3, 2), [500, 31, 1200], 2, recent=128, headroom=128)
    rope, freq, axis = _rope(256, 64)
    qn, wq = _norm(rng, 256, 24, "one")
    kn, wk = _norm(rng, 256, 4, "one")
    kinds = [dict(window=200, sinks=rng.standard_normal(24).astype(np.float32)), dict(cap=6.0)]
    sh = [_shaping(kw) for kw in kinds]
    ws = mk.workspace(t.gpu, 3, t.max_pages)
    q, k, v = [torch.zeros((2, 3, h, 256), dtype=torch.int16, device="cuda") for h in (24, 4, 4)]
    sb, out, lse = _i32(t.cur), torch.zeros((2, 3, 24, 256), device="cuda"), torch.zeros((2, 3, 24), device="cuda")

    def call(i):
        mk.paged_attn_decode_append_shaped(t.gpu, sh[i], rope, qn, kn, i, q[i], k[i], v[i], None, t.bt, t.tags, sb, out[i], lse[i], ws)

    def feed():
        for x in (q, k, v):
            x.copy_(_i16(_bits(rng, *x.shape)))
        sb.copy_(_i32(t.cur))

    def check():
        torch.cuda.synchronize()
        s = np.array(t.cur, np.int32)
        pos = s[None]
        for i in range(2):
            qb, kb, vb = [x[i].cpu().numpy().view(np.uint16) for x in (q, k, v)]
            kr = nref.norm_rotate(kb, wk, 1e-5, 0.0, pos, freq, axis, False)
            assert t.orc.append(i, t.obt, t.otags, s, np.arange(4, dtype=np.int32), kr[None], vb[None]) == 0
            qr = nref.norm_rotate(qb, wq, 1e-5, 0.0, pos, freq, axis, False)
            want = sref.decode(t.orc, i, ref.bf16_f64(qr), t.obt, t.otags, s + 1, kinds[i])
            _near(out[i].cpu().numpy().astype(np.float64), lse[i].cpu().numpy().astype(np.float64), want)
        t.check_tables()
        t.check_pages()
        t.advance()
    feed()
    call(0)
    call(1)
    check()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    for _ in range(20):
        feed()
        for g in graphs:
            g.replay()
        check()
