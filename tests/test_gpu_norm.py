"""Head norms with the rotation in the same pass, and appends of normed keys, against a 64-bit numpy
form and the CPU oracle.  Everything is fp64 with one rounding to bf16, so bits are compared: 2^-50
of a value moves a rounding once in 2^41 values, and these tests hold fewer than 2^27."""
import dataclasses

import numpy as np
import pytest

import _norm_ref as nref
import _rope_ref as ref
import mkv_workloads as wl

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _gpu(a):
    return _torch().from_numpy(np.ascontiguousarray(a)).cuda()


def _i16(bits):
    return _gpu(np.asarray(bits).view(np.int16))


def _rope(d, rot, axes=1, interleaved=False, scale=1.0, base=1e4):
    import paper_2608_23834_amd as mk
    m = rot // 2
    freq = base ** (-np.arange(m) / max(m, 1))
    axis = (np.arange(m) % axes).astype(np.uint8)
    return mk.Rope(d, freq, axis, axes, interleaved=interleaved, scale=scale) if m else None, freq, axis


def _bits(rng, *shape):
    return wl.bf16_round(rng.standard_normal(shape).astype(np.float32))


def _weights(rng, *shape):
    return wl.bf16_round((1.0 + 0.3 * rng.standard_normal(shape)).astype(np.float32))


ROWS = [  # d, rot, axes, interleaved, tokens, heads, rope scale, weights, add, eps
    (256, 256, 1, False, 1, 24, 1.0, "one", 0.0, 1e-6), (256, 256, 3, True, 33, 5, 1.0, "heads", 0.0, 1e-5),
    (256, 64, 1, False, 70, 24, 1.0, "one", 1.0, 1e-6), (256, 0, 1, False, 3, 7, 1.0, "heads", 1.0, 1e-6),
    (128, 128, 4, False, 1025, 8, 1.25, "none", 1.0, 1e-6), (128, 96, 3, True, 17, 3, 0.5, "one", 0.0, 1.0),
    (128, 20, 1, False, 5, 2, 1.0, "heads", 0.0, 1e-30), (256, 20, 2, True, 9, 7, 1.0, "one", 0.0, 1e-6),
    (256, 2, 1, False, 2, 1, 1.0, "one", 0.0, 1e-6), (128, 126, 1, False, 6, 4, 1.0, "heads", 0.0, 1e-6),
    (256, 254, 3, True, 4, 6, 1.0, "heads", 1.0, 1e-6), (256, 10, 1, False, 130, 9, 2.0, "one", 0.0, 1e-6),
    (128, 0, 1, False, 300, 1, 1.0, "none", 0.0, 1e-6),
]


@pytest.mark.parametrize("d,rot,axes,inter,n,heads,scale,weights,add,eps", ROWS)
def test_rows_match_64_bits(d, rot, axes, inter, n, heads, scale, weights, add, eps):
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(rot * 7 + n)
    rope, freq, axis = _rope(d, rot, axes, inter, scale)
    w = {"none": None, "one": _weights(rng, d), "heads": _weights(rng, heads, d)}[weights]
    norm = mk.HeadNorm(d, None if w is None else _i16(w), eps=eps, unit_offset=add == 1.0)
    x = _bits(rng, n, heads + 3, d)
    x[0, 1] = 0  # eps alone
    x[-1, heads] = np.uint16(0x0001)
    pos = rng.integers(-1000, 2000000, (axes, n)).astype(np.int32)
    want = nref.norm_rotate(x[:, 1:1 + heads], w, eps, add, pos, freq, axis, inter, scale)
    xg = _i16(x)
    out = torch.full((n, heads + 1, d), 77, dtype=torch.int16, device="cuda")
    at = _gpu(pos) if rope else None
    mk.kv_norm_rope_apply(rope, norm, xg[:, 1:1 + heads], at, out[:, :heads])  # out of packed rows into others
    got = out.cpu().numpy()
    assert np.all(got[:, heads] == 77)
    assert ref.same_bits(got[:, :heads], want)
    assert np.array_equal(xg.cpu().numpy().view(np.uint16), x)
    mk.kv_norm_rope_apply(rope, norm, xg[:, 1:1 + heads], at, xg[:, 1:1 + heads])  # in place
    got = xg.cpu().numpy().view(np.uint16)
    assert ref.same_bits(got[:, 1:1 + heads], want)
    assert np.array_equal(got[:, :1], x[:, :1]) and np.array_equal(got[:, 1 + heads:], x[:, 1 + heads:])


@pytest.mark.parametrize("d", [128, 256])
def test_rows_of_special_values(d):
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(3)
    rope, freq, axis = _rope(d, d // 2)
    x = _bits(rng, 9, 2, d)
    x[0, 0, 5] = 0x7F80                                 # one infinity: the others become zeros
    x[1, 1, 7] = 0x7FC0                                 # NaN: the whole head, and no other
    x[2] = np.uint16(0x7F7F)                            # the largest finite value throughout
    x[3] = rng.choice(np.array([0x0001, 0x8001, 0x007F, 0], np.uint16), (2, d))
    x[4, 0, 3], x[4, 1, 3] = 0x7F7F, 0x0001
    w = _weights(rng, d)
    w[9] = 0                                            # a weight of zero, and a negative one
    w[10] = 0xBF80
    pos = rng.integers(0, 100, (1, 9)).astype(np.int32)
    out = torch.zeros((9, 2, d), dtype=torch.int16, device="cuda")
    mk.kv_norm_rope_apply(rope, mk.HeadNorm(d, _i16(w)), _i16(x), _gpu(pos), out)
    got, want = out.cpu().numpy().view(np.uint16), nref.norm_rotate(x, w, 1e-6, 0.0, pos, freq, axis, False)
    assert np.isnan(ref.bf16_f64(want[1, 1])).all() and not np.isnan(ref.bf16_f64(want[1, 0])).any()
    zero = (got & 0x7FFF == 0) & (want & 0x7FFF == 0)   # (a zero's sign comes from the order of a sum)
    assert ref.same_bits(np.where(zero, 0, got).astype(np.uint16), np.where(zero, 0, want).astype(np.uint16))


def test_rows_on_a_stream_and_in_a_graph():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(5)
    rope, freq, axis = _rope(256, 128)
    w = _weights(rng, 4, 256)
    norm = mk.HeadNorm(256, _i16(w))
    x, pos = _bits(rng, 300, 4, 256), rng.integers(0, 5000, (1, 300)).astype(np.int32)
    xg, pg = _i16(x), _gpu(pos)
    out = torch.zeros_like(xg)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    mk.kv_norm_rope_apply(rope, norm, xg, pg, out, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert ref.same_bits(out.cpu().numpy(), nref.norm_rotate(x, w, 1e-6, 0.0, pos, freq, axis, False))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mk.kv_norm_rope_apply(rope, norm, xg, pg, out)
    for k in range(3):
        x = _bits(rng, 300, 4, 256)
        xg.copy_(_i16(x))
        pg += 100 * k
        g.replay()
        torch.cuda.synchronize()
        assert ref.same_bits(out.cpu().numpy(), nref.norm_rotate(x, w, 1e-6, 0.0, pg.cpu().numpy(), freq, axis, False))


# ---------------------------------------------------------------- appends

def _w(d, hq, hkv, n_req, layers=1):
    return dataclasses.replace(wl.scaled(wl.workload(2), (16,) * n_req, layers), head_dim=d, n_q_heads=hq, n_kv_heads=hkv)


def _twin(w, lens, layers, recent=64):
    from _harness import Twin
    t = Twin(w, n_layers=layers, lens=lens, recent=recent)
    t.cur = [0] * len(lens)
    return t


def _append(t, rope_args, norm_args, counts, rng, layer=-1, positions=True, pad=0, grow=1.0):
    """The same raw rows to the GPU and, normed and rotated in numpy, to the oracle."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    rope, freq, axis, inter = rope_args
    norm, nw, eps, add = norm_args
    w, n = t.w, int(sum(counts))
    axes = rope.n_axes if rope else 1
    LL = t.L if layer < 0 else 1
    # (a norm takes the rows' size away: what grows is the values, and by rows the keys)
    K = wl.bf16_round((rng.uniform(0.1, 5.0, (LL, n, 1, 1)) * rng.standard_normal((LL, n, w.n_kv_heads, w.head_dim))).astype(np.float32))
    V = wl.bf16_round((grow * rng.standard_normal((LL, n, w.n_kv_heads, w.head_dim))).astype(np.float32))
    sb = np.array(t.cur, np.int32)
    cu = np.r_[0, np.cumsum(counts)].astype(np.int32)
    cache = np.concatenate([np.arange(c) + b for b, c in zip(sb, counts)] + [np.zeros(0, int)]).astype(np.int32)
    pos = rng.integers(0, 100000, (axes, n)).astype(np.int32) if positions else np.tile(cache, (axes, 1))

    def rows(x):  # pad: rows of a wider buffer
        if not pad:
            return _i16(x if layer < 0 else x[0])
        big = torch.full((LL, n, w.n_kv_heads + pad, w.head_dim), 12345, dtype=torch.int16, device="cuda")
        big[:, :, :w.n_kv_heads] = _i16(x)
        return (big if layer < 0 else big[0])[..., :w.n_kv_heads, :]
    mk.kv_append_fp8_norm_rope(t.gpu, rope, norm, layer, t.bt, t.tags, _gpu(sb), _gpu(cu),
                               _gpu(pos) if positions and rope else None, rows(K), rows(V))
    lw = [None if nw is None else nw[i] if nw.ndim == 3 else nw for i in range(LL)]
    Kr = np.stack([nref.norm_rotate(k, x, eps, add, pos, freq, axis, inter) for k, x in zip(K, lw)])
    assert t.orc.append(layer, t.obt, t.otags, sb, cu, Kr, V) == 0
    t.cur = [c + k for c, k in zip(t.cur, counts)]
    torch.cuda.synchronize()
    t.check_tables()
    t.check_pages()


@pytest.mark.parametrize("d,hq,hkv,rot,axes,inter,weights,add", [
    (256, 24, 4, 256, 3, False, "layers", 0.0), (256, 24, 4, 64, 1, True, "one", 1.0), (128, 32, 8, 128, 1, True, "heads", 0.0),
    (128, 8, 1, 20, 2, False, "one", 0.0), (256, 16, 2, 250, 2, True, "heads", 0.0), (128, 32, 2, 96, 4, False, "none", 0.0),
    (256, 8, 1, 0, 1, False, "layers", 1.0), (128, 8, 1, 128, 1, False, "one", 0.0), (256, 8, 1, 256, 1, True, "one", 0.0),
    (256, 8, 1, 10, 1, False, "one", 0.0), (128, 16, 4, 0, 1, False, "one", 0.0),
])
def test_append_bit_exact(d, hq, hkv, rot, axes, inter, weights, add):
    import paper_2608_23834_amd as mk
    L = 1 if hkv == 1 and weights == "one" else 2  # one (layer, head) pair, and more
    w = _w(d, hq, hkv, 5, L)
    rng = np.random.default_rng(rot + d)
    ra = (*_rope(d, rot, axes, inter), inter)
    nw = {"none": None, "one": _weights(rng, d), "heads": _weights(rng, hkv, d), "layers": _weights(rng, L, hkv, d)}[weights]
    na = (mk.HeadNorm(d, None if nw is None else _i16(nw), eps=1e-5, unit_offset=add == 1.0), nw, 1e-5, add)
    t = _twin(w, [600, 200, 100, 40, 700], L)
    # small calls (one wave per task), then large ones (plan and quantize), partly filled pages
    # kept, grown (their codes re-rounded) and opened
    for i, (counts, grow) in enumerate([([1, 0, 3, 17, 1], 1.0), ([1, 1, 1, 1, 1], 3.0), ([300, 5, 0, 1, 333], 1.0),
                                        ([7, 100, 90, 20, 200], 5.0), ([1, 1, 1, 1, 1], 0.1), ([260, 0, 0, 0, 0], 1.0)]):
        _append(t, ra, na, counts, rng, positions=i % 2 == 0, pad=i % 3, grow=grow)


def test_append_single_layers():
    import paper_2608_23834_amd as mk
    w = _w(256, 24, 4, 3, 3)
    rng = np.random.default_rng(8)
    ra = (*_rope(256, 128, 2), False)
    nw = _weights(rng, 4, 256)
    na = (mk.HeadNorm(256, _i16(nw)), nw, 1e-6, 0.0)
    for counts in ([2, 0, 40], [300, 17, 600]):
        t = _twin(w, [700, 100, 700], 3)
        for layer in (1, 0, 2):
            t.cur = [0] * 3
            _append(t, ra, na, counts, rng, layer=layer, positions=layer != 0, pad=layer)


def test_append_equals_rows_then_append():
    """Normed and rotated rows appended plainly leave the same pages, NaN and infinities among them."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(21)
    vals = np.array([0x0000, 0x8000, 0x0001, 0x8001, 0x0080, 0x7F7F, 0x7F80, 0x7FC0, 0x3F80, 0xBF81], np.uint16)
    n, w = 640, _w(256, 8, 2, 1)
    K, V = _bits(rng, n, 2, 256), _bits(rng, n, 2, 256)
    for p in range(20):
        sel = rng.random((16, 2, 256)) < (0.001, 0.02, 1.0)[p % 3]
        K[16 * p: 16 * p + 16] = np.where(sel, rng.choice(vals[: 6 + p % 5], (16, 2, 256)), K[16 * p: 16 * p + 16])
    K[16 * 21: 16 * 22] = 0
    rope, _, _ = _rope(256, 64, 1)
    norm = mk.HeadNorm(256, _i16(_weights(rng, 256)))
    pos = _gpu(np.arange(n, dtype=np.int32)[None])
    rows = torch.zeros((n, 2, 256), dtype=torch.int16, device="cuda")
    mk.kv_norm_rope_apply(rope, norm, _i16(K), pos, rows)
    got = []
    for form in range(3):
        t = _twin(w, [n], 1)
        for a, b in [(0, n)] if form < 2 else [(16 * i, 16 * i + 16) for i in range(n // 16)]:
            sb, cu = _gpu(np.array([a], np.int32)), _gpu(np.array([0, b - a], np.int32))
            if form == 0:
                mk.kv_append_fp8(t.gpu, 0, t.bt, t.tags, sb, cu, rows, _i16(V))
            else:
                mk.kv_append_fp8_norm_rope(t.gpu, rope, norm, 0, t.bt, t.tags, sb, cu, pos[:, a:b].contiguous(),
                                           _i16(K[a:b]), _i16(V[a:b]))
        torch.cuda.synchronize()
        order = t.bt[0].long()
        got.append((t.gpu.fp8_view()[0, order].cpu().numpy(), t.gpu.fp8_scales_view()[0, order].cpu().numpy().view(np.uint32)))
    for g in got[1:]:
        assert np.array_equal(g[0], got[0][0])
        nan = np.isnan(got[0][1].view(np.float32))  # (any NaN equals any NaN)
        assert np.array_equal(np.isnan(g[1].view(np.float32)), nan) and np.array_equal(g[1][~nan], got[0][1][~nan])


def test_append_that_fails_changes_nothing():
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(2)
    w = _w(128, 8, 2, 2)
    nw = _weights(rng, 128)
    norm = mk.HeadNorm(128, _i16(nw))
    ra = (*_rope(128, 64), False)
    t = _twin(w, [400, 40], 1)
    _append(t, ra, (norm, nw, 1e-6, 0.0), [30, 20], rng)
    before = t.gpu.fp8_view().clone()
    for n, start in ((3, -1), (3, 16 * t.max_pages - 2), (300, 16 * t.max_pages - 200)):
        k = _i16(_bits(rng, n, 2, 128))
        mk.kv_append_fp8_norm_rope(t.gpu, ra[0], norm, 0, t.bt, t.tags, _gpu(np.array([start, 20], np.int32)),
                                   _gpu(np.array([0, n, n], np.int32)), None, k, k)
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]
    assert _torch().equal(before, t.gpu.fp8_view())
    t.check_tables()
