"""Rotation of rows, appends that rotate their keys and the decode step that rotates both,
against a 64-bit numpy rotation, the plain append and the CPU oracle: bit for bit wherever
bf16 rows or FP8 pages come out."""
import ctypes
import dataclasses

import numpy as np
import pytest

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
    freq = base ** (-np.arange(m) / m)
    axis = (np.arange(m) % axes).astype(np.uint8)
    return mk.Rope(d, freq, axis, axes, interleaved=interleaved, scale=scale), freq, axis


def _bits(rng, *shape):
    return wl.bf16_round(rng.standard_normal(shape).astype(np.float32))


@pytest.mark.parametrize("d,rot,axes,inter,n,heads,scale", [
    (256, 256, 1, False, 1, 24, 1.0), (256, 256, 3, True, 33, 5, 1.0), (256, 64, 1, False, 70, 24, 1.0),
    (256, 64, 2, True, 3, 1, 1.25), (128, 128, 4, False, 1025, 8, 1.0), (128, 96, 3, True, 17, 3, 0.5),
    (128, 20, 1, False, 5, 2, 1.0), (256, 20, 2, True, 9, 7, 1.0), (256, 2, 1, False, 2, 1, 1.0),
    (128, 126, 1, False, 6, 4, 1.0), (256, 254, 3, True, 4, 6, 1.0), (256, 8, 1, False, 3, 2, 2.0),
])
def test_apply_matches_64_bits(d, rot, axes, inter, n, heads, scale):
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(rot * 7 + n)
    rope, freq, axis = _rope(d, rot, axes, inter, scale)
    x = _bits(rng, n, heads + 3, d)
    pos = rng.integers(-1000, 2000000, (axes, n)).astype(np.int32)
    pos[:, 0] = 0
    if n > 2:
        pos[0, 1], pos[-1, 2] = 2 ** 31 - 1, -2 ** 31
    want = ref.rotate(x[:, 1:1 + heads], pos, freq, axis, inter, scale)
    xg = _i16(x)
    out = torch.full((n, heads + 1, d), 77, dtype=torch.int16, device="cuda")
    mk.kv_rope_apply(rope, xg[:, 1:1 + heads], _gpu(pos), out[:, :heads])  # out of packed rows into others
    got = out.cpu().numpy()
    assert np.all(got[:, heads] == 77)
    assert ref.same_bits(got[:, :heads], want)
    assert np.array_equal(xg.cpu().numpy().view(np.uint16), x)
    mk.kv_rope_apply(rope, xg[:, 1:1 + heads], _gpu(pos), xg[:, 1:1 + heads])  # in place
    got = xg.cpu().numpy().view(np.uint16)
    assert ref.same_bits(got[:, 1:1 + heads], want)
    assert np.array_equal(got[:, :1], x[:, :1]) and np.array_equal(got[:, 1 + heads:], x[:, 1 + heads:])


def test_apply_special_values():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rope, freq, axis = _rope(128, 64)
    vals = np.array([0x0000, 0x8000, 0x0001, 0x8001, 0x007F, 0x0080, 0x7F7F, 0xFF7F, 0x7F80, 0xFF80, 0x7FC0, 0x3F80],
                    np.uint16)
    rng = np.random.default_rng(3)
    x = rng.choice(vals, (64, 2, 128)).astype(np.uint16)
    pos = rng.integers(0, 100, (1, 64)).astype(np.int32)
    pos[0, :4] = 0
    out = torch.zeros((64, 2, 128), dtype=torch.int16, device="cuda")
    mk.kv_rope_apply(rope, _i16(x), _gpu(pos), out)
    got, want = out.cpu().numpy().view(np.uint16), ref.rotate(x, pos, freq, axis, False)
    # a sum that cancels exactly is +0 or -0 with the order of its terms
    zero = (got & 0x7FFF == 0) & (want & 0x7FFF == 0)
    assert ref.same_bits(np.where(zero, 0, got).astype(np.uint16), np.where(zero, 0, want).astype(np.uint16))


def test_apply_refusals_and_empty():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rope, _, _ = _rope(128, 64)
    L = mk.lib()
    x = torch.zeros((4, 4, 128), dtype=torch.int16, device="cuda")
    pos = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
    p, q = ctypes.c_void_p(x.data_ptr()), ctypes.c_void_p(pos.data_ptr())

    def call(n=4, h=2, src=p, xs=512, ps=q, out=p, os=512):
        return L.kv_rope_apply(rope.handle, n, h, src, xs, ps, out, os, None)
    assert call(n=0) == 0 and call(n=0, src=None, ps=None, out=None) == 0
    assert call(n=-1) == 1 and call(h=0) == 1 and call(src=None) == 1 and call(ps=None) == 1 and call(out=None) == 1
    assert call(xs=255) == 1 and call(xs=252) == 1 and call(os=514) == 1 and call(xs=1 << 32) == 4
    assert call(out=ctypes.c_void_p(x.data_ptr() + 256)) == 1  # overlapping, not in place
    assert call(out=ctypes.c_void_p(x.data_ptr() + 4)) == 1    # misaligned
    with pytest.raises(ValueError):
        mk.kv_rope_apply(rope, x, pos[:, :3], x)
    with pytest.raises(ValueError):
        mk.kv_rope_apply(rope, x[..., ::2], pos, x[..., ::2])


def test_apply_other_stream():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rope, freq, axis = _rope(256, 256)
    rng = np.random.default_rng(5)
    x, pos = _bits(rng, 300, 4, 256), rng.integers(0, 5000, (1, 300)).astype(np.int32)
    xg, pg = _i16(x), _gpu(pos)
    out = torch.zeros_like(xg)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    mk.kv_rope_apply(rope, xg, pg, out, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert ref.same_bits(out.cpu().numpy(), ref.rotate(x, pos, freq, axis, False))


@pytest.mark.parametrize("rot", [128, 6])
def test_apply_of_many_tokens(rot):
    """More tokens than one launch takes, byte offsets past 2^31 between input and positions."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    n = (1 << 23) + 77
    rope, freq, axis = _rope(128, rot, 2)
    rng = np.random.default_rng(rot)
    some = _bits(rng, 4096, 1, 128)
    x = _i16(some).repeat((n + 4095) // 4096, 1, 1)[:n].contiguous()
    pos = torch.arange(2 * n, dtype=torch.int32, device="cuda").view(2, n)
    mk.kv_rope_apply(rope, x, pos, x)
    for a in (0, (1 << 22) - 40, (1 << 23) - 40, n - 50):
        i = np.arange(a, a + 50)
        want = ref.rotate(some[i % 4096], np.stack([i, n + i]).astype(np.int32), freq, axis, False)
        assert ref.same_bits(x[a:a + 50].cpu().numpy(), want), a


def test_wrapper_refusals():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rope, _, _ = _rope(128, 64, 2)
    x = torch.zeros((4, 2, 128), dtype=torch.int16, device="cuda")
    pos = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    for bad in (pos.long(), pos[:1], pos.cpu(), pos.t().contiguous().t()):
        with pytest.raises(ValueError):
            mk.kv_rope_apply(rope, x, bad, x)
    rope.device += 1  # as if its table lay on another card
    with pytest.raises(ValueError):
        mk.kv_rope_apply(rope, x, pos, x)
    rope.device -= 1
    t = _twin(_w(128, 8, 2, 1), [64], 2)
    z, cu = torch.zeros(1, dtype=torch.int32, device="cuda"), _gpu(np.array([0, 4], np.int32))
    two = torch.zeros((2, 4, 2, 128), dtype=torch.int16, device="cuda")
    for layer, k, v in ((0, x, x[:3]), (-1, x, x), (0, two, two), (-1, two[:1], two[:1]), (0, x[:, :1], x[:, :1])):
        with pytest.raises(ValueError):
            mk.kv_append_fp8_rope(t.gpu, rope, layer, t.bt, t.tags, z, cu, pos, k, v)
    t.check_tables()


# ---------------------------------------------------------------- appends

def _w(d, hq, hkv, n_req, layers=1):
    return dataclasses.replace(wl.scaled(wl.workload(2), (16,) * n_req, layers), head_dim=d, n_q_heads=hq, n_kv_heads=hkv)


def _twin(w, lens, layers, recent=64):
    from _harness import Twin
    t = Twin(w, n_layers=layers, lens=lens, recent=recent)
    t.cur = [0] * len(lens)
    return t


def _append(t, rope_args, counts, rng, layer=-1, positions=True, pad=0, grow=1.0):
    """The same unrotated rows to the GPU (rotated append) and, rotated in numpy, to the oracle."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    rope, freq, axis, inter = rope_args
    w, n = t.w, int(sum(counts))
    LL = t.L if layer < 0 else 1
    K = wl.bf16_round((grow * rng.standard_normal((LL, n, w.n_kv_heads, w.head_dim))).astype(np.float32))
    V = wl.bf16_round((grow * rng.standard_normal((LL, n, w.n_kv_heads, w.head_dim))).astype(np.float32))
    sb = np.array(t.cur, np.int32)
    cu = np.r_[0, np.cumsum(counts)].astype(np.int32)
    cache = np.concatenate([np.arange(c) + b for b, c in zip(sb, counts)] + [np.zeros(0, int)]).astype(np.int32)
    pos = rng.integers(0, 100000, (rope.n_axes, n)).astype(np.int32) if positions else np.tile(cache, (rope.n_axes, 1))

    def rows(x):  # pad: rows of a wider buffer
        if not pad:
            return _i16(x if layer < 0 else x[0])
        big = torch.full((LL, n, w.n_kv_heads + pad, w.head_dim), 12345, dtype=torch.int16, device="cuda")
        big[:, :, :w.n_kv_heads] = _i16(x)
        return (big if layer < 0 else big[0])[..., :w.n_kv_heads, :]
    mk.kv_append_fp8_rope(t.gpu, rope, layer, t.bt, t.tags, _gpu(sb), _gpu(cu), _gpu(pos) if positions else None,
                          rows(K), rows(V))
    Kr = np.stack([ref.rotate(k, pos, freq, axis, inter) for k in K])
    assert t.orc.append(layer, t.obt, t.otags, sb, cu, Kr, V) == 0
    t.cur = [c + k for c, k in zip(t.cur, counts)]
    torch.cuda.synchronize()
    t.check_tables()
    t.check_pages()


@pytest.mark.parametrize("d,hq,hkv,rot,axes,inter", [
    (256, 24, 4, 256, 3, False), (256, 24, 4, 64, 1, True), (128, 32, 8, 128, 1, True), (128, 8, 1, 20, 2, False),
    (256, 16, 2, 250, 2, True), (128, 32, 2, 96, 4, False),
])
def test_append_bit_exact(d, hq, hkv, rot, axes, inter):
    w = _w(d, hq, hkv, 5, 2)
    rng = np.random.default_rng(rot + d)
    rope, freq, axis = _rope(d, rot, axes, inter)
    ra = (rope, freq, axis, inter)
    t = _twin(w, [600, 200, 100, 40, 700], 2)
    # small calls (one wave per task), then large ones (plan and quantize), partly filled pages
    # kept, grown (their codes re-rounded) and opened
    for i, (counts, grow) in enumerate([([1, 0, 3, 17, 1], 1.0), ([1, 1, 1, 1, 1], 3.0), ([300, 5, 0, 1, 333], 1.0),
                                        ([7, 100, 90, 20, 200], 5.0), ([1, 1, 1, 1, 1], 0.1), ([260, 0, 0, 0, 0], 1.0)]):
        _append(t, ra, counts, rng, positions=i % 2 == 0, pad=i % 3, grow=grow)


def test_append_single_layers():
    w = _w(256, 24, 4, 3, 3)
    rng = np.random.default_rng(8)
    rope, freq, axis = _rope(256, 128, 2)
    for counts in ([2, 0, 40], [300, 17, 600]):
        t = _twin(w, [700, 100, 700], 3)
        for layer in (1, 0, 2):
            t.cur = [0] * 3
            _append(t, (rope, freq, axis, False), counts, rng, layer=layer, positions=layer != 0, pad=layer)


@pytest.mark.parametrize("turned", [False, True])
def test_append_special_values(turned):
    """NaN, infinities, zeros and the smallest and largest values: one large call and calls of single
    pages leave the same pages (different kernels)."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(21)
    vals = np.array([0x0000, 0x8000, 0x0001, 0x8001, 0x0080, 0x7F7F, 0xFF7F, 0x7F80, 0xFF80, 0x7FC0, 0x3F80, 0xBF81], np.uint16)
    n, w = 640, _w(256, 8, 2, 1)
    K, V = _bits(rng, n, 2, 256), _bits(rng, n, 2, 256)
    for x in (K, V):  # page by page: a few special values, whole rows of them, tiny scales
        for p in range(0, 20):
            sel = rng.random((16, 2, 256)) < (0.001, 0.02, 1.0)[p % 3]
            x[16 * p: 16 * p + 16] = np.where(sel, rng.choice(vals[: 7 + p % 6], (16, 2, 256)), x[16 * p: 16 * p + 16])
        x[16 * 20: 16 * 21] = rng.choice(np.array([0x0001, 0x8001, 0x0003, 0], np.uint16), (16, 2, 256))
        x[16 * 21: 16 * 22] = 0
    rope, _, _ = _rope(256, 64, 1)
    pos = _gpu(np.arange(n, dtype=np.int32)[None])

    def put(t, a, b):
        sb, cu = _gpu(np.array([a], np.int32)), _gpu(np.array([0, b - a], np.int32))
        if turned:
            mk.kv_append_fp8_rope(t.gpu, rope, 0, t.bt, t.tags, sb, cu, pos[:, a:b].contiguous(), _i16(K[a:b]), _i16(V[a:b]))
        else:
            mk.kv_append_fp8(t.gpu, 0, t.bt, t.tags, sb, cu, _i16(K[a:b]), _i16(V[a:b]))
    ta, tb = _twin(w, [n], 1), _twin(w, [n], 1)
    put(ta, 0, n)
    for a in range(0, n, 16):
        put(tb, a, a + 16)
    torch.cuda.synchronize()
    assert torch.equal(ta.bt, tb.bt)
    assert torch.equal(ta.gpu.fp8, tb.gpu.fp8)
    assert np.array_equal(ta.gpu.fp8_scales.cpu().numpy().view(np.uint32), tb.gpu.fp8_scales.cpu().numpy().view(np.uint32))


@pytest.mark.parametrize("hkv", [1, 2, 3, 5])
@pytest.mark.parametrize("d,rot,inter", [(256, 64, False), (256, 20, True), (256, 22, False), (128, 128, True),
                                         (128, 36, False), (128, 126, True), (256, 256, False), (256, 100, True),
                                         (256, 250, False), (128, 32, False), (128, 12, True), (128, 6, False)])
def test_append_grown_pages_of_any_magnitude(d, rot, inter, hkv):
    """Pages that three large calls fill in turn, with values from bf16's subnormals up, equal, a
    little larger or much larger from call to call: the pages of a rotation and a plain append."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(d + rot)
    n_req, w = 96, _w(d, 2 * hkv, hkv, 96)
    ta, tb = _twin(w, [64] * n_req, 1), _twin(w, [64] * n_req, 1)
    rope, _, _ = _rope(d, rot, 2, inter)
    mag = 2.0 ** rng.integers(-134, 4, (n_req, 1, hkv, 1))
    at = np.zeros(n_req, np.int32)
    for call in range(3):
        c = rng.integers(1, 21, n_req)
        cu = np.r_[0, np.cumsum(c)].astype(np.int32)
        n, r = int(cu[-1]), np.repeat(np.arange(n_req), c)
        assert n > 512
        f = rng.choice([0.25, 1.0, 1.0, 1.01, 8.0], (n_req, 1, hkv, 1))
        mag = mag * f
        base = np.sign(rng.standard_normal((n, hkv, d))) * rng.choice([0.5, 1.0, 0.01], (n, hkv, d))
        K, V = (wl.bf16_round((base * mag[r][:, 0]).astype(np.float32)) for _ in range(2))
        pos = np.where(rng.random((2, n)) < 0.5, 0, rng.integers(0, 5000, (2, n))).astype(np.int32)
        kg, vg, pg, sb, cug = _i16(K), _i16(V), _gpu(pos), _gpu(at), _gpu(cu)
        mk.kv_append_fp8_rope(ta.gpu, rope, 0, ta.bt, ta.tags, sb, cug, pg, kg, vg)
        mk.kv_rope_apply(rope, kg, pg, kg)
        mk.kv_append_fp8(tb.gpu, 0, tb.bt, tb.tags, sb, cug, kg, vg)
        torch.cuda.synchronize()
        assert torch.equal(ta.bt, tb.bt) and torch.equal(ta.gpu.fp8, tb.gpu.fp8), call
        assert torch.equal(ta.gpu.fp8_scales.view(torch.int32), tb.gpu.fp8_scales.view(torch.int32)), call
        at = at + c.astype(np.int32)


def test_append_nothing_and_refusals():
    import paper_2608_23834_amd as mk
    torch = _torch()
    w = _w(128, 8, 2, 2)
    t = _twin(w, [64, 64], 1)
    rope, _, _ = _rope(128, 128)
    other, _, _ = _rope(256, 128)
    none = torch.zeros((0, 2, 128), dtype=torch.int16, device="cuda")
    z = torch.zeros(2, dtype=torch.int32, device="cuda")
    mk.kv_append_fp8_rope(t.gpu, rope, 0, t.bt, t.tags, z, torch.zeros(3, dtype=torch.int32, device="cuda"), None, none, none)
    t.check_tables()
    k = torch.zeros((2, 2, 128), dtype=torch.int16, device="cuda")
    cu = _gpu(np.array([0, 1, 2], np.int32))
    with pytest.raises(mk.MkvError) as e:
        mk.kv_append_fp8_rope(t.gpu, other, 0, t.bt, t.tags, z, cu, None, k, k)
    assert e.value.code == 1
    with pytest.raises(mk.MkvError) as e:
        mk.kv_append_fp8_rope(t.gpu, rope, 1, t.bt, t.tags, z, cu, None, k, k)
    assert e.value.code == 4
    # a call that the device refuses changes nothing: a page past the table's end
    bt0 = t.bt.clone()
    mk.kv_append_fp8_rope(t.gpu, rope, 0, t.bt, t.tags, _gpu(np.array([0, 64], np.int32)), cu, None, k, k)
    torch.cuda.synchronize()
    assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]
    assert torch.equal(bt0, t.bt)
    t.check_tables()


# ---------------------------------------------------------------- the decode step

def _step(t, ra, rng, positions, ws=None, stream=None):
    import paper_2608_23834_amd as mk
    torch = _torch()
    rope, freq, axis, inter = ra
    w, n_req = t.w, t.n_req
    K, V = _bits(rng, n_req, w.n_kv_heads, w.head_dim), _bits(rng, n_req, w.n_kv_heads, w.head_dim)
    q = _bits(rng, n_req, w.n_q_heads, w.head_dim)
    sb = np.array(t.cur, np.int32)
    pos = rng.integers(0, 1000000, (rope.n_axes, n_req)).astype(np.int32) if positions else np.tile(sb, (rope.n_axes, 1))
    out = torch.full((n_req, w.n_q_heads, w.head_dim), float("nan"), device="cuda")
    lse = torch.full((n_req, w.n_q_heads), float("nan"), device="cuda")
    ws = t._ws(float("nan")) if ws is None else ws
    args = (_i16(q), _i16(K), _i16(V), _gpu(pos) if positions else None, t.bt, t.tags, _gpu(sb), out, lse, ws)
    mk.paged_attn_decode_append_rope(t.gpu, rope, 0, *args)
    torch.cuda.synchronize()
    Kr, qr = ref.rotate(K, pos, freq, axis, inter), ref.rotate(q, pos, freq, axis, inter)
    assert t.orc.append(0, t.obt, t.otags, sb, np.arange(n_req + 1, dtype=np.int32), Kr[None], V[None]) == 0
    t.cur = [c + 1 for c in t.cur]
    t.check_tables()
    t.check_pages()
    o, l, tol = ref.attend(t.orc, 0, qr, t.obt, t.otags, t.cur)
    go, gl = out.cpu().numpy(), lse.cpu().numpy()
    print(f"  max|dO| {np.abs(go - o).max():.2e} (rel {np.linalg.norm(go - o) / np.linalg.norm(o):.2e}) "
          f"max|dlse| {np.abs(gl - l).max():.2e} smallest bound {tol.min():.2e}", flush=True)
    assert np.all(np.abs(go - o) <= tol[..., None])
    assert np.all(np.abs(gl - l) <= tol + 2.0 ** -22 * np.abs(l))


@pytest.mark.parametrize("d,hq,hkv,rot,axes,inter", [
    (256, 24, 4, 64, 3, False), (256, 16, 2, 256, 1, True), (256, 32, 2, 256, 2, False), (128, 32, 8, 128, 1, False),
    (128, 16, 2, 20, 2, True), (128, 16, 1, 96, 4, False), (256, 24, 4, 250, 1, False), (128, 8, 1, 128, 1, True),
])
def test_decode_step(d, hq, hkv, rot, axes, inter):
    w = _w(d, hq, hkv, 6)
    rng = np.random.default_rng(d + hq + rot)
    rope, freq, axis = _rope(d, rot, axes, inter, base=1e6)
    ra = (rope, freq, axis, inter)
    t = _twin(w, [1500, 333, 64, 17, 3, 900], 1)
    _append(t, ra, [1400, 319, 47, 15, 0, 640], rng)
    t.migrate()
    t.check_tables()
    for i in range(3):  # pages opened, filled and left partly filled
        print(f"\n[rope step] d={d} {hq}/{hkv} rot={rot} axes={axes} step {i}", flush=True)
        _step(t, ra, rng, positions=i != 1)


def test_decode_step_failure_gives_zeros():
    import paper_2608_23834_amd as mk
    torch = _torch()
    w = _w(256, 24, 4, 2)
    rng = np.random.default_rng(4)
    rope, freq, axis = _rope(256, 256)
    t = _twin(w, [64, 64], 1)
    _append(t, (rope, freq, axis, False), [40, 20], rng)
    before = t.gpu.fp8.clone()
    out = torch.full((2, 24, 256), float("nan"), device="cuda")
    lse = torch.zeros((2, 24), device="cuda")
    q, k = _i16(_bits(rng, 2, 24, 256)), _i16(_bits(rng, 2, 4, 256))
    mk.paged_attn_decode_append_rope(t.gpu, rope, 0, q, k, k, None, t.bt, t.tags, _gpu(np.array([40, 64], np.int32)), out,
                                     lse, t._ws(None))
    torch.cuda.synchronize()
    assert mk.kv_pool_check_errors(t.gpu, clear=True) & mk.DEVERR["RANGE"]
    assert torch.equal(before, t.gpu.fp8) and not out.any()
    other, _, _ = _rope(128, 128)
    with pytest.raises(mk.MkvError) as e:
        mk.paged_attn_decode_append_rope(t.gpu, other, 0, q, k, k, None, t.bt, t.tags, _gpu(np.array([40, 20], np.int32)),
                                         out, lse, t._ws(None))
    assert e.value.code == 1


def test_decode_step_captured():
    """A captured step replayed over changing inputs equals the separate calls."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    w = _w(256, 24, 4, 3)
    rng = np.random.default_rng(11)
    rope, freq, axis = _rope(256, 64, 2)
    ta, tb = (_twin(w, [500, 100, 37], 1) for _ in range(2))
    for t in (ta, tb):
        _append(t, (rope, freq, axis, False), [450, 64, 15], np.random.default_rng(2))
        t.migrate()
        mk.paged_attn_set_deterministic(t.gpu, True)
    q = torch.zeros((3, 24, 256), dtype=torch.int16, device="cuda")
    k, v = (torch.zeros((3, 4, 256), dtype=torch.int16, device="cuda") for _ in range(2))
    pos, sb = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros((3, 24, 256), device="cuda"), torch.zeros((3, 24), device="cuda")
    ref_out, ref_lse = torch.zeros_like(out), torch.zeros_like(lse)
    wa, wb = ta._ws(None), tb._ws(None)
    g = None
    for step in range(6):
        q.copy_(_i16(_bits(rng, 3, 24, 256)))
        k.copy_(_i16(_bits(rng, 3, 4, 256)))
        v.copy_(_i16(_bits(rng, 3, 4, 256)))
        pos.copy_(_gpu(rng.integers(0, 10000, (2, 3)).astype(np.int32)))
        sb.copy_(_gpu(np.array(ta.cur, np.int32) + step))
        torch.cuda.synchronize()
        mk.paged_attn_decode_append_rope(ta.gpu, rope, 0, q, k, v, pos, ta.bt, ta.tags, sb, ref_out, ref_lse, wa)
        if step == 1:
            g = torch.cuda.CUDAGraph()
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(g, stream=s):
                mk.paged_attn_decode_append_rope(tb.gpu, rope, 0, q, k, v, pos, tb.bt, tb.tags, sb, out, lse, wb)
            torch.cuda.current_stream().wait_stream(s)
        if g is None:
            mk.paged_attn_decode_append_rope(tb.gpu, rope, 0, q, k, v, pos, tb.bt, tb.tags, sb, out, lse, wb)
        else:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref_out) and torch.equal(lse, ref_lse), step
        assert torch.equal(ta.bt, tb.bt) and torch.equal(ta.gpu.fp8, tb.gpu.fp8), step
    assert mk.kv_pool_check_errors(tb.gpu) == 0
