"""Chunked prefill with shaped scores (bf16 rows) against 64-bit numpy over the CPU oracle's
reconstructed pages, then a run of the operators as a layer of a model makes them."""
import dataclasses

import numpy as np
import pytest

import _norm_ref as nref
import _rope_ref as ref
import _shape_ref as sref
import mkv_workloads as wl
from test_gpu_shaped import _bits, _gpu, _i16, _i32, _norm, _rope, _shaping, _slopes, _twin, _w

pytestmark = pytest.mark.gpu
PAGE = 16


def _torch():
    import torch
    return torch


def _chunk(t, q, cu, kw, lens=None, ws=None, guard=True):
    import paper_2608_23834_amd as mk
    torch = _torch()
    n = len(q)
    out = torch.full((n + 2, t.w.n_q_heads, t.w.head_dim), 0x7FC1, dtype=torch.int16, device="cuda")
    ws = mk.workspace(t.gpu, t.n_req, t.max_pages, n) if ws is None else ws
    ws.fill_(0xFF)
    mk.paged_attn_chunk_shaped(t.gpu, _shaping(kw), 0, _i16(q), _i32(cu), t.bt, t.tags, _i32(t.cur if lens is None else lens),
                               out[:n], ws)
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    assert np.all(got[n:] == 0x7FC1)
    return ref.bf16_f64(got[:n])


def _near(got, want):
    err = np.linalg.norm(got - want[0], axis=2)
    assert np.all(err <= want[1]), (np.argwhere(~(err <= want[1]))[:4], np.nanmax(err / np.maximum(want[1], 1e-30)))


LENS, NQ = [1, 17, 700, 333, 40, 2003], [1, 17, 100, 40, 33, 5]


def _kinds(hq, cu):
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(LENS, NQ)])
    sinks = np.random.default_rng(hq).standard_normal(hq).astype(np.float32)
    sinks[-1] = -np.inf
    docs = np.maximum(0, pos // 50 * 50 - 7)
    odd = docs.copy()
    odd[::3] = pos[::3] + 1          # rows that see nothing
    odd[1::7] = -9
    odd[2::5] = 2 ** 31 - 1
    return [
        {}, dict(cap=5.0), dict(slopes=_slopes(hq)), dict(sinks=sinks + 2), dict(window=1), dict(window=16, sinks=sinks),
        dict(window=50, cap=3.0, slopes=_slopes(hq)), dict(window=1000), dict(first_keys=docs), dict(first_keys=odd, sinks=sinks),
        dict(first_keys=odd, cap=4.0, window=60), dict(prefix_lens=[1, 9, 640, 10 ** 6, 0, 2001]),
        dict(prefix_lens=[0, 17, 700, 300, -4, 5], window=30, slopes=_slopes(hq)), dict(scale=0.02, cap=50.0, prefix_lens=[5] * 6),
        dict(cap=128.0, scale=0.5), dict(cap=200.0, scale=0.5), dict(cap=1e6, scale=0.5), dict(cap=1e-6),
    ]


@pytest.mark.parametrize("d,hq,hkv", [(256, 24, 4), (128, 8, 1), (128, 32, 8), (256, 16, 1), (128, 3, 3)])
def test_chunk(d, hq, hkv):
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(d + hq)
    t = _twin(_w(d, hq, hkv, 6), LENS, recent=128)
    assert (t.otags == 2).any() and (t.otags == 1).any() and (t.otags == 0).any()
    cu = np.r_[0, np.cumsum(NQ)]
    q = wl.bf16_round((2 * rng.standard_normal((cu[-1], hq, d))).astype(np.float32))
    for kw in _kinds(hq, cu):
        want = sref.chunk(t.orc, 0, ref.bf16_f64(q), cu, t.obt, t.otags, t.cur, kw)
        for det in (False, True):  # blocks cut along their pages, and whole
            mk.paged_attn_set_deterministic(t.gpu, det)
            _near(_chunk(t, q, cu, kw), want)
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_long_chunks_and_few_blocks():
    """Blocks cut in many parts, windows that leave a few pages of a long table, a workspace without room for parts."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(3)
    lens, nq = [9000, 5003], [300, 21]
    t = _twin(_w(128, 8, 1, 2), lens, recent=512)
    cu = np.r_[0, np.cumsum(nq)]
    q = wl.bf16_round((2 * rng.standard_normal((cu[-1], 8, 128))).astype(np.float32))
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, nq)])
    small = mk.workspace(t.gpu, 2, t.max_pages, 1)
    for kw in (dict(cap=6.0, sinks=np.ones(8)), dict(window=700), dict(window=4000, slopes=_slopes(8)),
               dict(first_keys=pos // 2500 * 2500, cap=5.0), dict(prefix_lens=[8800, 5003], cap=9.0)):
        want = sref.chunk(t.orc, 0, ref.bf16_f64(q), cu, t.obt, t.otags, t.cur, kw)
        _near(_chunk(t, q, cu, kw), want)
        _near(_chunk(t, q, cu, kw, ws=small), want)
    assert mk.kv_pool_check_errors(t.gpu) == 0


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("power,shift,gain", [(-8, 0.0, 1.0), (-5, 0.0, 1.0), (4, 0.0, 1.0), (11, 0.0, 1.0), (0, 5.0, 2.0 ** -9),
                                              (0, -3.0, 2.0 ** -13), (0, 0.0, 2.0 ** -11), (0, 20.0, 1.0)])
def test_values_of_every_size_and_nearly_equal_scores(d, power, shift, gain):
    """Values times a power of two, or about a common one, and queries whose scores hardly differ: what the
    rounded weights share then must not reach the rows."""
    import paper_2608_23834_amd as mk
    from _harness import Twin
    rng = np.random.default_rng(d + power + 20)
    nq, w = [150, 40], _w(d, 8, 2, 2)
    t = Twin(w, n_layers=1, lens=[1500, 40], recent=256)
    for counts in ([1350, 0], [150, 40]):
        k, v = zip(*(wl.kv_layer(w, 0, n, token_offset=r * 1_000_000 + t.cur[r]) for r, n in enumerate(counts) if n))
        v = wl.bf16_round((wl.bf16_to_f32(np.concatenate(v)) * np.float32(2.0 ** power) + np.float32(shift)).astype(np.float32))
        t.append(counts, layer_kv=(np.concatenate(k)[None], v[None]))
    t.migrate()
    assert (t.otags == 2).any() and (t.otags != 2).any()
    cu = np.r_[0, np.cumsum(nq)]
    q = wl.bf16_round((gain * rng.standard_normal((cu[-1], 8, d))).astype(np.float32))
    for kw in ({}, dict(cap=30.0, first_keys=np.ones(cu[-1], np.int32))):
        want = sref.chunk(t.orc, 0, ref.bf16_f64(q), cu, t.obt, t.otags, t.cur, kw)
        for det in (False, True):
            mk.paged_attn_set_deterministic(t.gpu, det)
            _near(_chunk(t, q, cu, kw), want)
    assert mk.kv_pool_check_errors(t.gpu) == 0


@pytest.mark.parametrize("lens,nq", [([2100, 700], [1100, 300]), ([1200, 1200], [640, 640]), ([1300], [1300])])
def test_second_round_in_parts(lens, nq):
    """More row blocks than compute units per KV head: the cheapest are cut behind the others."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(len(lens) + nq[0])
    t = _twin(_w(128, 32, 32, len(lens)), lens, recent=256)
    cu = np.r_[0, np.cumsum(nq)]
    q = wl.bf16_round((2 * rng.standard_normal((cu[-1], 32, 128))).astype(np.float32))
    for kw in (dict(cap=6.0, sinks=np.ones(32)), dict(window=900, prefix_lens=[900] * len(lens))):
        want = sref.chunk(t.orc, 0, ref.bf16_f64(q), cu, t.obt, t.otags, t.cur, kw)
        for det in (False, True):
            mk.paged_attn_set_deterministic(t.gpu, det)
            _near(_chunk(t, q, cu, kw), want)
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_more_row_blocks_than_a_grid_axis_holds():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(2)
    t = _twin(_w(128, 16, 1, 1), [16])
    kw, n, m = dict(window=9, sinks=np.ones(16)), 8, 40000
    q = _bits(rng, 9 * n, 16, 128)  # nine queries of sixteen heads: two blocks a request

    def call(k):
        out = torch.zeros((9 * k, 16, 128), dtype=torch.int16, device="cuda")
        mk.paged_attn_chunk_shaped(t.gpu, _shaping(kw), 0, _i16(q).repeat(k // n, 1, 1), _i32(9 * np.arange(k + 1)),
                                   t.bt.repeat(k, 1), t.tags.repeat(k, 1), _i32([16] * k), out,
                                   mk.workspace(t.gpu, k, t.max_pages, 9 * k))
        return out

    few, many = call(n), call(m)
    assert few.any() and torch.equal(many, few.repeat(m // n, 1, 1))
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_pages_that_no_row_sees_are_not_read():
    """A page without a readable id is left out; wholly outside the window it is listed but never read."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(5)
    t = _twin(_w(256, 8, 2, 1), [1200], recent=64)
    q = _bits(rng, 40, 8, 256)
    t.gpu.tq3_view()[0, t.bt[0, 3].long()] = 0x7F  # gamma, scale and zero become NaN there
    kw = dict(window=100)
    got = _chunk(t, q, [0, 40], kw)
    _near(got, sref.chunk(t.orc, 0, ref.bf16_f64(q), [0, 40], t.obt, t.otags, [1200], kw))
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_wrong_ranges():
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(8)
    t = _twin(_w(128, 8, 2, 3), [100, 100, 100])
    q = _bits(rng, 30, 8, 128)
    for lens in ([100, 9, 100], [100, 0, 100], [100, 16 * t.max_pages + 1, 100], [100, -2 ** 31, 100]):
        got = _chunk(t, q, [0, 10, 20, 30], dict(window=20, prefix_lens=[50, 2 ** 31 - 1, -1], sinks=np.ones(8)), lens=lens)
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]
        assert np.all(got[10:20] == 0) and np.isfinite(got).all() and got[:10].any() and got[20:].any()


def test_captured():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(11)
    lens, nq = [700, 1300], [64, 30]
    t = _twin(_w(256, 24, 4, 2), lens, recent=256)
    cu = np.r_[0, np.cumsum(nq)]
    kw = dict(cap=5.0, window=500, first_keys=np.zeros(94, np.int32))
    sh, cug, sl = _shaping(kw), _i32(cu), _i32(lens)
    q, out = torch.zeros((94, 24, 256), dtype=torch.int16, device="cuda"), torch.zeros((94, 24, 256), dtype=torch.int16, device="cuda")
    ws = mk.workspace(t.gpu, 2, t.max_pages, 94)

    def call():
        mk.paged_attn_chunk_shaped(t.gpu, sh, 0, q, cug, t.bt, t.tags, sl, out, ws)
    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for k in range(4):
        q.copy_(_i16(_bits(rng, 94, 24, 256)))
        kw["first_keys"] = np.full(94, 200 * k)
        sh.first_keys.fill_(200 * k)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        _near(ref.bf16_f64(out.cpu().numpy()), sref.chunk(t.orc, 0, ref.bf16_f64(q.cpu().numpy()), cu, t.obt, t.otags, lens, kw))


@pytest.mark.parametrize("d,hq,hkv", [(256, 24, 4), (128, 8, 2)])
def test_a_layer_as_a_model_runs_it(d, hq, hkv):
    """Two chunks of a prompt and three decode steps of a layer with norms, rotation, capped scores, a window and
    sinks, pages turning Stale in between; then the cache is read back."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(d)
    t = _twin(_w(d, hq, hkv, 2), [0, 0], recent=64, headroom=400)
    rope, freq, axis = _rope(d, d // 2)
    qn, wq = _norm(rng, d, hq, "one")
    kn, wk = _norm(rng, d, hkv, "heads")
    kw = dict(cap=8.0, window=150, sinks=rng.standard_normal(hq).astype(np.float32))
    sh = _shaping(kw)
    anchor = np.zeros((2, t.max_pages), np.uint8)

    def made(x, w, add, pos):
        return nref.norm_rotate(x, w, 1e-5, add, pos[None], freq, axis, False)
    for counts in ([200, 131], [150, 61]):
        n = sum(counts)
        q, k, v = _bits(rng, n, hq, d), _bits(rng, n, hkv, d), _bits(rng, n, hkv, d)
        sb, cu = np.array(t.cur, np.int32), np.r_[0, np.cumsum(counts)].astype(np.int32)
        pos = np.concatenate([s + np.arange(c) for s, c in zip(sb, counts)])
        mk.kv_append_fp8_norm_rope(t.gpu, rope, kn, 0, t.bt, t.tags, _gpu(sb), _gpu(cu), None, _i16(k), _i16(v))
        assert t.orc.append(0, t.obt, t.otags, sb, cu, made(k, wk, 1.0, pos)[None], v[None]) == 0
        t.cur = [int(s + c) for s, c in zip(sb, counts)]
        qg = _i16(q)
        mk.kv_norm_rope_apply(rope, qn, qg, _i32(pos[None]), qg)
        qr = made(q, wq, 0.0, pos)
        assert ref.same_bits(qg.cpu().numpy(), qr)
        out = torch.zeros((n, hq, d), dtype=torch.bfloat16, device="cuda")
        mk.paged_attn_chunk_shaped(t.gpu, sh, 0, qg, _i32(cu), t.bt, t.tags, _i32(t.cur), out,
                                   mk.workspace(t.gpu, 2, t.max_pages, n))
        want = sref.chunk(t.orc, 0, ref.bf16_f64(qr), cu, t.obt, t.otags, t.cur, kw)
        _near(out.double().cpu().numpy(), want)
        t.migrate(anchor)
    ws = mk.workspace(t.gpu, 2, t.max_pages)
    for _ in range(3):
        q, k, v = _bits(rng, 2, hq, d), _bits(rng, 2, hkv, d), _bits(rng, 2, hkv, d)
        sb = np.array(t.cur, np.int32)
        out, lse = torch.zeros((2, hq, d), device="cuda"), torch.zeros((2, hq), device="cuda")
        mk.paged_attn_decode_append_shaped(t.gpu, sh, rope, qn, kn, 0, _i16(q), _i16(k), _i16(v), None, t.bt, t.tags, _gpu(sb),
                                           out, lse, ws)
        assert t.orc.append(0, t.obt, t.otags, sb, np.arange(3, dtype=np.int32), made(k, wk, 1.0, sb)[None], v[None]) == 0
        t.advance()
        o, l, to, tl = sref.decode(t.orc, 0, ref.bf16_f64(made(q, wq, 0.0, sb)), t.obt, t.otags, t.cur, kw)
        assert np.all(np.abs(out.double().cpu().numpy() - o).max(2) <= to)
        assert np.all(np.abs(lse.double().cpu().numpy() - l) <= tl)
        t.migrate(anchor)
    t.check_tables()
    t.check_pages()
    n = sum(t.cur)
    kv = torch.zeros((2, n, hkv, d), dtype=torch.bfloat16, device="cuda")
    mk.kv_read_tokens(t.gpu, 0, t.bt, t.tags, _i32([0, 0]), _i32([0, t.cur[0], n]), kv[0], kv[1])
    for r in range(2):
        for h in range(hkv):
            want = t.orc.reconstruct(0, r, h, t.obt, t.otags, t.cur[r])
            for j in range(2):
                got = kv[j, sum(t.cur[:r]):sum(t.cur[:r + 1]), h].double().cpu().numpy()
                assert np.all(np.abs(got - want[j]) <= (2.0 ** -8 + 5 * 2.0 ** -24) * np.abs(want[j]))
    assert mk.kv_pool_check_errors(t.gpu) == 0
