"""kv_read_tokens against the CPU oracle's reconstruction of the pages in 64 bits.

A value is evaluated in fp32 and rounded to bf16 once: the FP8 product and the TQ3 value are one
fp32 rounding each, a TQ3 key three (gamma / sqrt d, the constant 1 / sqrt d, the product with the
exact sum), each 2^-24 of it; then half a bf16 step, 2^-8 of it; one fp32 rounding more where the
oracle holds fp32."""
import dataclasses

import numpy as np
import pytest

import _rope_ref as ref
import mkv_workloads as wl

pytestmark = pytest.mark.gpu
PAGE = 16
REL = 2.0 ** -8 + 5 * 2.0 ** -24


def _torch():
    import torch
    return torch


def _gpu(a):
    return _torch().from_numpy(np.ascontiguousarray(a)).cuda()


def _i32(v):
    return _gpu(np.asarray(v, np.int32))


def _w(d, hq, hkv, n_req, layers=1):
    return dataclasses.replace(wl.scaled(wl.workload(2), (16,) * n_req, layers), head_dim=d, n_q_heads=hq, n_kv_heads=hkv)


def _twin(w, lens, layers=1, recent=64):
    from _harness import Twin
    t = Twin(w, n_layers=layers, lens=lens, recent=recent)
    t.fill()
    t.migrate()
    return t


def _want(t, layers, frm, n):
    """K and V [layers][sum n][H][d] in 64 bits."""
    H, d = t.w.n_kv_heads, t.w.head_dim
    out = np.zeros((2, len(layers), sum(n), H, d))
    at = 0
    for r in range(t.n_req):
        if n[r]:
            for i, layer in enumerate(layers):
                for h in range(H):
                    kv = t.orc.reconstruct(layer, r, h, t.obt, t.otags, t.cur[r])
                    for j in range(2):
                        out[j, i, at:at + n[r], h] = kv[j][frm[r]:frm[r] + n[r]]
        at += n[r]
    return out


def _near(got, want):
    got = ref.bf16_f64(got.cpu().numpy())
    err = np.abs(got - want) - REL * np.abs(want)
    assert err.max(initial=-1.0) <= 0.0, (np.argwhere(err > 0)[:4], err.max())


LENS = [1, 16, 17, 700, 2003, 333]


@pytest.mark.parametrize("d,hq,hkv", [(256, 24, 4), (128, 8, 1), (128, 32, 8), (256, 6, 3)])
def test_reads_what_attention_reads(d, hq, hkv):
    import paper_2608_23834_amd as mk
    torch = _torch()
    t = _twin(_w(d, hq, hkv, len(LENS), 2), LENS, 2)
    assert (t.otags == 2).any() and (t.otags == 1).any() and (t.otags == 0).any()
    frm, n = [0, 3, 0, 5, 1990, 48], [1, 13, 17, 690, 0, 16]
    for frm, n in ((frm, n), ([0] * 6, LENS), ([0, 15, 16, 699, 1024, 333], [0, 1, 1, 1, 979, 0])):
        want = _want(t, (0, 1), frm, n)
        cu = _i32(np.r_[0, np.cumsum(n)])
        tot = sum(n)
        # all layers, contiguous
        k = torch.full((2, tot, hkv, d), 7, dtype=torch.int16, device="cuda")
        v = torch.full_like(k, 7)
        mk.kv_read_tokens(t.gpu, -1, t.bt, t.tags, _i32(frm), cu, k, v)
        _near(k, want[0])
        _near(v, want[1])
        # one layer into packed rows, the memory between them as it was; one of the two alone
        packed = torch.full((tot, hq + 2 * hkv, d), 7, dtype=torch.int16, device="cuda")
        kk, vv = packed[:, hq:hq + hkv], packed[:, hq + hkv:]
        mk.kv_read_tokens(t.gpu, 1, t.bt, t.tags, _i32(frm), cu, None, vv)
        assert bool((packed[:, :hq + hkv] == 7).all())
        mk.kv_read_tokens(t.gpu, 1, t.bt, t.tags, _i32(frm), cu, kk, None)
        assert bool((packed[:, :hq] == 7).all())
        assert torch.equal(kk, k[1]) and torch.equal(vv, v[1])
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_many_requests():
    import paper_2608_23834_amd as mk
    torch = _torch()
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 90, 2100)]
    lens[0], lens[63], lens[64], lens[1024], lens[2099] = 0, 300, 1, 0, 129
    t = _twin(_w(128, 8, 1, len(lens)), lens, recent=16)
    frm = [int(rng.integers(0, x + 1)) for x in lens]
    n = [x - f for x, f in zip(lens, frm)]
    k = torch.zeros((sum(n), 1, 128), dtype=torch.int16, device="cuda")
    v = torch.zeros_like(k)
    mk.kv_read_tokens(t.gpu, 0, t.bt, t.tags, _i32(frm), _i32(np.r_[0, np.cumsum(n)]), k, v)
    want = _want(t, (0,), frm, n)
    _near(k, want[0, 0])
    _near(v, want[1, 0])
    assert mk.kv_pool_check_errors(t.gpu) == 0


def test_pages_and_ranges_that_are_not_there():
    import paper_2608_23834_amd as mk
    torch = _torch()
    t = _twin(_w(256, 8, 2, 5), [400] * 5)
    bt, tags = t.bt.clone(), t.tags.clone()
    bt[0, 3], tags[0, 5], bt[1, 20], bt[2, 1] = t.n_fp8 + t.n_tq3, 0xFF, -1, -7
    frm, n = [0, 300, 10, -1, 16 * t.max_pages - 3], [100, 100, 50, 20, 4]
    cu = np.r_[0, np.cumsum(n)]
    want = np.zeros((2, cu[-1], 2, 256))
    for r in range(3):
        for h in range(2):
            kv = t.orc.reconstruct(0, r, h, t.obt, t.otags, 400)
            for j in range(2):
                want[j, cu[r]:cu[r + 1], h] = kv[j][frm[r]:frm[r] + n[r]]
    for r, p in ((0, 3), (0, 5), (1, 20), (2, 1)):
        a = np.arange(p * PAGE, (p + 1) * PAGE)
        a = a[(a >= frm[r]) & (a < frm[r] + n[r])]
        want[:, cu[r] + a - frm[r]] = 0.0
    k = torch.full((cu[-1] + 3, 2, 256), 7, dtype=torch.int16, device="cuda")
    v = torch.full_like(k, 7)
    mk.kv_read_tokens(t.gpu, 0, bt, tags, _i32(frm), _i32(cu), k[:-3], v[:-3])
    _near(k[:-3], want[0])
    _near(v[:-3], want[1])
    assert bool((k[-3:] == 7).all()) and bool((v[-3:] == 7).all())
    assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["BAD_TAG"] | mk.DEVERR["RANGE"]
    # row offsets that are not this call's: nothing is written
    k.fill_(7)
    for bad in (cu + 1, np.r_[cu[:-1], cu[-1] - 1]):
        mk.kv_read_tokens(t.gpu, 0, bt, tags, _i32(frm), _i32(bad), k[:-3], None)
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]
    assert bool((k == 7).all())
    # offsets that fall: the request whose rows cannot be is left out, no row outside is written
    bad = cu.copy()
    bad[2] = cu[-1] + 5
    mk.kv_read_tokens(t.gpu, 0, bt, tags, _i32([0] * 5), _i32(bad), k[:-3], None)
    assert mk.kv_pool_check_errors(t.gpu, clear=True) & mk.DEVERR["RANGE"]
    assert bool((k[-3:] == 7).all())


def test_rows_past_32_bits():
    """2^31 elements of keys and more: one physical page behind every table entry."""
    import paper_2608_23834_amd as mk
    torch = _torch()
    H, d, pages = 4, 256, (1 << 21) // PAGE + 5
    t = _twin(_w(d, 24, H, 1), [128], recent=16)
    ids = t.bt[0, : 8].clone()
    bt = ids.repeat(pages // 8 + 1)[None, :pages].contiguous()
    tags = t.tags[0, :8].repeat(pages // 8 + 1)[None, :pages].contiguous()
    n = pages * PAGE
    k = torch.zeros((n, H, d), dtype=torch.int16, device="cuda")
    mk.kv_read_tokens(t.gpu, 0, bt, tags, _i32([0]), _i32([0, n]), k, None)
    assert mk.kv_pool_check_errors(t.gpu) == 0
    want = _want(t, (0,), [0], [128])[0, 0]
    _near(k[:128], want)
    whole = pages // 8
    assert k.numel() > 1 << 31
    assert bool((k[: whole * 128].view(whole, 128 * H * d) == k[:128].view(-1)).all())
    assert torch.equal(k[whole * 128:], k[: n - whole * 128])


def test_on_a_stream_and_in_a_graph():
    import paper_2608_23834_amd as mk
    torch = _torch()
    t = _twin(_w(128, 8, 2, 3), [100, 300, 40])
    frm, cu = _i32([0, 200, 7]), _i32([0, 100, 200, 233])
    k = torch.zeros((233, 2, 128), dtype=torch.int16, device="cuda")
    v = torch.zeros_like(k)

    def call(stream=None):
        mk.kv_read_tokens(t.gpu, 0, t.bt, t.tags, frm, cu, k, v, stream)
    call()
    want = k.clone(), v.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    k.zero_()
    torch.cuda.synchronize()
    call(s)
    torch.cuda.synchronize()
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for start in (0, 50):  # the ranges are read when the graph runs
        frm[1] = start
        call()
        want = k.clone(), v.clone()
        k.zero_()
        v.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    assert mk.kv_pool_check_errors(t.gpu) == 0
