"""Refusals of the normed append, shaped attention and the reading back of the cache that need a pool:
nothing is launched, no buffer changes."""
import ctypes

import numpy as np
import pytest

from test_gpu_shaped import _gpu, _rope, _twin, _w

pytestmark = pytest.mark.gpu


def _p(x):
    return ctypes.c_void_p(x.data_ptr()) if hasattr(x, "data_ptr") else x


def _off(t, by):
    return ctypes.c_void_p(t.data_ptr() + by)


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2608_23834_amd as mk
    t = _twin(_w(128, 8, 2, 1), [64], headroom=2)
    ws = mk.workspace(t.gpu, 1, t.max_pages, 4)
    z = lambda *s: torch.zeros(s, dtype=torch.int16, device="cuda")  # noqa: E731
    other = _rope(256, 64)[0]
    bufs = dict(q=z(8, 128), k=z(4, 2, 128), v=z(4, 2, 128), k_new=z(2, 128), v_new=z(2, 128), out=torch.zeros(8, 128, device="cuda"),
                out16=z(4, 8, 128), q4=z(4, 8, 128), seq=_gpu(np.array([64], np.int32)), cu=_gpu(np.array([0, 4], np.int32)), ws=ws,
                shaping=mk.ShapingDesc(), norm=mk.HeadNormDesc(128, 1e-6, 0.0, None, 0, 0), rope=None, other=other)
    return mk, t, bufs


def _calls(env):
    mk, t, b = env
    L = mk.lib()
    ref = lambda d: None if d is None else ctypes.byref(d)  # noqa: E731

    def a(kw, name):
        return _p(kw.get(name, b.get(name)))

    def decode(layer=0, n=1, mp=t.max_pages, wsb=b["ws"].numel(), **kw):
        return L.paged_attn_decode_shaped(t.gpu.handle, ref(kw.get("shaping", b["shaping"])), layer, n, a(kw, "q"), _p(t.bt),
                                          _p(t.tags), mp, a(kw, "seq"), a(kw, "out"), None, a(kw, "ws"), wsb, None)

    def step(layer=0, n=1, mp=t.max_pages, wsb=b["ws"].numel(), **kw):
        norm = ref(kw.get("norm", b["norm"]))
        return L.paged_attn_decode_append_shaped(
            t.gpu.handle, ref(kw.get("shaping", b["shaping"])), kw.get("rope"), norm, norm, layer, n, a(kw, "q"), a(kw, "k_new"),
            a(kw, "v_new"), None, _p(t.bt), _p(t.tags), mp, a(kw, "seq"), a(kw, "out"), None, a(kw, "ws"), wsb, None)

    def chunk(layer=0, n=1, mp=t.max_pages, wsb=b["ws"].numel(), total=4, **kw):
        return L.paged_attn_chunk_shaped(t.gpu.handle, ref(kw.get("shaping", b["shaping"])), layer, n, a(kw, "q4"), a(kw, "cu"),
                                         total, _p(t.bt), _p(t.tags), mp, a(kw, "seq"), a(kw, "out16"), a(kw, "ws"), wsb, None)

    def append(layer=0, n=1, mp=t.max_pages, total=4, ks=256, vs=256, **kw):
        return L.kv_append_fp8_norm_rope(t.gpu.handle, kw.get("rope"), ref(kw.get("norm", b["norm"])), layer, n, _p(t.bt),
                                         _p(t.tags), mp, a(kw, "seq"), a(kw, "cu"), total, None, a(kw, "k"), ks, a(kw, "v"), vs,
                                         None)

    def read(layer=0, n=1, mp=t.max_pages, total=4, ks=256, vs=256, **kw):
        return L.kv_read_tokens(t.gpu.handle, layer, n, _p(t.bt), _p(t.tags), mp, a(kw, "seq"), a(kw, "cu"), total, a(kw, "k"), ks,
                                a(kw, "v"), vs, None)
    return dict(decode=decode, step=step, chunk=chunk, append=append, read=read)


NULLS = dict(decode=("q", "seq", "out", "ws", "shaping"), step=("q", "k_new", "v_new", "seq", "out", "ws", "shaping"),
             chunk=("q4", "cu", "seq", "out16", "ws", "shaping"), append=("seq", "cu", "k", "v", "norm"), read=("seq", "cu"))


@pytest.mark.parametrize("name", sorted(NULLS))
def test_refusals(env, name):
    import torch
    mk, t, b = env
    call = _calls(env)[name]
    before = {k: x.clone() for k, x in b.items() if hasattr(x, "data_ptr")}
    state = t.bt.clone(), t.tags.clone()
    for key in NULLS[name]:
        assert call(**{key: None}) == 1, key
    assert call(n=0) == 1 and call(n=-1) == 1 and call(mp=0) == 1
    assert call(layer=1) == 4 and call(layer=-2) == 4
    if name in ("decode", "step", "chunk"):
        assert call(layer=-1) == 4 and call(n=65536) == 4 and call(mp=(1 << 18) + 1) == 4
        assert call(wsb=16) == 3 and call(wsb=0) == 3
        assert call(ws=_off(b["ws"], 8)) == 1
        q = "q4" if name == "chunk" else "q"
        out = "out16" if name == "chunk" else "out"
        assert call(**{q: _off(b[q], 2)}) == 1 and call(**{out: _off(b[out], 8)}) == 1
        assert call(shaping=mk.ShapingDesc(window=-1)) == 1 and call(shaping=mk.ShapingDesc(cap=-1.0)) == 4
    if name == "step":
        assert call(k_new=_off(b["k_new"], 2)) == 1 and call(v_new=_off(b["v_new"], 4)) == 1
    if name in ("step", "append"):
        assert call(rope=b["other"].handle) == 1  # another head dim
        assert call(norm=mk.HeadNormDesc(256, 1e-6, 0.0, None, 0, 0)) == 1 and call(norm=mk.HeadNormDesc(128, 0.0, 0.0, None, 0, 0)) == 4
    if name == "chunk":
        assert call(total=0) == 1 and call(total=-3) == 1 and call(total=1 << 29) == 4
    if name in ("append", "read"):
        assert call(total=-1) == 1
        for s in ("ks", "vs"):
            assert call(**{s: 252}) == 1 and call(**{s: 258}) == 1 and call(**{s: (1 << 31) + 4}) == 4
        for key in ("k", "v"):
            assert call(**{key: _off(b[key], 2)}) == 1
        if name == "append":
            assert call(ks=(1 << 26) + 4) == 4
        else:
            assert call(v=b["k"]) == 1 and call(k=None, v=None) == 1 and call(mp=(1 << 18) + 1) == 4
            assert call(total=0, k=None, v=None) == 0
    torch.cuda.synchronize()
    for k, x in before.items():
        assert torch.equal(b[k], x), k
    assert torch.equal(t.bt, state[0]) and torch.equal(t.tags, state[1]) and mk.kv_pool_check_errors(t.gpu) == 0
    assert call() == 0
    torch.cuda.synchronize()
    mk.kv_pool_check_errors(t.gpu, clear=True)
