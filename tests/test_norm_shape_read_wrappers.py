"""The Python forms of the normed rotation and append, shaped attention and the reading back of the
cache, on the CPU: what they hand to the library and what they refuse before it is called.  The library
is a recorder here and the current device the CPU's (-1), so nothing is launched."""
import ctypes
import types

import pytest
import torch

import paper_2608_23834_amd as mk

H, HQ, D, L, N, M = 2, 8, 128, 3, 3, 7
BF16, F16, F32, F64, I64, U8 = torch.bfloat16, torch.float16, torch.float32, torch.float64, torch.int64, torch.uint8


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def rec(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(mk, "lib", lambda: r)
    monkeypatch.setattr(mk, "_current", lambda: (-1, 0))
    return r


def _pool(layers=1):
    return types.SimpleNamespace(handle=1, n_layers=layers, n_q_heads=HQ, n_kv_heads=H, d=D, device=-1)


def _rope(axes=2):
    return types.SimpleNamespace(handle=2, head_dim=D, rot_dim=64, n_axes=axes, device=-1)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _i16(*shape):
    return torch.zeros(shape, dtype=torch.int16)


def _good(name):
    """(call, its arguments) of a call that is taken."""
    table = dict(block_table=_i32(N, 4), tags=torch.zeros((N, 4), dtype=U8))
    ws = torch.zeros(64, dtype=U8)
    sh = mk.Shaping(scale=0.5, cap=20.0, window=9, slopes=torch.ones(HQ), sinks=torch.ones(HQ), first_keys=_i32(M),
                    prefix_lens=_i32(N))
    if name == "rows":
        return mk.kv_norm_rope_apply, dict(rope=_rope(), norm=mk.HeadNorm(D, _i16(HQ, D)), x=_i16(N, HQ, D),
                                           positions=_i32(2, N), out=_i16(N, HQ, D))
    if name == "append":
        return mk.kv_append_fp8_norm_rope, dict(
            pool=_pool(L), rope=_rope(), norm=mk.HeadNorm(D, _i16(L, H, D)), layer=-1, **table, seq_lens_before=_i32(N),
            cu_new_tokens=_i32(N + 1), positions=_i32(2, M), k=_i16(L, M, H, D), v=_i16(L, M, H, D))
    if name == "decode":
        return mk.paged_attn_decode_shaped, dict(pool=_pool(), shaping=sh, layer=0, q=_i16(N, HQ, D), **table,
                                                 seq_lens=_i32(N), out=torch.zeros(N, HQ, D), lse=torch.zeros(N, HQ), ws=ws)
    if name == "step":
        return mk.paged_attn_decode_append_shaped, dict(
            pool=_pool(), shaping=sh, rope=_rope(), q_norm=mk.HeadNorm(D, _i16(HQ, D)), k_norm=mk.HeadNorm(D, _i16(D)),
            layer=0, q=_i16(N, HQ, D), k_new=_i16(N, H, D), v_new=_i16(N, H, D), positions=_i32(2, N), **table,
            seq_lens_before=_i32(N), out=torch.zeros(N, HQ, D), lse=torch.zeros(N, HQ), ws=ws)
    if name == "chunk":
        return mk.paged_attn_chunk_shaped, dict(pool=_pool(), shaping=sh, layer=0, q=_i16(M, HQ, D), cu_q=_i32(N + 1),
                                                **table, seq_lens=_i32(N), out=_i16(M, HQ, D), ws=ws)
    return mk.kv_read_tokens, dict(pool=_pool(L), layer=-1, **table, seq_from=_i32(N), cu_tokens=_i32(N + 1),
                                   k=_i16(L, M, H, D), v=_i16(L, M, H, D))


CALLS = ("rows", "append", "decode", "step", "chunk", "read")
STRIDED = {("rows", "x"), ("rows", "out"), ("append", "k"), ("append", "v"), ("read", "k"), ("read", "v")}


@pytest.mark.parametrize("name", CALLS)
def test_good_calls_are_taken(rec, name):
    call, a = _good(name)
    call(**a)
    # bf16 tensors are rows as their bits are; more requests' room than there are requests is fine
    more = {"q": _i16(*a["q"].shape).view(BF16)} if "q" in a else {}
    for key in ("seq_lens", "seq_lens_before", "seq_from"):
        if key in a:
            more[key] = _i32(N + 2)
    for key in ("cu_new_tokens", "cu_tokens", "cu_q"):
        if key in a:
            more[key] = _i32(N + 9)
    for key in ("x", "k", "v"):
        if key in a:
            more[key] = a[key].view(BF16)
    call(**{**a, **more})
    for key in ("lse", "rope", "q_norm", "k_norm"):
        if key in a:
            call(**{**a, key: None})
    if name in ("rows", "append", "step"):  # without a rope positions are not looked at
        call(**{**a, "rope": None, "positions": None})
    if name == "read":
        call(**{**a, "k": None})
        call(**{**a, "v": None})
        with pytest.raises(ValueError):
            call(**{**a, "k": None, "v": None})
    for got, args in rec.calls:
        assert got == call.__name__ and (name == "rows" or args[0] == 1)


def test_what_the_library_gets(rec):
    """Rows out of packed ones, one layer's and all layers'; the descriptions of norms and shapings."""
    packed = _i16(L, M, HQ + 2 * H, D)
    call, a = _good("append")
    call(**{**a, "k": packed[:, :, HQ:HQ + H], "v": packed[:, :, HQ + H:], "rope": None})
    (_, g), = rec.calls
    assert g[1] is None and g[11] is None and g[10] == M and g[3] == -1 and g[4] == N
    assert g[12] == packed[:, :, HQ:].data_ptr() and g[13] == g[15] == (HQ + 2 * H) * D
    d = g[2]._obj
    w = a["norm"].weight
    assert (d.head_dim, d.weight, d.head_stride, d.layer_stride, d.add) == (D, w.data_ptr(), D, H * D, 0.0)
    rec.calls.clear()
    call, a = _good("read")
    call(**{**a, "layer": 2, "k": packed[1, :, :H], "v": packed[0, :, H:2 * H]})
    (_, g), = rec.calls
    assert g[1] == 2 and g[8] == M and g[9] == packed[1].data_ptr() and g[11] == packed[0, :, H:].data_ptr()
    assert g[10] == g[12] == (HQ + 2 * H) * D
    rec.calls.clear()
    call, a = _good("chunk")
    call(**a)
    (_, g), = rec.calls
    d, sh = g[1]._obj, a["shaping"]
    assert (d.scale, d.cap, d.window) == (0.5, 20.0, 9) and g[6] == M
    assert (d.slopes, d.sinks, d.first_keys, d.prefix_lens) == tuple(
        t.data_ptr() for t in (sh.slopes, sh.sinks, sh.first_keys, sh.prefix_lens))


def test_descriptions():
    one = mk.HeadNorm(D, unit_offset=True)._desc
    assert one.weight is None and one.add == 1.0 and one.head_stride == one.layer_stride == 0
    assert mk.HeadNorm(D, _i16(D))._desc.head_stride == 0
    for bad in (_i16(D + 1), _i16(D, 2)[:, 0], torch.zeros(D), torch.zeros(D, dtype=F16), _i16(1, 1, 1, D), _i16(2 * D)[::2],
                _i16()):
        with pytest.raises(ValueError):
            mk.HeadNorm(D, bad)
    for bad in (dict(slopes=torch.ones(HQ, dtype=F64)), dict(sinks=torch.ones(HQ, dtype=BF16)), dict(first_keys=torch.zeros(4, dtype=I64)),
                dict(prefix_lens=torch.zeros(4)), dict(slopes=torch.ones(2 * HQ)[::2])):
        with pytest.raises(ValueError):
            mk.Shaping(**bad)
    for cls, obj in ((mk.HeadNorm, mk.HeadNorm(D, _i16(D))), (mk.Shaping, mk.Shaping(sinks=torch.ones(3)))):
        for name in ("weight",) if cls is mk.HeadNorm else ("slopes", "sinks", "first_keys", "prefix_lens"):
            with pytest.raises(AttributeError):  # the library's description would not follow
                setattr(obj, name, None)
    assert ctypes.sizeof(mk.HeadNormDesc) == 48 and ctypes.sizeof(mk.ShapingDesc) == 48


@pytest.mark.parametrize("name,key,bad", [
    ("rows", "norm", (H, D)), ("rows", "norm", (1, H, D)), ("rows", "norm", (2, HQ, D)), ("append", "norm", (HQ, D)),
    ("append", "norm", (1, H, D)), ("step", "q_norm", (H, D)), ("step", "k_norm", (HQ, D)), ("step", "k_norm", (2, H, D)),
])
def test_norms_of_other_heads_are_refused(rec, name, key, bad):
    call, a = _good(name)
    with pytest.raises(ValueError):
        call(**{**a, key: mk.HeadNorm(D, _i16(*bad))})
    assert not rec.calls


@pytest.mark.parametrize("name", ("decode", "step", "chunk"))
def test_shapings_of_fewer_rows_are_refused(rec, name):
    call, a = _good(name)
    rows = M if name == "chunk" else N
    for kw in (dict(slopes=torch.ones(HQ - 1)), dict(sinks=torch.ones(H)), dict(first_keys=_i32(rows - 1)),
               dict(prefix_lens=_i32(N - 1))):
        with pytest.raises(ValueError):
            call(**{**a, "shaping": mk.Shaping(**kw)})
    assert not rec.calls


def _short(t):
    return t.flatten()[:-1]


@pytest.mark.parametrize("name", CALLS)
def test_wrong_types_are_refused(rec, name):
    call, good = _good(name)
    for key, t in good.items():
        if not isinstance(t, torch.Tensor) or key == "ws":
            continue
        bad = {torch.int16: (F32, F16, U8, torch.int32), torch.int32: (F32, I64, torch.int16), U8: (torch.int32, torch.int16),
               F32: (F64, F16, torch.int32)}[t.dtype]
        for dtype in bad:
            with pytest.raises(ValueError):
                call(**{**good, key: t.to(dtype)})
            assert not rec.calls, (key, dtype)


@pytest.mark.parametrize("name", CALLS)
def test_short_tensors_are_refused(rec, name):
    call, good = _good(name)
    for key, t in good.items():
        if not isinstance(t, torch.Tensor) or key in ("ws", "block_table"):
            continue
        with pytest.raises((ValueError, IndexError)):
            call(**{**good, key: _short(t)})
        assert not rec.calls, key


@pytest.mark.parametrize("name", CALLS)
def test_other_heads_are_refused(rec, name):
    call, good = _good(name)
    for key in ("q", "k_new", "v_new", "out", "x", "k", "v"):
        if key in good:
            *n, h, d = good[key].shape
            for shape in ((*n, 2 * h, d), (*n, h, 2 * d), (*n, h // 2, 2 * d)):
                with pytest.raises(ValueError):
                    call(**{**good, key: torch.zeros(shape, dtype=good[key].dtype)})
                assert not rec.calls, (key, shape)


@pytest.mark.parametrize("name", CALLS)
def test_gaps_and_other_cards_are_refused(rec, name, monkeypatch):
    call, good = _good(name)
    for key, t in good.items():
        if not isinstance(t, torch.Tensor):
            continue
        wide = torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype)[..., ::2]
        with pytest.raises(ValueError):
            call(**{**good, key: wide})
        if (name, key) in STRIDED and t.dim() == 4:  # rows of a layer that do not follow the last layer's
            with pytest.raises(ValueError):
                call(**{**good, key: torch.zeros((L, M + 1, H, D), dtype=t.dtype)[:, :M]})
        assert not rec.calls, key
    if "pool" in good:
        far = _pool(good["pool"].n_layers)
        far.device = 1
        with pytest.raises(ValueError):
            call(**{**good, "pool": far})
    if good.get("rope"):
        far = _rope()
        far.device = 1
        with pytest.raises(ValueError):
            call(**{**good, "rope": far})
    monkeypatch.setattr(mk, "_current", lambda: (0, 0))
    with pytest.raises(ValueError):  # (the tensors are not on card 0)
        call(**good)
    assert not rec.calls
