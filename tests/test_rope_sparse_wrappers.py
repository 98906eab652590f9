"""The Python forms of the rotation, selection and sparse-attention calls, on the CPU: what they hand
to the library and what they refuse before it is called.  The library is a recorder here and the
current device the CPU's (-1), so nothing is launched."""
import types

import numpy as np
import pytest
import torch

import paper_2608_23834_amd as mk

H, HQ, D, L = 2, 8, 128, 3
BOUNDS_LAYERS = 1


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name == "kv_page_bounds_bytes":
                n_req, max_pages = args[1:3]
                args[3]._obj.value = BOUNDS_LAYERS * n_req * H * max_pages * 2 * D
                args[4]._obj.value = BOUNDS_LAYERS * n_req * H * max_pages * 4
            else:
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
    return types.SimpleNamespace(handle=1, n_layers=layers, n_q_heads=HQ, n_kv_heads=H, d=D,
                                 device=-1)


def _rope(axes=1):
    return types.SimpleNamespace(handle=2, head_dim=D, rot_dim=64, n_axes=axes, device=-1)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _i16(*shape):
    return torch.zeros(shape, dtype=torch.int16)


def _table(n):
    return dict(block_table=_i32(n, 4), tags=torch.zeros((n, 4), dtype=torch.uint8))


@pytest.mark.parametrize("n", [1, 2, 5])
def test_rows_of_all_layers_out_of_packed_ones(rec, n):
    """[layers][n][H][d] views of packed q/k/v rows, one token among them."""
    packed = _i16(L, n, HQ + 2 * H, D)
    k, v = packed[:, :, HQ:HQ + H], packed[:, :, HQ + H:]
    mk.kv_append_fp8_rope(_pool(L), _rope(), -1, **_table(1), seq_lens_before=_i32(1), cu_new_tokens=_i32(2),
                          positions=None, k=k, v=v)
    (name, a), = rec.calls
    assert name == "kv_append_fp8_rope" and a[9] == n
    assert a[11] == k.data_ptr() and a[13] == v.data_ptr() and a[12] == a[14] == (HQ + 2 * H) * D
    rec.calls.clear()
    wide = _i16(L, n + 1, H, D)  # the layers further apart than the rows
    if n > 1:
        with pytest.raises(ValueError):
            mk.kv_append_fp8_rope(_pool(L), _rope(), -1, **_table(1), seq_lens_before=_i32(1), cu_new_tokens=_i32(2),
                                  positions=None, k=wide[:, :n], v=wide[:, :n])
        assert not rec.calls
    else:  # one row a layer: their distance is the stride
        mk.kv_append_fp8_rope(_pool(L), _rope(), -1, **_table(1), seq_lens_before=_i32(1), cu_new_tokens=_i32(2),
                              positions=None, k=wide[:, :n], v=wide[:, :n])
        assert rec.calls[0][1][12] == 2 * H * D


def _update(b, n=2):
    mk.kv_page_bounds_update(_pool(), 0, **_table(n), seq_lens_from=_i32(n), seq_lens=_i32(n), bounds=b)


def _select(b, n=2, k=3, q=None):
    mk.paged_attn_select_pages(_pool(), 0, _i16(n, HQ, D) if q is None else q, _i32(n), b, 1, 1, _i32(n, H, k),
                               _i32(n, H), torch.zeros(64, dtype=torch.uint8))


def test_bounds_are_the_tensors_they_hold_now(rec):
    """A caller may put other tensors in the place of codes and scales: the calls use those."""
    b = mk.PageBounds(_pool(), 2, 4, device="cpu")
    old = b.codes, b.scales  # (kept, so that no new tensor lies at their addresses)
    for codes, scales in ((b.codes, b.scales), (b.codes.flip(1).contiguous(), b.scales), (b.codes, b.scales.flip(1).contiguous()),
                          (old[0].clone(), old[1].clone())):
        b.codes, b.scales = codes, scales
        rec.calls.clear()
        _update(b)
        _select(b)
        for (_, a), at in zip(rec.calls, (8, 6)):
            assert a[at:at + 4] == (codes.data_ptr(), codes.numel(), scales.data_ptr(), 4 * scales.numel())
    rec.calls.clear()
    for codes, scales in ((old[0].flip(5)[..., ::2], old[1]), (old[0].transpose(1, 2), old[1]), (old[0], old[1].transpose(1, 2)),
                          (old[0], old[1].double()), (old[0].int(), old[1])):
        b.codes, b.scales = codes, scales
        for call in (_update, _select):
            with pytest.raises(ValueError):
                call(b)
    assert not rec.calls
    b.codes, b.scales = old[0][:, :1], old[1][:, :1]  # fewer than the library asks for: it has the true sizes
    _update(b)
    assert rec.calls[0][1][8:12] == (old[0].data_ptr(), old[0].numel() // 2, old[1].data_ptr(), 2 * old[1].numel())


# ---------------------------------------------------------------- what is refused

N, K, MP = 3, 5, 4
BF16, F16, F32, F64, I64, U8 = torch.bfloat16, torch.float16, torch.float32, torch.float64, torch.int64, torch.uint8


def _good(name):
    """(call, its arguments) of a call that is taken."""
    table = _table(N)
    f32 = lambda *s: torch.zeros(s)  # noqa: E731
    ws = torch.zeros(64, dtype=U8)
    if name == "apply":
        return mk.kv_rope_apply, dict(rope=_rope(2), x=_i16(N, HQ, D), positions=_i32(2, N), out=_i16(N, HQ, D))
    if name == "append":
        return mk.kv_append_fp8_rope, dict(pool=_pool(), rope=_rope(2), layer=0, **table, seq_lens_before=_i32(N),
                                           cu_new_tokens=_i32(N + 1), positions=_i32(2, 7), k=_i16(7, H, D), v=_i16(7, H, D))
    if name == "step":
        return mk.paged_attn_decode_append_rope, dict(
            pool=_pool(), rope=_rope(2), layer=0, q=_i16(N, HQ, D), k_new=_i16(N, H, D), v_new=_i16(N, H, D),
            positions=_i32(2, N), **table, seq_lens_before=_i32(N), out=f32(N, HQ, D), lse=f32(N, HQ), ws=ws)
    b = mk.PageBounds(_pool(), N, MP, device="cpu")
    if name == "bounds":
        return mk.kv_page_bounds_update, dict(pool=_pool(), layer=0, **table, seq_lens_from=_i32(N), seq_lens=_i32(N), bounds=b)
    if name == "select":
        return mk.paged_attn_select_pages, dict(pool=_pool(), layer=0, q=_i16(N, HQ, D), seq_lens=_i32(N), bounds=b, n_first=1,
                                                n_last=1, pages=_i32(N, H, K), counts=_i32(N, H), ws=ws)
    return mk.paged_attn_decode_sparse, dict(pool=_pool(), layer=0, q=_i16(N, HQ, D), **table, seq_lens=_i32(N),
                                             pages=_i32(N, H, K), counts=_i32(N, H), out=f32(N, HQ, D), lse=f32(N, HQ), ws=ws)


CALLS = ("apply", "append", "step", "bounds", "select", "sparse")


@pytest.mark.parametrize("name", CALLS)
def test_good_calls_are_taken(rec, name):
    call, a = _good(name)
    call(**a)
    assert len(rec.calls) == 1
    # bf16 tensors are rows as their bits are; more requests' room than there are requests is fine
    more = {"q": _i16(N + 2, HQ, D).view(BF16), "out": torch.zeros(N + 2, HQ, D), "lse": torch.zeros(N + 2, HQ),
            "seq_lens": _i32(N + 2), "seq_lens_before": _i32(N + 2), "seq_lens_from": _i32(N + 2), "cu_new_tokens": _i32(N + 9),
            "k_new": _i16(N, H * D).view(BF16), "v_new": _i16(N * H * D)}
    if name == "apply":
        more = {"x": a["x"].view(BF16), "out": _i16(N, HQ, D).view(torch.uint16)}
    call(**{**a, **{k: v for k, v in more.items() if k in a}})
    if "lse" in a:
        call(**{**a, "lse": None})
    assert len(rec.calls) == (3 if "lse" in a else 2)


def _short(t):
    return t.flatten()[:-1]


@pytest.mark.parametrize("name", CALLS)
def test_wrong_types_are_refused(rec, name):
    """Element types that the kernels would read as others, each argument for itself."""
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
    """Tensors of fewer elements than the kernels read or write."""
    call, good = _good(name)
    for key, t in good.items():
        if not isinstance(t, torch.Tensor) or key in ("ws", "block_table"):
            continue
        with pytest.raises(ValueError):
            call(**{**good, key: _short(t)})
        assert not rec.calls, key


@pytest.mark.parametrize("name", CALLS)
def test_gaps_and_other_cards_are_refused(rec, name, monkeypatch):
    call, good = _good(name)
    for key, t in good.items():
        if not isinstance(t, torch.Tensor) or (name, key) in (("apply", "x"), ("apply", "out")) or key in ("k", "v"):
            continue
        wide = torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype)[..., ::2]
        with pytest.raises(ValueError):
            call(**{**good, key: wide})
        assert not rec.calls, key
    if "pool" in good:  # the pool on another card than the current one
        far = _pool()
        far.device = 1
        with pytest.raises(ValueError):
            call(**{**good, "pool": far})
    monkeypatch.setattr(mk, "_current", lambda: (0, 0))
    with pytest.raises(ValueError):  # (the tensors are not on card 0)
        call(**good)
    assert not rec.calls


@pytest.mark.parametrize("name,heads", [("step", HQ), ("select", HQ), ("sparse", HQ)])
def test_wrong_heads_are_refused(rec, name, heads):
    """Three axes of another head count or head dim than the pool's, also where that is more."""
    call, good = _good(name)
    for key in ("q", "k_new", "v_new", "out"):
        if key in good:
            n, h, d = good[key].shape
            for shape in ((n, 2 * h, d), (n, h, 2 * d), (n, h // 2, 2 * d), (2 * n, h // 2, d)):
                with pytest.raises(ValueError):
                    call(**{**good, key: torch.zeros(shape, dtype=good[key].dtype)})
                assert not rec.calls, (key, shape)


def test_rope_waits_for_the_card_of_its_table(rec, monkeypatch):
    """The table is filled by a copy outside torch's streams: what torch still does to its memory has to
    be over on the table's card, which need not be the current one."""
    waited = []
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: waited.append((device, len(rec.calls))))
    rope = mk.Rope(D, np.ones(32), device="cpu")
    names = [name for name, _ in rec.calls]
    assert names == ["kv_rope_bytes", "kv_rope_create"]
    assert waited == [(rope.table.device, 1)]  # before the second call, for that card
    rope.handle = None
