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
                                 ctrl=torch.zeros(4, dtype=torch.int32))


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
