"""The Python forms of the rotation, selection and sparse-attention calls, on the CPU: what they hand
to the library and what they refuse before it is called.  The library is a recorder here and the
current device the CPU's (-1), so nothing is launched."""
import types

import numpy as np
import pytest
import torch

import paper_2608_23834_amd as mk

H, HQ, D, L = 2, 8, 128, 3


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
