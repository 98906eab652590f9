"""HeadNorm and Shaping whose tensors got other memory after the object was made, as moving a module's
parameters does: calls use what the tensors hold now, and check it anew.  The library is a recorder here and
the current device the CPU's (-1), so nothing is launched."""
import pytest
import torch

import paper_2608_23834_amd as mk
from test_norm_shape_read_wrappers import D, HQ, H, L, M, N, _good, _i16, _i32, rec  # noqa: F401


def _desc(call, name):
    place = {"rows": 1, "append": 2, "decode": 1, "chunk": 1, "step": 1}[name]
    return call[1][place]._obj


@pytest.mark.parametrize("name,shape", [("rows", (HQ, D)), ("append", (L, H, D))])
def test_weights(rec, name, shape):  # noqa: F811
    call, a = _good(name)
    w = torch.nn.Parameter(torch.zeros(shape, dtype=torch.bfloat16))
    a["norm"] = mk.HeadNorm(D, w)
    call(**a)
    assert _desc(rec.calls[-1], name).weight == w.data_ptr()
    for new in (torch.ones(shape, dtype=torch.bfloat16), torch.ones(D, dtype=torch.bfloat16), torch.ones(shape, dtype=torch.bfloat16)):
        w.data = new
        call(**a)
        d = _desc(rec.calls[-1], name)
        assert d.weight == new.data_ptr() == a["norm"].weight.data_ptr()
        assert (d.head_stride, d.layer_stride) == ((0, 0) if new.dim() == 1 else (D, H * D if new.dim() == 3 else 0))
    n = len(rec.calls)
    for bad in (torch.ones(shape), torch.ones(2 * D, dtype=torch.bfloat16)[::2], torch.ones((7, D), dtype=torch.bfloat16),
                torch.ones(shape, dtype=torch.bfloat16)[..., : D // 2]):
        w.data = bad
        with pytest.raises(ValueError):
            call(**a)
    w.data = torch.ones((*shape[:-2], shape[-2] - 1, D), dtype=torch.bfloat16)  # heads too few
    with pytest.raises(ValueError):
        call(**a)
    assert len(rec.calls) == n


@pytest.mark.parametrize("name", ("decode", "step", "chunk"))
@pytest.mark.parametrize("key", ("slopes", "sinks", "first_keys", "prefix_lens"))
def test_shapings(rec, name, key):  # noqa: F811
    call, a = _good(name)
    need = dict(slopes=HQ, sinks=HQ, first_keys=M if name == "chunk" else N, prefix_lens=N)[key]
    t = torch.ones(HQ) if key in ("slopes", "sinks") else _i32(M)
    a["shaping"] = mk.Shaping(window=5, **{key: t})
    call(**a)
    old = t.data_ptr()
    assert getattr(_desc(rec.calls[-1], name), key) == old
    keep, t.data = t.data, torch.ones(need, dtype=t.dtype)
    call(**a)
    d = _desc(rec.calls[-1], name)
    assert getattr(d, key) == t.data_ptr() != old and d.window == 5 and keep.numel()
    n = len(rec.calls)
    for bad in (torch.ones(need - 1, dtype=t.dtype), torch.ones(2 * need, dtype=t.dtype)[::2], torch.ones(need, dtype=torch.float64)):
        t.data = bad
        with pytest.raises(ValueError):
            call(**a)
    assert len(rec.calls) == n
