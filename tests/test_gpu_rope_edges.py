"""Rotated appends at the edges of what they take: layouts of their rows and scales of their pages."""
import numpy as np
import pytest

import mkv_workloads as wl
import test_gpu_rope as rp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 3])
def test_append_of_all_layers_out_of_packed_rows(n):
    """K and V of every layer as views of packed q/k/v rows, down to one token a layer."""
    import paper_2608_23834_amd as mk
    torch = rp._torch()
    w = rp._w(128, 8, 2, 1, 3)
    rng = np.random.default_rng(n)
    rope, _, _ = rp._rope(128, 64)
    packed = rp._i16(rp._bits(rng, 3, n, 12, 128))
    k, v = packed[:, :, 8:10], packed[:, :, 10:]
    cu, zero = rp._gpu(np.array([0, n], np.int32)), rp._gpu(np.zeros(1, np.int32))
    pages = []
    for x, y in ((k, v), (k.contiguous(), v.contiguous())):
        t = rp._twin(w, [32], 3)
        mk.kv_append_fp8_rope(t.gpu, rope, -1, t.bt, t.tags, zero, cu, None, x, y)
        torch.cuda.synchronize()
        assert mk.kv_pool_check_errors(t.gpu) == 0
        pages.append((t.bt, t.gpu.fp8, t.gpu.fp8_scales.view(torch.int32)))
    assert all(torch.equal(x, y) for x, y in zip(*pages))
    assert pages[0][1].any()


@pytest.mark.parametrize("kind", ["prompt", "step", "decode"])
def test_scales_are_quotients(kind):
    """Largest values of every bf16 mantissa: a page's scale is the largest value divided by 448, which for
    71 of the 128 is not its product with the rounded 1 / 448, and its codes follow from that scale: the
    oracle's bytes, from a prompt's append, the appends of single tokens and the decode step."""
    import paper_2608_23834_amd as mk
    torch = rp._torch()
    n, d, H = 128, 128, 2
    top = ((128 + np.arange(n)) / 128 * 2.0 ** (np.arange(n) % 7 - 3)).astype(np.float32)
    assert (top / np.float32(448) != top * (np.float32(1) / np.float32(448))).sum() == 71
    w = rp._w(d, 2 * H, H, n)
    rng = np.random.default_rng(9)
    rope, _, _ = rp._rope(d, 64)
    c = 16 if kind == "prompt" else 1
    K, V = (wl.bf16_round((rng.uniform(-1, 1, (n, c, H, d)) * top[:, None, None, None]).astype(np.float32)) for _ in range(2))
    for x in (K, V):
        x[:, c // 2, :, 5] = wl.bf16_round(top)[:, None]
    K, V = K.reshape(n * c, H, d), V.reshape(n * c, H, d)
    t = rp._twin(w, [16] * n, 1)
    pos = torch.zeros((1, n * c), dtype=torch.int32, device="cuda")  # (no rotation: the largest values stay)
    zero, cu = np.zeros(n, np.int32), (c * np.arange(n + 1)).astype(np.int32)
    if kind == "decode":
        out, lse = torch.zeros((n, 2 * H, d), device="cuda"), torch.zeros((n, 2 * H), device="cuda")
        mk.paged_attn_decode_append_rope(t.gpu, rope, 0, rp._i16(rp._bits(rng, n, 2 * H, d)), rp._i16(K), rp._i16(V), pos, t.bt,
                                         t.tags, rp._gpu(zero), out, lse, t._ws(None))
    else:
        mk.kv_append_fp8_rope(t.gpu, rope, 0, t.bt, t.tags, rp._gpu(zero), rp._gpu(cu), pos, rp._i16(K), rp._i16(V))
    assert t.orc.append(0, t.obt, t.otags, zero, cu, K[None], V[None]) == 0
    torch.cuda.synchronize()
    t.check_tables()
    t.check_pages()
    got = t.gpu.fp8_scales_view()[0, t.bt[:, 0].long()].cpu().numpy()
    assert np.array_equal(got, np.broadcast_to((top / np.float32(448))[:, None, None], got.shape))
