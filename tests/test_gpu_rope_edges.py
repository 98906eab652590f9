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
