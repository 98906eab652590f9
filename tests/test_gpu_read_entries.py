"""Reading back with entries of cu_tokens that fall: always an error, also where no slot leads to the request."""
import numpy as np
import pytest

from test_gpu_read import _i32
from test_gpu_shaped import _twin, _w

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cu", [
    [0, 100, 70, 200],   # the second request's first slot is the third one's
    [0, 100, 50, 200], [0, 100, 99, 200], [0, 250, 240, 200], [0, -5, 100, 200], [0, 300, 200, 200], [0, 200, 0, 200],
])
def test_entries_that_fall(cu):
    import paper_2608_23834_amd as mk
    import torch
    t = _twin(_w(128, 8, 2, 3), [400, 400, 400])

    def read(cu):
        k = torch.full((203, 2, 128), 7, dtype=torch.int16, device="cuda")
        v = torch.full((203, 2, 128), 7, dtype=torch.int16, device="cuda")
        mk.kv_read_tokens(t.gpu, 0, t.bt, t.tags, _i32([0, 3, 90]), _i32(cu), k[:200], v[:200])
        torch.cuda.synchronize()
        return k.cpu().numpy(), v.cpu().numpy()
    want = read([0, 200, 200, 200])
    assert mk.kv_pool_check_errors(t.gpu) == 0
    got = read(cu)
    assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"]
    n = max(0, min(cu[1:]))  # rows that are the first request's alone, where its entries are whole
    for a, b in zip(got, want):
        assert np.all(a[200:] == 7)
        if 0 <= cu[1] <= 200:
            assert np.array_equal(a[:n], b[:n])
    read([0, 100, 100, 200])
    assert mk.kv_pool_check_errors(t.gpu) == 0
