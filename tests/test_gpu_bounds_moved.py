"""Page bounds whose tensors the caller has replaced, as a batch that was put in another order is."""
import numpy as np
import pytest

import _rope_ref as ref
import mkv_workloads as wl
import test_gpu_sparse as sp

pytestmark = pytest.mark.gpu


def test_bounds_in_another_order():
    """Requests change places: their rows are copied into new tensors, and the update and the
    selection after it work on those; the old ones stay as they were."""
    import paper_2608_23834_amd as mk
    torch = sp._torch()
    t = sp._twin(sp._w(128, 8, 2, 3), [700, 500, 900])
    t.fill()
    b = mk.PageBounds(t.gpu, 3, t.max_pages)
    zero, lens = sp._gpu(np.zeros(3, np.int32)), np.array(t.cur, np.int32)
    mk.kv_page_bounds_update(t.gpu, 0, t.bt, t.tags, zero, sp._gpu(lens), b)
    want, sc = ref.bounds(t.orc.fp8, t.orc.fp8_scale, t.obt, t.cur, 128)
    order = [2, 0, 1]
    was = b.codes, b.scales, b.codes.clone(), b.scales.clone()
    b.codes, b.scales = b.codes[:, order].contiguous(), b.scales[:, order].contiguous()
    bt, tags, lens = t.bt[order].contiguous(), t.tags[order].contiguous(), lens[order]
    b.codes[:, :, :, 0] = 0  # a page of each that the update has to bring back
    frm = sp._gpu(np.zeros(3, np.int32))
    mk.kv_page_bounds_update(t.gpu, 0, bt, tags, frm, sp._gpu(lens), b)
    got, gs = sp._values(b)
    assert np.array_equal(got, want[:, order]) and np.array_equal(gs, sc[:, order])
    q = wl.bf16_round(np.random.default_rng(5).standard_normal((3, 8, 128)).astype(np.float32))
    wp, wc = ref.select(ref.scores(q, want[0, order], sc[0, order]), lens, 9, 1, 2)
    gp, gc = sp._select(t.gpu, b, q, lens, 9, 1, 2)
    assert np.array_equal(gp, wp) and np.array_equal(gc, wc)
    assert torch.equal(was[0], was[2]) and torch.equal(was[1], was[3])
    assert mk.kv_pool_check_errors(t.gpu) == 0
