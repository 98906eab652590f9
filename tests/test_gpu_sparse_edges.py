"""Page lists and queries at the edges of what sparse attention and page selection take: each
against the plain 64-bit forms of _rope_ref."""
import numpy as np
import pytest

import _rope_ref as ref
import mkv_workloads as wl
import test_gpu_sparse as sp

pytestmark = pytest.mark.gpu
PAGE = 16


def test_negative_entries_are_left_out():
    """Negative entries anywhere in a list are left out, also those above the entry before them; page 0,
    whose table entry stands in for theirs, counts only where it is listed."""
    import paper_2608_23834_amd as mk
    t = sp._twin(sp._w(128, 16, 2, 3), [500, 400, 300])
    t.fill()
    t.migrate()
    rng = np.random.default_rng(22)
    q = wl.bf16_round(rng.standard_normal((3, 16, 128)).astype(np.float32))
    good, cnt = sp._choose(rng, t.cur, 2, 8)
    for r, h, entries, keep in [(0, 0, [-2, -1], []), (1, 1, [0, -5, -3], [0]), (2, 0, [-7, -3, 0, 2], [0, 2]),
                                (0, 1, [-2 ** 31, -2 ** 31 + 1, 5, -4, -1, 6], [5, 6]),
                                (1, 0, [-8, -7, -6, -5, -4, -3, -2, -1], [])]:
        pages, counts = good.copy(), cnt.copy()
        pages[r, h] = -1
        pages[r, h, :len(entries)], counts[r, h] = entries, len(entries)
        kp, kc = good.copy(), cnt.copy()
        kp[r, h] = -1
        kp[r, h, :len(keep)], kc[r, h] = keep, len(keep)
        got = sp._sparse(t, q, pages, counts)
        assert mk.kv_pool_check_errors(t.gpu, clear=True) == mk.DEVERR["RANGE"], entries
        want = ref.attend(t.orc, 0, q, t.obt, t.otags, t.cur, kp, kc)
        if not keep:
            heads = slice(8 * h, 8 * h + 8)
            assert not got[0][r, heads].any() and np.all(got[1][r, heads] == -np.inf), entries
        sp._close(got, want)
