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


@pytest.mark.parametrize("top", [120, 117])
def test_selection_of_queries_that_overflow_fp32(top):
    """A head whose products leave fp32's range both ways (its fp32 sum is a NaN or an infinity, its true
    score is neither) beside one whose scores are finite and spread widely: the choice is the fp64 scores'."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(top)
    pool = mk.Pool(1, 2, 1, 128, 1, 1, 64, np.ones(128, np.int8))
    n = 400
    b = mk.PageBounds(pool, 1, n)
    big = rng.integers(0x78, 0x7F, (n, 2)).astype(np.uint8)  # E4M3 256 .. 448
    codes = np.zeros(b.codes.shape, np.uint8)
    codes[0, 0, 0, :, :, :64] = big[:, None, :1]
    codes[0, 0, 0, :, :, 64:] = 0x80 | big[:, None, 1:]
    b.codes.copy_(sp._gpu(codes))
    b.scales.fill_(1.0)
    q = np.zeros((1, 2, 128), np.float32)
    q[0, 0] = 2.0 ** top
    q[0, 1, :64] = 2.0 ** 112
    q = wl.bf16_round(q)
    vals, sc = sp._values(b)
    score = ref.scores(q, vals[0], sc[0])
    assert np.isfinite(score).all()
    for k, first, last in ((20, 0, 0), (130, 2, 3)):
        want, cnt = ref.select(score, [n * PAGE], k, first, last)
        got, gc = sp._select(pool, b, q, [n * PAGE], k, first, last)
        assert np.array_equal(gc, cnt) and np.array_equal(got, want)


def test_selection_of_zero_scales_and_infinite_queries():
    """Scales of zero with an infinite query entry: a page where that entry meets a zero code, or where
    the product with the scale is inf * 0, has a NaN for a score and comes after the zeros."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(4)
    pool = mk.Pool(1, 2, 1, 128, 1, 1, 64, np.ones(128, np.int8))
    b = sp._random_bounds(rng, pool, 1, 200)
    codes = b.codes.cpu().numpy()
    codes[0, 0, 0, :, :, 7] = np.where(rng.random((200, 1)) < 0.5, 0x00, 0xB8)  # 0 or -1
    b.codes.copy_(sp._gpu(codes))
    b.scales.zero_()
    q = wl.bf16_round(rng.standard_normal((1, 2, 128)).astype(np.float32))
    q[0, 0, 7] = 0x7F80
    vals, sc = sp._values(b)
    score = ref.scores(q, vals[0], sc[0])
    assert np.isnan(score).any() and (score == 0).any()
    want, _ = ref.select(score, [3200], 30, 0, 0)
    got, _ = sp._select(pool, b, q, [3200], 30, 0, 0)
    assert np.array_equal(got, want)
