"""Shaped chunks over FP8 pages: what the rounding of the weights shares must not reach the rows.

With queries of zeros every weight of a row is the same number, and so is its rounding to fp16 after the rest of the
page's value scale (1 to 2) is folded in: delta, up to 2^-11.  A row's output is then (1 + delta) times the mean of its
values unless its sum holds the rounded weights.  What else is off, sums in fp32 and a reciprocal, is below 2^-20; the
bf16 rounding of an entry is at most 2^-8 of it, of either sign, sqrt(1/3) of that rms."""
import numpy as np
import pytest

import mkv_workloads as wl
import _rope_ref as ref
from test_gpu_shaped import _w
from test_gpu_shaped_chunk import _chunk

pytestmark = pytest.mark.gpu
PAGE = 16


def _filled(d, lens, values):
    """A twin of eight KV heads whose requests hold these values [n][8][d], in FP8 pages."""
    from _harness import Twin
    w = _w(d, 8, 8, len(lens))
    t = Twin(w, n_layers=1, lens=lens, recent=1 << 20)
    k = wl.bf16_round(np.random.default_rng(1).standard_normal((sum(lens), 8, d)).astype(np.float32))
    t.append(lens, layer_kv=(k[None], wl.bf16_round(values.astype(np.float32))[None]))
    return t


def _rows(t, cu, first=None):
    """Means of the values that each row sees."""
    out = []
    for r, n in enumerate(t.cur):
        v = np.stack([t.orc.reconstruct(0, r, h, t.obt, t.otags, n)[1] for h in range(8)], 1)
        c = np.r_[np.zeros((1, *v.shape[1:])), np.cumsum(v, 0)]
        for i in range(cu[r], cu[r + 1]):
            end = n - (cu[r + 1] - i) + 1
            f = 0 if first is None else min(first[i], end - 1)
            out.append((c[end] - c[f]) / (end - f))
    return np.array(out)


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("top", [225, 230])  # over 448, of what power of two ever: delta of 4.2e-4 and -4.1e-4
def test_equal_weights(d, top):
    rng = np.random.default_rng(top + d)
    lens, nq = [5, 33, 70, 300, 901], [2, 3, 2, 4, 3]
    v = rng.uniform(0.25, 0.9, (sum(lens), 8, d)) * top
    at = np.concatenate([np.arange(n) for n in lens])
    v[at % PAGE == 0, :, 0] = top  # every page's largest value
    t = _filled(d, lens, v)
    assert np.all(t.orc.fp8_scale.reshape(-1, 2)[:, 1][t.orc.fp8_scale.reshape(-1, 2)[:, 1] > 0] == np.float32(top) / np.float32(448))
    cu = np.r_[0, np.cumsum(nq)]
    q = np.zeros((cu[-1], 8, d), np.uint16)
    want = _rows(t, cu)
    n = 8 * d * len(lens)  # means that are independent: of a request's last row
    last = cu[1:] - 1
    for kw in ({}, dict(cap=5.0), dict(slopes=np.zeros(8, np.float32))):
        got = _chunk(t, q, cu, kw)
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * (1 + 2.0 ** -8) * np.abs(want))
        g, x = got[last], want[last]
        # (four standard deviations and the rest; a square's share of the sum is at most 1.7 / n here)
        off = (g * x).sum() / (x * x).sum() - 1
        print(f"d {d} top {top} {sorted(kw)}: {off:.2e}", flush=True)
        assert abs(off) <= 4 * 2.0 ** -8 * np.sqrt(1.7 / (3 * n)) + 2.0 ** -20


@pytest.mark.parametrize("d", [128, 256])
def test_pages_without_values_and_scales_of_any_size(d):
    """Zeros in every second page, whose weights count all the same, and scales outside the powers of two that the
    kernel takes from them (2^-15 to 2^7).  A weight is off by 2^-11 there, and below 2^-14 by 2^-25, of a reference
    of 2^3; times the scale's rest that is at least 2^-9 here."""
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(d)
    lens, nq = [40, 200, 777], [7, 40, 33]
    cu = np.r_[0, np.cumsum(nq)]
    q = np.zeros((cu[-1], 8, d), np.uint16)
    at = np.concatenate([np.arange(n) for n in lens])
    for power in (-15, -11, 0, 15):
        v = rng.standard_normal((sum(lens), 8, d)) * 2.0 ** power
        for gaps in (False, True):
            if gaps:
                v[at // PAGE % 2 == 1] = 0.0
            t = _filled(d, lens, v)
            want = _rows(t, cu)
            big = np.abs(v).max()
            for det in (False, True):
                mk.paged_attn_set_deterministic(t.gpu, det)
                for kw in ({}, dict(cap=2.0)):
                    err = np.abs(_chunk(t, q, cu, kw) - want)
                    assert np.all(err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -11 * big)
            assert mk.kv_pool_check_errors(t.gpu) == 0
