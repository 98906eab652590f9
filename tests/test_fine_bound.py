"""What the error bound of the rotating step and of sparse attention can tell apart, on the CPU: over
pages of both formats every form with a part held in fewer bits leaves it, the form as it is does not."""
import dataclasses

import numpy as np
import pytest

import _fine_ref as fr
import mkv_workloads as wl


def _pages(d, hq, hkv, n, recent, k, v, sigma):
    import oracle
    pg = (n + 15) // 16
    orc = oracle.Pool(1, hq, hkv, d, pg + 4, pg + 4, recent, sigma, None, None)
    bt, tags = np.full((1, pg), -1, np.int32), np.full((1, pg), 0xFF, np.uint8)
    assert orc.append(0, bt, tags, np.zeros(1, np.int32), np.array([0, n], np.int32), k[None], v[None]) == 0
    orc.migrate(bt, tags, np.zeros((1, pg), np.uint8), np.array([n], np.int32))
    return orc, bt, tags


@pytest.mark.parametrize("d,hq,hkv,n", [(256, 8, 2, 1200), (128, 8, 1, 500), (256, 6, 1, 90), (128, 4, 4, 110)])
def test_fewer_bits_leave_the_bound(d, hq, hkv, n):
    w = dataclasses.replace(wl.scaled(wl.workload(2), (16,), 1), head_dim=d, n_q_heads=hq, n_kv_heads=hkv)
    sigma = wl.rot_signs(w)
    orc, bt, tags = _pages(d, hq, hkv, n, 64, *wl.kv_layer(w, 0, n), sigma)
    assert (tags == 2).any() and (tags == 0).any()
    q = wl.bf16_round(np.random.default_rng(n).standard_normal((1, hq, d)).astype(np.float32))
    worst = {}
    for _, _, k, v, x, at in fr.rows(orc, 0, q, bt, tags, [n]):
        b, _ = fr.bound(k, v, x, at)
        o = fr.attend(k, v, x)[2]
        assert b <= 1e-5 * np.linalg.norm(o)
        for name, y in fr.forms(k, v, x, sigma.astype(np.float64)).items():
            worst[name] = max(worst.get(name, 0.0), np.linalg.norm(y - o) / b)
    assert worst.pop("pairs") < 0.1
    worst.pop("weights against the largest")  # (these weights are too even for it to show)
    assert min(worst.values()) > 1.5, worst


def test_weights_against_the_largest_leave_the_bound():
    k, v, q = fr.few_large()
    one = np.ones(fr.FEW_D, np.int8)
    orc, bt, tags = _pages(fr.FEW_D, 1, 1, fr.FEW_TOKENS, 4096, k[:, None], v[:, None], one)
    (_, _, kk, vv, x, at), = fr.rows(orc, 0, q[None, None], bt, tags, [fr.FEW_TOKENS])
    o = fr.attend(kk, vv, x)[2]
    b = fr.FEW_BOUND * np.linalg.norm(o)
    off = {name: np.linalg.norm(y - o) / b for name, y in fr.forms(kk, vv, x, one.astype(np.float64)).items()}
    assert off["pairs"] < 0.1 and off["weights against the largest"] > 1.3 and off["weights once"] > 1.3, off


def test_pair_and_terms():
    x = np.float64(1 + 2.0 ** -10 + 2.0 ** -20)
    assert fr.fp16(x) == 1 + 2.0 ** -10 and fr.pair(x) == x
    assert abs(fr.e4m3_terms(np.array([300.7]), 3)[0] - 300.7) <= 300.7 * 2.0 ** -12
    # a rotation of everything by exact parts changes nothing
    q = np.random.default_rng(1).standard_normal(128)
    assert np.allclose(fr.rotated_query(q, np.ones(128), lambda y: y), q, rtol=0, atol=1e-14)
