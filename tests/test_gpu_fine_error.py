"""The rotating decode step and sparse attention answer with fp32's error: every query's output and lse
against 64 bits within a bound that a query or weights of fewer bits leave (test_fine_bound.py)."""
import numpy as np
import pytest

import _fine_ref as fr
import _rope_ref as ref
import mkv_workloads as wl
import test_gpu_rope as rp
import test_gpu_sparse as sp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,hkv", [(256, 24, 4), (256, 16, 2), (256, 32, 2), (128, 32, 8), (128, 24, 4), (128, 16, 1)])
def test_sparse_error(d, hq, hkv):
    import paper_2608_23834_amd as mk
    t = sp._twin(sp._w(d, hq, hkv, 4), [2100, 333, 64, 17])
    t.fill()
    t.migrate()
    rng = np.random.default_rng(d + hq + 1)
    q = wl.bf16_round(rng.standard_normal((4, hq, d)).astype(np.float32))
    for k in (20, 132):
        pages, counts = sp._choose(rng, t.cur, hkv, k)
        got = sp._sparse(t, q, pages, counts)
        worst = fr.check(*got, t.orc, 0, q, t.obt, t.otags, t.cur, pages, counts)
        print(f"  d={d} {hq}/{hkv} k={k}: {worst[0]:.2f} and {worst[1]:.2f} of the bounds", flush=True)
        assert max(worst) <= 1
    assert mk.kv_pool_check_errors(t.gpu) == 0


@pytest.mark.parametrize("d,hq,hkv,rot", [(256, 24, 4, 64), (256, 16, 2, 256), (256, 32, 2, 128), (128, 32, 8, 128), (128, 16, 1, 20)])
def test_step_error(d, hq, hkv, rot):
    import paper_2608_23834_amd as mk
    torch = rp._torch()
    w = rp._w(d, hq, hkv, 4)
    rng = np.random.default_rng(d + hq + rot + 1)
    rope, freq, axis = rp._rope(d, rot, 2, base=1e6)
    t = rp._twin(w, [2100, 333, 64, 17], 1)
    rp._append(t, (rope, freq, axis, False), [2080, 319, 47, 0], rng)
    t.migrate()
    K, V, q = (rp._bits(rng, 4, h, d) for h in (hkv, hkv, hq))
    sb, pos = np.array(t.cur, np.int32), rng.integers(0, 100000, (2, 4)).astype(np.int32)
    out, lse = torch.zeros((4, hq, d), device="cuda"), torch.zeros((4, hq), device="cuda")
    mk.paged_attn_decode_append_rope(t.gpu, rope, 0, rp._i16(q), rp._i16(K), rp._i16(V), rp._gpu(pos), t.bt, t.tags,
                                     rp._gpu(sb), out, lse, t._ws(None))
    torch.cuda.synchronize()
    Kr, qr = ref.rotate(K, pos, freq, axis, False), ref.rotate(q, pos, freq, axis, False)
    assert t.orc.append(0, t.obt, t.otags, sb, np.arange(5, dtype=np.int32), Kr[None], V[None]) == 0
    t.cur = [c + 1 for c in t.cur]
    t.check_tables()
    t.check_pages()
    worst = fr.check(out.cpu().numpy(), lse.cpu().numpy(), t.orc, 0, qr, t.obt, t.otags, t.cur)
    print(f"  d={d} {hq}/{hkv} rot={rot}: {worst[0]:.2f} and {worst[1]:.2f} of the bounds", flush=True)
    assert max(worst) <= 1


def test_small_weights_beside_large_ones():
    """Thousands of equal weights of 2^-11 of the first ones that a wave meets: 64 requests over the same
    pages, so that one workgroup takes all pages of a (request, head) and each of its waves 25 of them."""
    import paper_2608_23834_amd as mk
    torch = sp._torch()
    n, d, H, n_req = fr.FEW_TOKENS, fr.FEW_D, 8, 64
    k, v, q = (np.repeat(x[..., None, :], H, -2) for x in fr.few_large())
    t = sp._twin(sp._w(d, H, H, 1), [n], recent=4096)
    t.append([n], (np.ascontiguousarray(k), np.ascontiguousarray(v)), layer=0)
    mk.paged_attn_set_deterministic(t.gpu, True)
    bt, tags = t.bt.repeat(n_req, 1), t.tags.repeat(n_req, 1)
    pages = torch.arange(n // 16, dtype=torch.int32, device="cuda").repeat(n_req, H, 1)
    counts = torch.full((n_req, H), n // 16, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros((n_req, H, d), device="cuda"), torch.zeros((n_req, H), device="cuda")
    mk.paged_attn_decode_sparse(t.gpu, 0, sp._i16(q).repeat(n_req, 1, 1), bt, tags,
                                torch.full((n_req,), n, dtype=torch.int32, device="cuda"), pages, counts, out, lse,
                                mk.workspace(t.gpu, n_req, n // 16))
    torch.cuda.synchronize()
    assert mk.kv_pool_check_errors(t.gpu) == 0
    got, gl = out.cpu().numpy(), lse.cpu().numpy()
    assert (got == got[:1]).all() and (gl == gl[:1]).all()
    for r, g, kk, vv, x, at in fr.rows(t.orc, 0, q[None], t.obt, t.otags, [n]):
        _, _, o, l = fr.attend(kk, vv, x)
        off, b = np.linalg.norm(got[r, g] - o) / np.linalg.norm(o), fr.bound(kk, vv, x, at)[1]
        print(f"  {off / fr.FEW_BOUND:.2f} and {abs(gl[r, g] - l) / b:.2f} of the bounds", flush=True)
        assert off <= fr.FEW_BOUND and abs(gl[r, g] - l) <= b
