"""Normed append, shaped attention and the reading back over page ids whose bytes lie past 2^32, and calls
on two streams at a time: the same answers, bit for bit, as from a small pool and one call after the other."""
import numpy as np
import pytest

import mkv_workloads as wl
from test_gpu_shaped import _gpu, _i16

pytestmark = pytest.mark.gpu

D, HQ, HKV, LENS, NQ = 256, 24, 4, [900, 33, 17], [40, 33, 1]
SIZES = (80, 140000), (80, 280000)  # pages of each format: 32 KB and 16 KB and more each


def _i32(x):
    return _gpu(np.asarray(x, np.int32))


class Filled:
    """A pool with the three requests' tokens in it, old pages in TQ3."""

    def __init__(self, far, down):
        import torch
        import paper_2608_23834_amd as mk
        rng = np.random.default_rng(21)
        rows = _i16(wl.bf16_round(rng.standard_normal((sum(LENS), HQ + 2 * HKV, D)).astype(np.float32)))
        self.q = _i16(wl.bf16_round(rng.standard_normal((sum(NQ), HQ, D)).astype(np.float32)))
        n8, n3 = (s[far] for s in SIZES)
        order = lambda n: np.arange(n, dtype=np.int32)[::-1] if down else None  # noqa: E731
        self.pool = mk.Pool(1, HQ, HKV, D, n8, n3, 64, np.where(np.arange(D) % 3, 1, -1), order(n8), order(n3))
        mk.paged_attn_set_deterministic(self.pool, True)
        self.bt = torch.full((3, 60), -1, dtype=torch.int32, device="cuda")
        self.tags = torch.full((3, 60), 0xFF, dtype=torch.uint8, device="cuda")
        self.rope = mk.Rope(D, 1e6 ** (-np.arange(32) / 32))
        self.norm = mk.HeadNorm(D, _i16(wl.bf16_round(rng.standard_normal(D).astype(np.float32))), unit_offset=True)
        self.lens, self.rows = _i32(LENS), rows
        mk.kv_append_fp8_norm_rope(self.pool, self.rope, self.norm, 0, self.bt, self.tags, _i32([0, 0, 0]),
                                   _i32(np.r_[0, np.cumsum(LENS)]), None, rows[:, HQ:HQ + HKV], rows[:, HQ + HKV:])
        mk.kv_migrate_to_tq3(self.pool, self.bt, self.tags, torch.zeros((3, 60), dtype=torch.uint8, device="cuda"), self.lens)

    def buffers(self):
        import torch
        import paper_2608_23834_amd as mk
        z = lambda *s, t=torch.int16: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
        return dict(k=z(944, HKV, D), v=z(944, HKV, D), chunk=z(sum(NQ), HQ, D), out=z(3, HQ, D, t=torch.float32),
                    lse=z(3, HQ, t=torch.float32), ws=mk.workspace(self.pool, 3, 60, sum(NQ)), ws1=mk.workspace(self.pool, 3, 60),
                    sh=mk.Shaping(cap=9.0, sinks=torch.ones(HQ, device="cuda"), window=700),
                    cu=_i32(np.r_[0, np.cumsum(NQ)]), frm=_i32([0, 1, 5]), cut=_i32([0, 900, 932, 944]))

    def calls(self, b, stream=None):
        import paper_2608_23834_amd as mk
        mk.kv_read_tokens(self.pool, 0, self.bt, self.tags, b["frm"], b["cut"], b["k"], b["v"], stream)
        mk.paged_attn_chunk_shaped(self.pool, b["sh"], 0, self.q, b["cu"], self.bt, self.tags, self.lens, b["chunk"], b["ws"], stream)
        mk.paged_attn_decode_shaped(self.pool, b["sh"], 0, self.q[:3], self.bt, self.tags, self.lens, b["out"], b["lse"], b["ws1"],
                                    stream)


NAMES = ("k", "v", "chunk", "out", "lse")


def _answers(f):
    import torch
    import paper_2608_23834_amd as mk
    b = f.buffers()
    f.calls(b)
    step, slse = torch.zeros((3, HQ, D), device="cuda"), torch.zeros((3, HQ), device="cuda")
    new = f.rows[:3]
    mk.paged_attn_decode_append_shaped(f.pool, b["sh"], f.rope, f.norm, f.norm, 0, new[:, :HQ].contiguous(),
                                       new[:, HQ:HQ + HKV].contiguous(), new[:, HQ + HKV:].contiguous(), None, f.bt, f.tags,
                                       f.lens, step, slse, b["ws1"])
    torch.cuda.synchronize()
    assert mk.kv_pool_check_errors(f.pool) == 0
    return [b[n] for n in NAMES] + [step, slse]


def test_far_pages():
    import torch
    near = Filled(0, False)
    assert all((near.tags == t).any() for t in (0, 2))
    want = _answers(near)
    assert all(torch.isfinite(x.float()).all() and x.any() for x in want)
    tops = []
    for down in (False, True):
        f = Filled(1, down)
        for k, (x, y) in enumerate(zip(want, _answers(f))):
            assert torch.equal(x, y), (down, k)
        tops.append([int(f.bt[f.tags == t].max()) for t in (0, 2)])
        del f
        torch.cuda.empty_cache()
    assert max(t[0] for t in tops) * 32768 > 2 ** 32 and max(t[1] for t in tops) * 16384 > 2 ** 32


def test_two_streams_at_a_time():
    """Every call with buffers and a workspace of its own on two streams, several times."""
    import torch
    import paper_2608_23834_amd as mk
    f = Filled(0, False)
    want, one, two = f.buffers(), f.buffers(), f.buffers()
    f.calls(want)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(4):
        for b in (one, two):
            for n in NAMES:
                b[n].zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            f.calls(one, s1)
            f.calls(two, s2)
        torch.cuda.synchronize()
        for b in (one, two):
            for n in NAMES:
                assert torch.equal(b[n], want[n]), n
    assert mk.kv_pool_check_errors(f.pool) == 0


def test_rows_far_apart():
    """Normed rows at the largest stride, in and out, and a weight stride of many heads."""
    import torch
    import paper_2608_23834_amd as mk
    rng = np.random.default_rng(4)
    rows = _i16(wl.bf16_round(rng.standard_normal((3, 3, D)).astype(np.float32)))
    norm, rope = mk.HeadNorm(D, _i16(wl.bf16_round(rng.standard_normal((3, D)).astype(np.float32)))), mk.Rope(D, np.ones(16))
    pos, want = _i32([[3, 70000, 0]]), torch.zeros_like(rows)
    mk.kv_norm_rope_apply(rope, norm, rows, pos, want)
    memory = torch.zeros(2 * 2 ** 31 + 3 * D, dtype=torch.int16, device="cuda")
    far = memory.as_strided((3, 3, D), (2 ** 31, D, 1))
    far.copy_(rows)
    got = torch.zeros_like(rows)
    mk.kv_norm_rope_apply(rope, norm, far, pos, got)
    assert want.any() and torch.equal(got, want)
    mk.kv_norm_rope_apply(rope, norm, far, pos, far)  # in place
    assert torch.equal(far, want)
    del far, memory
    torch.cuda.empty_cache()
