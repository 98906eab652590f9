"""Norms of query and key heads with their rotation, attention with capped, biased and masked
scores, and the way back out of the cache: what is measured.

A case is one call of

  rows    ``kv_norm_rope_apply``: bf16 query rows, every head normed, weighted and rotated
  append  ``kv_append_fp8_norm_rope``: new K/V rows appended to FP8 pages, keys normed and
          rotated on the way
  decode  ``paged_attn_decode_shaped``: one query per request over its FP8 and TQ3 pages, the
          scores capped by a tanh or biased by the distance, within a window or a document,
          with a sink logit per head
  step    ``paged_attn_decode_append_shaped``: a decode step of one layer from raw q, k and v:
          norms, rotation, append, attention
  chunk   ``paged_attn_chunk_shaped``: a chunk of queries per request over the same pages,
          also with a prefix that is seen from both sides; bf16 outputs
  read    ``kv_read_tokens``: bf16 K and V rows of token ranges out of the pages

With ``own`` false ``run`` computes the same in elementary torch operations.  Pages are in
the layouts of include/minima_kv.h: an FP8 page-head is 16 d bytes of K [token][channel],
then 16 d bytes of V [channel group][token group][channel][token]; a TQ3 page-head is 6 d
bytes of K codes, 6 d of V codes, then gamma, V scale and V zero in binary16.
"""
import math
import zlib

import numpy as np
import torch

own = False

PAGE = 16
GOLDEN = 0.6180339887498949
EPS = 1e-6
TAG_R, TAG_S, TAG_NONE = 0, 2, 0xFF
E4M3 = torch.float8_e4m3fn
LEVELS = (-2.25, -1.375, -0.75, -0.25, 0.25, 0.75, 1.375, 2.25)


# ---------------------------------------------------------------- the cases

def _case(name, kind, hq, hkv, d, n_req, lo, hi, **more):
    c = dict(kind=kind, hq=hq, hkv=hkv, d=d, n_req=n_req, lo=lo, hi=hi, **more)
    if name:
        c["name"] = name
    return c


def _shape(cap=0.0, window=0, slopes=False, sinks=False, docs=False, prefix=False):
    return dict(cap=cap, window=window, slopes=slopes, sinks=sinks, docs=docs, prefix=prefix)


def listed():
    return [
        # queries of one decode step of 64 requests, a quarter of the channels rotated, one weight for all heads
        _case("rows_step_64", "rows", 24, 4, 256, 64, 1, 1, rot=64, axes=1, pairs="halves", far=65536, packed=False,
              weight="shared"),
        # queries of a 16K-token prompt with images (three axes), taken out of packed q/k/v rows, a weight per head
        _case("rows_prompt_16k", "rows", 24, 4, 256, 1, 16384, 16384, rot=256, axes=3, pairs="halves", far=0,
              packed=True, weight="heads"),
        # one token of each of 24 short chats into one layer, neighbouring channels paired
        _case("append_step_24", "append", 32, 8, 128, 24, 1, 1, layers=1, start=3977, rot=128, axes=1,
              pairs="neighbours", far=0, weight="shared"),
        # eight ragged prompts taken into four layers, each with weights of its own
        _case("append_prompt_8x4k", "append", 24, 4, 256, 8, 2003, 6007, layers=4, start=0, rot=64, axes=3,
              pairs="halves", far=0, weight="layers"),
        # the smallest decode: one 2K-token request, one KV head, capped scores, a sink per head
        _case("decode_one_2k", "decode", 8, 1, 128, 1, 2048, 2048, recent=256, **_shape(cap=50.0, sinks=True)),
        # a layer with a sliding window in a batch of long requests
        _case("decode_32x32k_window", "decode", 24, 4, 256, 32, 8192, 32768, recent=1024,
              **_shape(window=4096, sinks=True)),
        # a decode step of one interactive user at 16K
        _case("step_one_16k", "step", 24, 4, 256, 1, 16384, 16384, recent=1024, rot=64, axes=1, pairs="halves", far=0,
              weight="shared", **_shape()),
        # a batch of eight long requests, all pages seen, capped scores
        _case("step_8x16k_cap", "step", 24, 4, 256, 8, 12001, 20011, recent=1024, rot=64, axes=3, pairs="halves",
              far=100000, weight="shared", **_shape(cap=30.0)),
        # six ragged chunks after short and long histories, a bias by distance
        _case("chunk_ragged_6", "chunk", 16, 4, 128, 6, 500, 8000, recent=1024, qlo=1, qhi=300,
              **_shape(slopes=True)),
        # chunked prefill of four long documents: capped scores, an image at the chunk's start seen as a whole
        _case("chunk_4x512_16k", "chunk", 24, 4, 256, 4, 12000, 16384, recent=1024, qlo=512, qhi=512,
              **_shape(cap=50.0, prefix=True)),
        # the last 2K tokens of one request, one layer
        _case("read_one_2k", "read", 24, 4, 256, 1, 16384, 16384, recent=1024, layers=1, part=2048),
        # eight whole requests, four layers
        _case("read_8x16k", "read", 24, 4, 256, 8, 12001, 20011, recent=1024, layers=4, part=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges; none costs more than the largest listed one."""
    kind = rng.choice(["rows", "append", "decode", "step", "chunk", "read"])
    hq, hkv, d = rng.choice([(8, 1, 128), (24, 4, 256), (24, 4, 256), (32, 8, 128), (16, 4, 128), (24, 2, 256),
                             (16, 2, 256), (32, 2, 128)])
    turn = dict(rot=rng.choice([0, d, d, d // 2, d // 4, 96, 20, 10]), axes=rng.choice([1, 1, 2, 3]),
                pairs=rng.choice(["halves", "neighbours"]), far=rng.choice([0, 0, 1000, 100000, 1000000]),
                weight=rng.choice(["none", "shared", "shared", "heads"]))
    if kind == "rows":
        n = _log(rng, 1, 16384 * 24 * 256 // (hq * d))
        n_req = rng.choice([1, min(n, 256)])
        each = max(1, n // n_req)
        return _case(None, kind, hq, hkv, d, n_req, each, each, packed=rng.random() < 0.5, **turn)
    if kind == "append":
        layers = rng.choice([1, 1, 2, 4])
        if layers > 1 and rng.random() < 0.5:
            turn["weight"] = "layers"
        n_req = _log(rng, 1, 64)
        hi = _log(rng, 1, max(1, 30000 * 16 * 256 // (n_req * layers * hkv * d)))
        return _case(None, kind, hq, hkv, d, n_req, max(1, int(hi * rng.uniform(0.1, 1.0))), hi, layers=layers,
                     start=rng.choice([0, 37, 500]), **turn)
    recent = rng.choice([256, 1000, 1024, 2048])
    if kind == "read":
        layers = rng.choice([1, 1, 2, 4])
        n_req = _log(rng, 1, 32)
        hi = _log(rng, 100, max(200, min(65536, 100000 * 16 * 256 // (n_req * layers * hkv * d))))
        return _case(None, kind, hq, hkv, d, n_req, max(1, int(hi * rng.uniform(0.1, 1.0))), hi, recent=recent,
                     layers=layers, part=rng.choice([0, 1, 77, 1000]))
    shape = _shape(cap=rng.choice([0.0, 20.0, 50.0]), window=rng.choice([0, 0, 1, 333, 1024, 4096]),
                   slopes=rng.random() < 0.3, sinks=rng.random() < 0.3, docs=rng.random() < 0.3,
                   prefix=kind == "chunk" and rng.random() < 0.3)
    n_req = _log(rng, 1, 32)
    if kind == "chunk":
        n_req = min(n_req, 8)
        hi = _log(rng, 100, min(32768, 65536 // n_req))
        qhi = max(1, min(hi, 1000, int(4 * 512 * 24 * 16384 * 256 / (n_req * hq * d * hi) * rng.uniform(0.02, 1.0))))
        qlo = rng.choice([1, qhi])
        return _case(None, kind, hq, hkv, d, n_req, max(qhi, int(hi * rng.uniform(0.1, 1.0))), hi, recent=recent,
                     qlo=qlo, qhi=qhi, **shape)
    hi = _log(rng, 100, min(65536, 8 * 16384 * 4 // (n_req * hkv)))
    lo = max(1, int(hi * rng.uniform(0.1, 1.0)))
    more = turn if kind == "step" else {}
    return _case(None, kind, hq, hkv, d, n_req, lo, hi, recent=recent, **more, **shape)


# ---------------------------------------------------------------- inputs

def _pages(n):
    return (n + PAGE - 1) // PAGE


def _spread(n, lo, hi):
    """n lengths spread over [lo, hi], the last one hi."""
    return [lo + int((hi - lo) * (((i + 1) * GOLDEN) % 1.0)) for i in range(n - 1)] + [hi]


def _gen(seed, *key):
    g = torch.Generator(device="cuda")
    g.manual_seed(zlib.crc32(repr((int(seed),) + key).encode()))
    return g


def _np(seed, *key):
    return np.random.default_rng([int(seed) & 0x7FFFFFFF, zlib.crc32(repr(key).encode())])


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _cum(v):
    return [0] + [int(x) for x in np.cumsum(v)]


def _rows(seed, what, n, heads, d):
    """bf16 rows [n][heads][d]: N(0,1) times log-normal scales of each head and channel."""
    scale = torch.exp(0.5 * torch.randn((heads, d), generator=_gen(seed, "scale", what), device="cuda"))
    x = torch.randn((n, heads, d), generator=_gen(seed, what), device="cuda")
    return (x * scale).to(torch.bfloat16)


def _turn(c):
    """(inverse frequencies, axis of each) of a case: base 1,000,000, axes in turns of 4 channels."""
    m = c["rot"] // 2
    return 1e6 ** (-np.arange(m) / max(m, 1)), ((np.arange(m) // 4) % c["axes"]).astype(np.uint8)


def _positions(c, starts, lens):
    """int32 [axes][tokens]: text runs on all axes; in the middle third of a request lies an image,
    whose first axis stands still while the others walk over its rows and columns."""
    out = []
    for s, n in zip(starts, lens):
        p = np.tile(np.arange(n) + s + c["far"], (c["axes"], 1))
        a, b = n // 3, 2 * n // 3
        if c["axes"] > 1 and b - a >= 64:
            w = max(1, math.isqrt(b - a))
            i = np.arange(b - a)
            p[0, a:b] = p[0, a]
            p[1, a:b] = p[1, a] + i // w
            if c["axes"] > 2:
                p[2, a:b] = p[2, a] + i % w
        out.append(p)
    return _i32(np.concatenate(out, 1))


def _fp8_pages(seed, n, hkv, d):
    """n page-heads of FP8 codes and their (K, V) scales."""
    n_base = min(n, 4096)
    x = torch.randn((n_base, 2, PAGE * d), generator=_gen(seed, "fp8"), device="cuda")
    x *= torch.exp(0.5 * torch.randn((n_base, 2, 1), generator=_gen(seed, "fp8s"), device="cuda"))
    s = x.abs().amax(2) / 448.0
    codes = (x / s[:, :, None]).to(E4M3).view(torch.uint8).view(n_base, 2 * PAGE * d)
    pick = torch.randint(n_base, (n,), generator=_gen(seed, "fp8p"), device="cuda")
    return codes[pick], s[pick]


def _pack(codes, d):
    """3-bit codes [..., chunk, quad, 4] into the chunks' bytes."""
    c = codes.to(torch.int32)
    quad = c[..., 0] | c[..., 1] << 8 | c[..., 2] << 16 | c[..., 3] << 24
    ndw = 3 * d // 128
    dw = quad[..., 0:2 * ndw:2] | quad[..., 1:2 * ndw:2] << 3
    a, b = quad[..., 2 * ndw::2], quad[..., 2 * ndw + 1::2]
    dw[..., 0::3] |= (a & 0x03030303) << 6
    dw[..., 1::3] |= (a & 0x04040404) << 4 | (b & 0x01010101) << 7
    dw[..., 2::3] |= (b & 0x06060606) << 5
    return dw.contiguous().view(torch.uint8)


def _tq3_pages(seed, n, d):
    """n TQ3 page-heads: K codes of normal variables, V codes of uniform cells over +-1.8 sigma."""
    n_base = min(n, 4096)
    mid = torch.tensor([(a + b) / 2 for a, b in zip(LEVELS, LEVELS[1:])], device="cuda")
    z = torch.randn((n_base, 64, d // 16, 4), generator=_gen(seed, "tq3k"), device="cuda")
    kc = _pack(torch.bucketize(z, mid), d).reshape(n_base, 6 * d)
    z = torch.randn((n_base, 64, d // 16, 4), generator=_gen(seed, "tq3v"), device="cuda")
    vc = _pack(((z + 1.8) * (7 / 3.6)).round().clamp(0, 7), d).reshape(n_base, 6 * d)
    sig = torch.exp(0.5 * torch.randn((n_base, d), generator=_gen(seed, "tq3s"), device="cuda"))
    gamma = torch.exp(0.3 * torch.randn((n_base, PAGE), generator=_gen(seed, "tq3g"), device="cuda"))
    meta = torch.cat([gamma, sig * (3.6 / 7), sig * -1.8], 1).to(torch.float16).view(torch.uint8)
    pick = torch.randint(n_base, (n,), generator=_gen(seed, "tq3p"), device="cuda")
    return torch.cat([kc, vc, meta], 1)[pick]


def _cache(s, c, seed, held, total, layers):
    """The cache of requests that hold held[r] tokens, with table room for total[r]: pages wholly outside
    the recent ones are TQ3 (none without `recent`), the others FP8; pages past held[r] are not mapped yet."""
    hkv, d, n_req = c["hkv"], c["d"], len(held)
    mp = _pages(max(total))
    bt = np.full((n_req, mp), -1, np.int32)
    tags = np.full((n_req, mp), TAG_NONE, np.uint8)
    for r, n in enumerate(held):
        old = max(0, n - c["recent"]) // PAGE if "recent" in c else 0
        tags[r, :_pages(n)] = TAG_R
        tags[r, :old] = TAG_S
    n8, n3 = int((tags == TAG_R).sum()), int((tags == TAG_S).sum())
    fresh = sum(_pages(t) - _pages(n) for n, t in zip(held, total))
    s["n8"], s["n3"] = n8 + fresh + 1, max(n3, 1)  # the last FP8 page is never used
    order = _np(seed, "order8").permutation(n8 + fresh).astype(np.int32)
    bt[tags == TAG_R] = order[fresh:]
    bt[tags == TAG_S] = _np(seed, "order3").permutation(n3)
    s["order"] = np.concatenate([order, [n8 + fresh]]).astype(np.int32)
    s["free"] = torch.from_numpy(s["order"]).cuda().long()
    s["bt"], s["tags"], s["mp"], s["layers"] = torch.from_numpy(bt).cuda(), torch.from_numpy(tags).cuda(), mp, layers
    codes, scales = _fp8_pages(seed, layers * s["n8"] * hkv, hkv, d)
    s["pages"] = codes.view(layers, s["n8"], hkv, 2 * PAGE * d)
    s["scales"] = scales.view(layers, s["n8"], hkv, 2).contiguous()
    tq3 = _tq3_pages(seed, layers * s["n3"] * hkv, d) if n3 else torch.zeros((layers * hkv, 16 * d + 32), dtype=torch.uint8, device="cuda")
    s["tq3"] = tq3.view(layers, s["n3"], hkv, 16 * d + 32)
    s["signs"] = np.where(_np(seed, "signs").integers(0, 2, d) == 1, 1, -1).astype(np.int8)
    if own:  # the same bytes in a pool
        import paper_2608_23834_amd as mk
        s["pool"] = pool = mk.Pool(layers, c["hq"], hkv, d, s["n8"], s["n3"], c.get("recent", 1024), s["signs"], s["order"])
        pool.fp8_view().copy_(s["pages"])
        pool.fp8_scales_view().copy_(s["scales"])
        pool.tq3_view().copy_(s["tq3"])
        s["pages"], s["scales"], s["tq3"] = pool.fp8_view(), pool.fp8_scales_view(), pool.tq3_view()
    s["sign"] = torch.from_numpy(s["signs"]).cuda()


def _weights(c, seed, what, heads):
    """Norm weights around one, as `weight` says: none, [d], [heads][d] or [layers][heads][d]."""
    lay = {"none": None, "shared": (c["d"],), "heads": (heads, c["d"]), "layers": (c.get("layers", 1), heads, c["d"])}
    shape = lay[c["weight"]]
    if shape is None:
        return None
    return (1.0 + 0.3 * torch.randn(shape, generator=_gen(seed, "w", what), device="cuda")).to(torch.bfloat16)


def _norm(c, w):
    import paper_2608_23834_amd as mk
    return mk.HeadNorm(c["d"], w, eps=EPS)


def _doc_starts(seed, what, pos, span):
    """Where the document of each position begins: documents of `span` tokens, laid out anew for each seed."""
    off = _np(seed, "docs", what).integers(0, span, 1)[0]
    return np.maximum(0, (pos + off) // span * span - off)


def prepare(case, seed):
    c = case
    lens = _spread(c["n_req"], c["lo"], c["hi"])
    hq, hkv, d, n_req, kind = c["hq"], c["hkv"], c["d"], c["n_req"], c["kind"]
    s = {"case": c, "seed": int(seed)}
    if "rot" in c:
        s["wq"], s["wk"] = _weights(c, seed, "q", hq), _weights(c, seed, "k", hkv)
        s["freq"], s["axis"] = [torch.from_numpy(x).cuda() for x in _turn(c)]
        s["axis"] = s["axis"].long()
        if own:
            import paper_2608_23834_amd as mk
            s["norm_q"], s["norm_k"] = _norm(c, s["wq"]), _norm(c, s["wk"])
            s["rope"] = mk.Rope(d, *_turn(c), c["axes"], interleaved=c["pairs"] == "neighbours", scale=1.0) if c["rot"] else None
    if kind == "rows":
        n = sum(lens)
        s["pos"] = _positions(c, _np(seed, "at").integers(0, 1000, n_req), lens)
        rows = _rows(seed, "q", n, hq + 2 * hkv if c["packed"] else hq, d)
        s["x"] = rows[:, :hq]
        s["out"] = torch.zeros((n, hq, d), dtype=torch.bfloat16, device="cuda")
        return s
    if kind == "append":
        held = _spread(n_req, c["start"] // 30, c["start"])
        _cache(s, c, seed, held, [a + b for a, b in zip(held, lens)], c["layers"])
        n = sum(lens)
        s["before"], s["cu"], s["pos"] = _i32(held), _i32(_cum(lens)), _positions(c, held, lens)
        s["touch"] = max(_pages(a + b) - a // PAGE for a, b in zip(held, lens))
        s["k"] = torch.stack([_rows(seed, "k%d" % l, n, hkv, d) for l in range(c["layers"])])
        s["v"] = torch.stack([_rows(seed, "v%d" % l, n, hkv, d) for l in range(c["layers"])])
        return s
    if kind == "read":
        _cache(s, c, seed, lens, lens, c["layers"])
        part = [min(n, c["part"]) if c["part"] else n for n in lens]
        s["from"], s["cu"] = _i32([n - p for n, p in zip(lens, part)]), _i32(_cum(part))
        row = np.concatenate([np.full(p, r) for r, p in enumerate(part)])
        at = np.concatenate([np.arange(n - p, n) for n, p in zip(lens, part)])
        # the table entries of the touched pages, each once, and each token's among them
        entry, which = np.unique(row * s["mp"] + at // PAGE, return_inverse=True)
        s["entry"], s["which"], s["slot"] = [torch.from_numpy(x).cuda() for x in (entry, which.reshape(-1), at % PAGE)]
        s["k"] = torch.zeros((c["layers"], sum(part), hkv, d), dtype=torch.bfloat16, device="cuda")
        s["v"] = torch.zeros_like(s["k"])
        return s
    # attention: the queries' rows of each request end at its length
    nq = _queries(c, lens)
    s["nq"], s["most"] = torch.tensor(nq, device="cuda"), max(nq)
    step = kind == "step"
    _cache(s, c, seed, lens, [n + 1 for n in lens] if step else lens, 1)
    seq = np.asarray(lens) + (1 if step else 0)
    s["seq"], s["cu"] = _i32(seq), _i32(_cum(nq))
    p0 = [max(0, int(n) - m - c["window"] + 1) // PAGE if c["window"] else 0 for n, m in zip(seq, nq)]
    s["p0"], s["span"] = torch.tensor(p0, device="cuda"), max(_pages(int(n)) - a for n, a in zip(seq, p0))
    row = np.concatenate([np.full(n, r) for r, n in enumerate(nq)])
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(seq, nq)])
    s["row"], s["qpos"] = torch.from_numpy(row).cuda(), torch.from_numpy(pos).cuda()
    # (capped scores are those that would otherwise grow large)
    gain = 4.0 if c["cap"] and not step else 1.0
    s["q"] = (_rows(seed, "q", len(row), hq, d).float() * gain).to(torch.bfloat16)
    s["slopes"] = torch.from_numpy(2.0 ** (-8.0 * np.arange(1, hq + 1) / hq)).float().cuda() if c["slopes"] else None
    s["sinks"] = torch.randn(hq, generator=_gen(seed, "sinks"), device="cuda") + 2.0 if c["sinks"] else None
    s["first"] = _i32(_doc_starts(seed, "f", pos, max(50, c["hi"] // 3))) if c["docs"] else None
    s["prefix"] = _i32([n - m + max(1, m // 3) for n, m in zip(lens, nq)]) if c["prefix"] else None
    if step:
        s["before"], s["cu"], s["touch"] = _i32(lens), _i32(_cum([1] * n_req)), 1
        s["pos"] = _positions(c, lens, [1] * n_req)
        s["k"], s["v"] = _rows(seed, "k0", n_req, hkv, d)[None], _rows(seed, "v0", n_req, hkv, d)[None]
    kind_of = torch.bfloat16 if kind == "chunk" else torch.float32
    s["out"] = torch.zeros((len(row), hq, d), dtype=kind_of, device="cuda")
    s["lse"] = torch.zeros((n_req, hq), device="cuda")
    if own:
        import paper_2608_23834_amd as mk
        s["shaping"] = mk.Shaping(cap=c["cap"], window=c["window"], slopes=s["slopes"], sinks=s["sinks"],
                                  first_keys=s["first"], prefix_lens=s["prefix"])
        s["ws"] = mk.workspace(s["pool"], n_req, s["mp"], len(row) if kind == "chunk" else 0)
    return s


def _queries(c, lens):
    if c["kind"] != "chunk":
        return [1] * len(lens)
    return [min(a, b) for a, b in zip(lens, _spread(len(lens), c["qlo"], c["qhi"]))]


# ---------------------------------------------------------------- one pass

def _bits(t):
    return t.view(torch.int16)


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        import paper_2608_23834_amd as mk
        if kind == "rows":
            mk.kv_norm_rope_apply(s["rope"], s["norm_q"], _bits(s["x"]), s["pos"] if s["rope"] else None, _bits(s["out"]))
        elif kind == "append":
            mk.kv_append_fp8_norm_rope(s["pool"], s["rope"], s["norm_k"], -1, s["bt"], s["tags"], s["before"], s["cu"],
                                       s["pos"] if s["rope"] else None, _bits(s["k"]), _bits(s["v"]))
        elif kind == "decode":
            mk.paged_attn_decode_shaped(s["pool"], s["shaping"], 0, _bits(s["q"]), s["bt"], s["tags"], s["seq"],
                                        s["out"], s["lse"], s["ws"])
        elif kind == "step":
            mk.paged_attn_decode_append_shaped(s["pool"], s["shaping"], s["rope"], s["norm_q"], s["norm_k"], 0,
                                               _bits(s["q"]), _bits(s["k"][0]), _bits(s["v"][0]), s["pos"] if s["rope"] else None,
                                               s["bt"], s["tags"], s["before"], s["out"], s["lse"], s["ws"])
        elif kind == "chunk":
            mk.paged_attn_chunk_shaped(s["pool"], s["shaping"], 0, _bits(s["q"]), s["cu"], s["bt"], s["tags"], s["seq"],
                                       _bits(s["out"]), s["ws"])
        else:
            mk.kv_read_tokens(s["pool"], -1, s["bt"], s["tags"], s["from"], s["cu"], _bits(s["k"]), _bits(s["v"]))
    elif kind == "rows":
        s["out"] = _rotate(s, s["x"], s["wq"])
    elif kind == "append":
        _append(s)
    elif kind == "read":
        s["k"], s["v"] = _read(s)
    else:
        if kind == "step":
            _append(s)
        o, l = _attend(s, _rotate(s, s["q"], s["wq"]) if kind == "step" else s["q"])
        s["out"] = o.to(s["out"].dtype)
        s["lse"] = l
    if kind == "rows":
        return {"out": s["out"]}
    got = {}
    if kind in ("append", "step"):
        got = {"codes": s["pages"][:, :-1].view(E4M3), "scales": s["scales"][:, :-1], "table": s["bt"], "tags": s["tags"]}
    if kind == "read":
        return {"k": s["k"], "v": s["v"]}
    if kind == "append":
        return got
    return {**got, "out": s["out"]} if kind == "chunk" else {**got, "out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------- the plain forms

def _pages_of(n):
    return (n + PAGE - 1) // PAGE


def _bf16(y):
    """float64 to bfloat16 in one rounding, to nearest even."""
    u = y.view(torch.int64)
    u = (u + (0xFFFFFFFFFFF + ((u >> 45) & 1))) & ~0x1FFFFFFFFFFF
    return u.view(torch.float64).to(torch.bfloat16)


def _rotate(s, x, w):
    """Rows [..., n, heads, d] normed, weighted (w: see _weights) and rotated by the n tokens' positions, in 64 bits
    with one rounding."""
    c = s["case"]
    xd = x.double()
    xd = xd / (xd.square().mean(-1, keepdim=True) + EPS).sqrt()
    if w is not None:
        xd = xd * (w[:, None] if w.dim() == 3 else w).double()
    ang = s["pos"].double()[s["axis"]].t() * s["freq"]  # [n][rot / 2]
    co, si = ang.cos()[:, None], ang.sin()[:, None]
    rot = c["rot"]
    if c["pairs"] == "halves":
        a, b = xd[..., :rot // 2], xd[..., rot // 2:rot]
        y = torch.cat([a * co - b * si, b * co + a * si], -1)
    else:
        a, b = xd[..., 0:rot:2], xd[..., 1:rot:2]
        y = torch.stack([a * co - b * si, b * co + a * si], -1).flatten(-2)
    return _bf16(torch.cat([y, xd[..., rot:]], -1))


def _append(s):
    """Touched pages of all requests as [request][page of the request], padded to the most any has."""
    c = s["case"]
    layers, hkv, d, n_req = s["k"].shape[0], c["hkv"], c["d"], len(s["before"])
    before = s["before"].long()
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    p = before[:, None] // PAGE + torch.arange(s["touch"], device="cuda")  # [r][j]
    at = p[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")  # position of each slot
    new = (at >= before[:, None, None]) & (at < (before + n)[:, None, None])
    there = new.any(2)
    r = torch.arange(n_req, device="cuda")[:, None].expand_as(p)
    ids = torch.where(there, s["bt"].long()[r, p.clamp(max=s["mp"] - 1)], 0)
    fresh = there & (ids < 0)
    rank = fresh.flatten().cumsum(0).view_as(p) - 1
    ids = torch.where(fresh, s["free"][rank.clamp(min=0)], ids)
    ids = torch.where(there, ids, s["n8"] - 1)  # what is not there goes to the page that is never used
    # (a padding entry repeats its request's first page)
    pc = torch.where(there, p, p[:, :1])
    table, tag = torch.where(there, ids, ids[:, :1]).int(), torch.full_like(s["tags"][r, pc], TAG_R)
    s["bt"][r, pc], s["tags"][r, pc] = table, tag
    row = torch.where(new, s["cu"][:-1].long()[:, None, None] + at - before[:, None, None], 0)
    x = torch.stack([_rotate(s, s["k"], s["wk"]), s["v"]], 1).float()[:, :, row]  # [layer][K, V][r][j][slot][head][d]
    x = x * new[None, None, :, :, :, None, None]
    x = x.permute(0, 2, 3, 5, 1, 4, 6)  # [layer][r][j][head][K, V][slot][d]
    amax = x.abs().amax((5, 6))
    old_s = s["scales"][:, ids]
    old = s["pages"][:, ids].view(E4M3).float().view(layers, n_req, s["touch"], hkv, 2, PAGE * d)
    first = (before[:, None] - p * PAGE).clamp(min=0)[None, :, :, None, None]  # slots held before
    grown = (first == 0) | ~(amax <= 448.0 * old_s)
    sc = torch.where(grown, amax / 448.0, old_s)
    k_old = old[..., 0, :].view(*old.shape[:4], PAGE, d)
    v_old = old[..., 1, :].view(*old.shape[:4], 16, 4, d // 16, 4).permute(0, 1, 2, 3, 5, 7, 4, 6).reshape_as(k_old)
    old = torch.stack([k_old, v_old], 4)
    div = torch.where(sc > 0, sc, 1.0)[..., None, None]
    slot = torch.arange(PAGE, device="cuda")[:, None]
    kept = torch.where(grown[..., None, None], old * old_s[..., None, None] / div, old)
    kept = torch.where(slot < first[..., None, None], kept, torch.where(first[..., None, None] == 0, 0.0, old))
    put = new[None, :, :, None, None, :, None]
    code = torch.where(put, x / div, kept).clamp(-448.0, 448.0).to(E4M3).view(torch.uint8)
    k, v = code[:, :, :, :, 0], code[:, :, :, :, 1]
    v = v.view(*v.shape[:4], 4, 4, 16, d // 16).permute(0, 1, 2, 3, 6, 4, 7, 5)
    s["pages"][:, ids] = torch.cat([k.flatten(4), v.flatten(4)], 4)
    s["scales"][:, ids] = sc


def _unpack(b, d):
    """The 3-bit codes of chunks [..., 3 d / 32 bytes] as [..., quad, 4]."""
    dw = b.contiguous().view(torch.int32)
    lo, hi = dw & 0x07070707, (dw >> 3) & 0x07070707
    x, y, z = dw[..., 0::3], dw[..., 1::3], dw[..., 2::3]
    a = ((x >> 6) & 0x03030303) | ((y >> 4) & 0x04040404)
    e = ((y >> 7) & 0x01010101) | ((z >> 5) & 0x06060606)
    quad = torch.cat([torch.stack([lo, hi], -1).flatten(-2), torch.stack([a, e], -1).flatten(-2)], -1)
    return quad.contiguous().view(torch.uint8).view(*quad.shape, 4)


def _hadamard(d):
    i = torch.arange(d, device="cuda")
    ones = ((i[:, None] & i)[..., None] >> torch.arange(8, device="cuda")) & 1
    return 1.0 - 2.0 * (ones.sum(2) & 1).float()


def _dense8(pages, scales, d):
    """K and V [..., 16, d] of FP8 page-heads, in 32 bits."""
    x = pages.contiguous().view(E4M3).float()
    k = x[..., :PAGE * d].unflatten(-1, (PAGE, d))
    v = x[..., PAGE * d:].unflatten(-1, (16, 4, d // 16, 4)).movedim((-3, -1), (-4, -3))
    return k * scales[..., 0, None, None], v.flatten(-4, -3).flatten(-2) * scales[..., 1, None, None]


def _dense3(pages, sign, d):
    """K and V [..., 16, d] of TQ3 page-heads, in 32 bits."""
    level = torch.tensor(LEVELS, device="cuda")
    meta = pages[..., 12 * d:].contiguous().view(torch.float16).float()
    mu = level[_unpack(pages[..., :6 * d].unflatten(-1, (4, 16, 3 * d // 32)), d).int()]  # [g][t][quad][4]
    mu = mu.flatten(-2).transpose(-2, -3).flatten(-2)
    k = (mu @ _hadamard(d)) * (sign.float() / math.sqrt(d)) * meta[..., :PAGE, None]
    code = _unpack(pages[..., 6 * d:12 * d].unflatten(-1, (4, 16, 3 * d // 32)), d).float()  # [g][r][m][token]
    code = code.movedim(-1, -3).flatten(-4, -3).flatten(-2)  # [token][channel]
    return k, meta[..., None, PAGE + d:] + meta[..., None, PAGE:PAGE + d] * code


def _attend(s, q):
    """Attention of the rows q [n][hq][d], row i at position qpos[i] of request row[i], over the whole cache of its
    request: the queries of a request side by side, padded to the most any has."""
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    n_req, g, n = len(s["seq"]), hq // hkv, s["nq"]
    seq, most, mp = s["seq"].long(), s["most"], s["span"]
    r = torch.arange(n_req, device="cuda")[:, None, None]
    h = torch.arange(hkv, device="cuda")[None, :, None]
    # the pages from the first that the window leaves on: [r][page], as many as any request has
    p = s["p0"][:, None] + torch.arange(mp, device="cuda")
    there = p < _pages_of(seq)[:, None]
    p = torch.where(there, p, s["p0"][:, None])
    ids, stale = s["bt"].long()[r[..., 0], p][:, None], (s["tags"][r[..., 0], p] == TAG_S)[:, None]
    i8, i3 = torch.where(stale, 0, ids), torch.where(stale, ids, 0)
    k8, v8 = _dense8(s["pages"][0][i8, h], s["scales"][0][i8, h], d)
    k3, v3 = _dense3(s["tq3"][0][i3, h], s["sign"], d)
    st = stale[..., None, None]
    k, v = torch.where(st, k3, k8).flatten(2, 3), torch.where(st, v3, v8).flatten(2, 3)  # [r][h][token][d]
    # rows in blocks [request][most queries], a row that is not there repeating the last
    begin = n.cumsum(0) - n
    idx = begin[:, None] + torch.minimum(torch.arange(most, device="cuda"), n[:, None] - 1)  # [r][i]
    qb = q[idx].float().view(n_req, most, hkv, g, d).permute(0, 2, 3, 1, 4)  # [r][h][g][i][d]
    sc = (qb.reshape(n_req, hkv, g * most, d) @ k.transpose(2, 3)) / math.sqrt(d)
    sc = sc.view(n_req, hkv, g, most, mp * PAGE)
    if c["cap"]:
        sc = c["cap"] * torch.tanh(sc / c["cap"])
    pos = s["qpos"][idx]
    t = ((s["p0"][:, None] + torch.arange(mp, device="cuda"))[..., None] * PAGE + torch.arange(PAGE, device="cuda")).flatten(1)[:, None]
    away = pos[..., None] - t  # [r][i][t]
    if c["slopes"]:
        sc = sc - s["slopes"].view(hkv, g, 1, 1) * away.abs()[:, None, None].float()
    last = pos
    if c["prefix"]:
        pre = s["prefix"].long()[:, None]
        last = torch.where(pos < pre, torch.maximum(pos, torch.minimum(pre, seq[:, None]) - 1), pos)
    ok = (t <= last[..., None]) & (t < seq[:, None, None])
    if c["window"]:
        ok &= away < c["window"]
    if c["docs"]:
        ok &= t >= s["first"].long()[idx][..., None]
    sc = torch.where(ok[:, None, None], sc, -math.inf)
    top = sc.amax(4, keepdim=True)
    if c["sinks"]:
        top = torch.maximum(top, s["sinks"].view(hkv, g, 1, 1))
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(sc - top)
    total = w.sum(4, keepdim=True)
    if c["sinks"]:
        total = total + torch.exp(s["sinks"].view(hkv, g, 1, 1) - top)
    o = (w.view(n_req, hkv, g * most, -1) @ v).view(n_req, hkv, g, most, d) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log())[..., 0, 0].reshape(n_req, hq)
    back = s["row"], torch.arange(len(s["row"]), device="cuda") - begin[s["row"]]
    return o.permute(0, 3, 1, 2, 4)[back].reshape(-1, hq, d), lse


def _read(s):
    d = s["case"]["d"]
    ids, stale = s["bt"].flatten().long()[s["entry"]], s["tags"].flatten()[s["entry"]] == TAG_S
    i8, i3 = torch.where(stale, 0, ids), torch.where(stale, ids, 0)
    k8, v8 = _dense8(s["pages"][:, i8], s["scales"][:, i8], d)  # [layer][page][head][token][d]
    k3, v3 = _dense3(s["tq3"][:, i3], s["sign"], d)
    st = stale[:, None, None, None]
    # (indexes on either side of a slice come first: [token][layer][head][d])
    return [torch.where(st, a, b).to(torch.bfloat16)[:, s["which"], :, s["slot"]].transpose(0, 1).contiguous()
            for a, b in ((k3, k8), (v3, v8))]


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    lens = _spread(c["n_req"], c["lo"], c["hi"])
    hq, hkv, d, kind, n = c["hq"], c["hkv"], c["d"], c["kind"], sum(lens)
    if kind == "rows":
        return {"bytes": n * (4 * hq * d + (4 * c["axes"] if c["rot"] else 0)), "flops": n * hq * (4 * d + 3 * c["rot"])}
    if kind == "append":
        return {"bytes": c["layers"] * n * hkv * d * 6 + (4 * n * c["axes"] if c["rot"] else 0),
                "flops": c["layers"] * n * hkv * (6 * d + 3 * c["rot"])}
    b8, b3 = 2 * PAGE * d + 8, 16 * d + 32

    def pages(n, a, b):  # bytes of the pages of tokens [a, b) of a request of n, per head and layer
        old = max(0, n - c["recent"]) // PAGE
        p0, p1 = a // PAGE, _pages(b)
        stale = max(0, min(p1, old) - p0)
        return stale * b3 + (p1 - p0 - stale) * b8

    if kind == "read":
        part = [min(m, c["part"]) if c["part"] else m for m in lens]
        return {"bytes": c["layers"] * hkv * (sum(pages(m, m - k, m) for m, k in zip(lens, part)) + 4 * d * sum(part)),
                "flops": c["layers"] * hkv * sum(part) * 2 * d}
    bytes_ = flops = 0
    for m, k in zip(lens, _queries(c, lens)):
        end = m + 1 if kind == "step" else m
        w = c["window"] or end
        span = min(w, c["hi"] // 6) if c["docs"] else w  # (a document's tokens before a place in it, on average)
        bytes_ += hkv * pages(m, max(0, end - k + 1 - max(1, span)), end)
        seen = sum(min(end - i, max(1, span)) for i in range(k))
        flops += 4 * hq * d * seen
        bytes_ += k * hq * d * (4 if kind == "chunk" else 6)
        if kind == "step":
            bytes_ += hkv * d * 6
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------- from the definition, in 64 bits

def _turned(s, x, w):
    """Normed, weighted and rotated rows, unrounded: every pair as a complex number times e^(i angle)."""
    c = s["case"]
    m = c["rot"] // 2
    freq, axis = _turn(c)
    pos = s["pos"].cpu().numpy().astype(np.float64)
    ang = torch.from_numpy(pos[axis].T * freq).cuda()
    y = x.double()
    y = y * torch.rsqrt((y * y).sum(-1, keepdim=True) / c["d"] + EPS)
    if w is not None:
        y = y * (w.double().unsqueeze(1) if w.dim() == 3 else w.double())
    at = torch.arange(m, device="cuda")
    i, j = (at, at + m) if c["pairs"] == "halves" else (2 * at, 2 * at + 1)
    z = torch.complex(y[..., i], y[..., j]) * torch.polar(torch.ones_like(ang), ang)[:, None]
    y[..., i], y[..., j] = z.real, z.imag
    return y


def _k_v(s, id_, tag, layer):
    """K and V [hkv][16][d] of pages id_ [n] of one tag, float64, from their bytes."""
    d, n = s["case"]["d"], len(id_)
    if tag != TAG_S:
        x = s["pages"][layer, id_].view(E4M3).float().double()
        sc = s["scales"][layer, id_].double()
        k = x[..., :PAGE * d].view(n, -1, PAGE, d)
        t = torch.arange(PAGE, device="cuda")[:, None]
        ch = torch.arange(d, device="cuda")[None]
        cl = d // 16
        at = PAGE * d + ((ch // cl * 4 + t // 4) * cl + ch % cl) * 4 + t % 4
        return k * sc[..., 0, None, None], x[..., at] * sc[..., 1, None, None]
    b = s["tq3"][layer, id_].long()  # [n][h][bytes]
    cb, nd = 3 * d // 32, 3 * d // 128
    kc = torch.zeros((*b.shape[:2], PAGE, d), dtype=torch.long, device="cuda")
    vc = torch.zeros_like(kc)
    lane = torch.arange(16, device="cuda")
    for part, out in ((0, kc), (6 * d, vc)):
        for g in range(4):
            for q in range(d // 16):
                for byte in range(4):
                    def word(w):
                        return b[..., part + (g * 16 + lane) * cb + 4 * w + byte]
                    if q < 2 * nd:
                        code = (word(q // 2) >> (3 * (q % 2))) & 7
                    else:
                        w = 3 * ((q - 2 * nd) // 2)
                        code = (word(w) >> 6) + 4 * ((word(w + 1) >> 6) & 1) if q % 2 == 0 else \
                            (word(w + 1) >> 7) + 2 * (word(w + 2) >> 6)
                    if part == 0:
                        out[:, :, lane, d // 4 * g + 4 * q + byte] = code
                    else:
                        out[:, :, 4 * g + byte, lane * (d // 16) + q] = code
    f16 = s["tq3"][layer, id_][..., 12 * d:].contiguous().view(torch.float16).double()
    y = torch.tensor(LEVELS, device="cuda", dtype=torch.float64)[kc]
    step = 1
    while step < d:  # the butterflies of a Walsh-Hadamard transform
        z = y.view(*y.shape[:3], d // (2 * step), 2, step)
        y = torch.stack([z[..., 0, :] + z[..., 1, :], z[..., 0, :] - z[..., 1, :]], -2).flatten(-3)
        step *= 2
    sign = torch.from_numpy(s["signs"].astype(np.float64)).cuda()
    return y * sign * f16[..., :PAGE, None] / math.sqrt(d), f16[..., None, PAGE + d:] + f16[..., None, PAGE:PAGE + d] * vc


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    kind, d, hq, hkv = c["kind"], c["d"], c["hq"], c["hkv"]
    if kind == "rows":
        return {"out": _turned(s, s["x"], s["wq"])}
    if kind == "read":
        return _exact_read(s)
    got = {}
    if kind in ("append", "step"):
        codes, scales = _exact_append(s)
        got = {"codes": codes[:, :-1] if kind == "append" else None, "scales": scales[:, :-1], "table": None, "tags": None}
        if kind == "append":
            return got
        run(s)  # (the pages that the attention then reads)
    q = _bf16(_turned(s, s["q"], s["wq"])).double() if kind == "step" else s["q"].double()
    out = torch.zeros((len(q), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((c["n_req"], hq), dtype=torch.float64, device="cuda")
    for r, n in enumerate(s["seq"].tolist()):
        k, v = _dense64(s, r, n)
        i = (s["row"] == r).nonzero()[:, 0]
        p = s["qpos"][i].double()[:, None]
        t = torch.arange(n, device="cuda").double()[None]
        seen = t <= p
        if c["prefix"]:
            pre = float(s["prefix"][r])
            seen |= (p < pre) & (t < pre)
        if c["window"]:
            seen &= t > p - c["window"]
        if c["docs"]:
            seen &= t >= s["first"][i].double()[:, None]
        for j in range(hq):
            x = q[i, j] @ k[j // (hq // hkv)].T / math.sqrt(d)
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if c["slopes"]:
                x = x - float(s["slopes"][j]) * (p - t).abs()
            x = x.masked_fill(~seen, -math.inf)
            if c["sinks"]:  # as a token without a value
                x = torch.cat([x, torch.full_like(x[:, :1], float(s["sinks"][j]))], 1)
            z = torch.logsumexp(x, 1)
            w = torch.exp(x - torch.where(z == -math.inf, 0.0, z)[:, None])
            out[i, j] = w[:, :n] @ v[j // (hq // hkv)]
            lse[r, j] = z[-1]
    return {**got, "out": out} if kind == "chunk" else {**got, "out": out, "lse": lse}


def _dense64(s, r, n, layer=0):
    """K and V [hkv][n][d] of a request in 64 bits."""
    np_, hkv, d = _pages(n), s["case"]["hkv"], s["case"]["d"]
    k = torch.zeros((np_, hkv, PAGE, d), dtype=torch.float64, device="cuda")
    v = torch.zeros_like(k)
    for tag in (TAG_R, TAG_S):
        i = (s["tags"][r, :np_] == tag).nonzero()[:, 0]
        if len(i):
            k[i], v[i] = _k_v(s, s["bt"][r, i].long(), tag, layer)
    return [x.transpose(0, 1).reshape(hkv, -1, d)[:, :n] for x in (k, v)]


def _exact_read(s):
    cu, first = s["cu"].tolist(), s["from"].tolist()
    shape = s["k"].shape
    k, v = [torch.zeros(shape, dtype=torch.float64, device="cuda") for _ in range(2)]
    for r, a in enumerate(first):
        for layer in range(shape[0]):
            n = a + cu[r + 1] - cu[r]
            x, y = _dense64(s, r, n, layer)
            k[layer, cu[r]:cu[r + 1]], v[layer, cu[r]:cu[r + 1]] = x[:, a:].transpose(0, 1), y[:, a:].transpose(0, 1)
    return {"k": k, "v": v}


def _exact_append(s):
    """The pages' values over their scales before E4M3's rounding, and the scales, request by request."""
    d, layers = s["case"]["d"], s["k"].shape[0]
    hkv = s["case"]["hkv"]
    codes = s["pages"].view(E4M3).double()
    scales = s["scales"].double()
    k, v = _bf16(_turned(s, s["k"], s["wk"])).double(), s["v"].double()
    bt, free = s["bt"].cpu().numpy(), list(s["order"])
    cu = s["cu"].tolist()
    t = torch.arange(PAGE, device="cuda")[:, None]
    ch = torch.arange(d, device="cuda")[None]
    at = (torch.arange(PAGE * d, device="cuda").view(PAGE, d),  # byte of (token, channel): K, V
          PAGE * d + ((ch // (d // 16) * 4 + t // 4) * (d // 16) + ch % (d // 16)) * 4 + t % 4)
    for r, b in enumerate(s["before"].tolist()):
        n = cu[r + 1] - cu[r]
        for p in range(b // PAGE, _pages(b + n)):
            id_ = int(bt[r, p]) if bt[r, p] >= 0 else int(free.pop(0))
            t0, t1 = max(0, b - p * PAGE), min(PAGE, b + n - p * PAGE)
            rows = slice(cu[r] + p * PAGE + t0 - b, cu[r] + p * PAGE + t1 - b)
            for kv, x in ((0, k), (1, v)):
                x = x[:, rows].transpose(1, 2)  # [layer][head][t][d]
                # (a scale is single precision, and whether it grows is decided in it)
                amax = x.abs().amax((2, 3)).float()
                was = scales[:, id_, :, kv].float()
                grown = ~(amax <= 448.0 * was) if t0 else torch.ones_like(amax, dtype=torch.bool)
                sc = torch.where(grown, amax.double() / 448.0, was.double())
                page = codes[:, id_][:, :, at[kv]]
                if t0 == 0:
                    page = torch.zeros_like(page)
                page[:, :, :t0] *= torch.where(grown, was.double() / sc, 1.0)[..., None, None]
                page[:, :, t0:t1] = x / torch.where(sc > 0, sc, 1.0)[..., None, None]
                rest = codes[:, id_]
                rest[:, :, at[kv]] = page
                codes[:, id_] = rest
                scales[:, id_, :, kv] = sc
    return codes, scales
