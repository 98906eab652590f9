"""Position rotation on the way into the paged cache, and decode attention over selected
pages: what is measured.

A case is one call of

  rope    ``kv_rope_apply``: bf16 query rows rotated by their positions
  append  ``kv_append_fp8_rope``: new K/V rows appended to FP8 pages, keys rotated on the way
  step    ``paged_attn_decode_append_rope``: a decode step of one layer, query and new key
          rotated, token appended, attention over the request's FP8 and TQ3 pages
  bounds  ``kv_page_bounds_update``: channelwise largest and smallest key of each page
  select  ``paged_attn_select_pages``: per request and KV head the pages whose bound on
          q.k is largest, the first and last ones always among them
  sparse  ``paged_attn_decode_sparse``: decode attention over the selected pages

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
TAG_R, TAG_S, TAG_NONE = 0, 2, 0xFF
E4M3 = torch.float8_e4m3fn
LEVELS = (-2.25, -1.375, -0.75, -0.25, 0.25, 0.75, 1.375, 2.25)


# ---------------------------------------------------------------- the cases

def _case(name, kind, hq, hkv, d, n_req, lo, hi, **more):
    c = dict(kind=kind, hq=hq, hkv=hkv, d=d, n_req=n_req, lo=lo, hi=hi, **more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # queries of one decode step of 64 requests, a quarter of the channels rotated
        _case("rope_step_64", "rope", 24, 4, 256, 64, 1, 1, rot=64, axes=1, pairs="halves", far=65536, packed=False),
        # queries of a 16K-token prompt with images (three axes), taken out of packed q/k/v rows
        _case("rope_prompt_16k", "rope", 24, 4, 256, 1, 16384, 16384, rot=256, axes=3, pairs="halves", far=0,
              packed=True),
        # one token of each of 24 short chats into one layer, neighbouring channels paired
        _case("append_step_24", "append", 32, 8, 128, 24, 1, 1, layers=1, start=3977, rot=128, axes=1,
              pairs="neighbours", far=0),
        # eight ragged prompts with images taken into four layers
        _case("append_prompt_8x4k", "append", 24, 4, 256, 8, 2003, 6007, layers=4, start=0, rot=256, axes=3,
              pairs="halves", far=0),
        # the smallest decode step: one 2K-token request, one KV head
        _case("step_one_2k", "step", 8, 1, 128, 1, 2048, 2048, window=256, rot=128, axes=1, pairs="halves", far=0),
        # a batch of eight long requests
        _case("step_8x16k", "step", 24, 4, 256, 8, 12001, 20011, window=1024, rot=64, axes=3, pairs="halves",
              far=100000),
        # after a decode step of 64 requests: the page that took the token, one layer
        _case("bounds_step_64", "bounds", 24, 4, 256, 64, 4096, 65536, layers=1, new=1),
        # after eight prompts: all their pages, four layers
        _case("bounds_prompt_8x4k", "bounds", 24, 4, 256, 8, 2003, 6007, layers=4, new=0),
        # one interactive user at 16K context
        _case("select_one_16k", "select", 24, 4, 256, 1, 16384, 16384, pages=128, first=4, last=16),
        # a full batch of long requests
        _case("select_64x32k", "select", 24, 4, 256, 64, 8192, 32768, pages=256, first=4, last=64),
        # attention over the pages selected for one user: 128 of 1,024
        _case("sparse_one_16k", "sparse", 24, 4, 256, 1, 16384, 16384, window=1024, pages=128, first=4, last=16),
        # and for a batch of long requests: 256 of up to 2,048
        _case("sparse_32x32k", "sparse", 24, 4, 256, 32, 8192, 32768, window=1024, pages=256, first=4, last=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges; none costs more than the largest listed one."""
    kind = rng.choice(["rope", "append", "step", "bounds", "select", "sparse"])
    hq, hkv, d = rng.choice([(8, 1, 128), (24, 4, 256), (24, 4, 256), (32, 8, 128), (16, 4, 128), (24, 2, 256),
                             (16, 2, 256), (32, 2, 128)])
    axes = rng.choice([1, 1, 2, 3])
    turn = dict(rot=rng.choice([d, d, d // 2, d // 4, 96, 20]), axes=axes, pairs=rng.choice(["halves", "neighbours"]),
                far=rng.choice([0, 0, 1000, 100000, 1000000]))
    if kind == "rope":
        n = _log(rng, 1, 16384 * 24 * 256 // (hq * d))
        n_req = rng.choice([1, min(n, 256)])
        each = max(1, n // n_req)
        return _case(None, kind, hq, hkv, d, n_req, each, each, packed=rng.random() < 0.5, **turn)
    if kind == "append":
        layers = rng.choice([1, 1, 2, 4])
        n_req = _log(rng, 1, 64)
        hi = _log(rng, 1, max(1, 30000 * 16 * 256 // (n_req * layers * hkv * d)))
        return _case(None, kind, hq, hkv, d, n_req, max(1, int(hi * rng.uniform(0.1, 1.0))), hi, layers=layers,
                     start=rng.choice([0, 37, 500]), **turn)
    if kind == "bounds":
        layers = rng.choice([1, 1, 2, 4])
        n_req = _log(rng, 1, 64)
        hi = _log(rng, 40, max(80, min(65536, 30000 * 16 * 256 // (n_req * layers * hkv * d))))
        return _case(None, kind, hq, hkv, d, n_req, max(1, int(hi * rng.uniform(0.1, 1.0))), hi, layers=layers,
                     new=rng.choice([0, 1, 33]))
    n_req = _log(rng, 1, 32)
    most = min(65536, 32 * 32768 * 4 // (n_req * hkv))
    hi = _log(rng, 100, most)
    lo = max(1, int(hi * rng.uniform(0.1, 1.0)))
    if kind == "step":
        hi = max(1, min(hi, 8 * 16384 * 4 // (n_req * hkv)))
        return _case(None, kind, hq, hkv, d, n_req, min(lo, hi), hi, window=rng.choice([256, 1000, 1024, 2048]), **turn)
    pages = _log(rng, 4, 300)
    first = min(rng.choice([0, 1, 4]), pages)
    last = min(rng.choice([1, 2, 16, 64]), pages - first)
    more = dict(window=rng.choice([256, 1000, 1024])) if kind == "sparse" else {}
    return _case(None, kind, hq, hkv, d, n_req, lo, hi, pages=pages, first=first, last=last, **more)


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
    return 1e6 ** (-np.arange(m) / m), ((np.arange(m) // 4) % c["axes"]).astype(np.uint8)


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
    the window are TQ3 (none without a window), the others FP8; pages past held[r] are not mapped yet."""
    hkv, d, n_req = c["hkv"], c["d"], len(held)
    mp = _pages(max(total))
    bt = np.full((n_req, mp), -1, np.int32)
    tags = np.full((n_req, mp), TAG_NONE, np.uint8)
    for r, n in enumerate(held):
        old = max(0, n - c["window"]) // PAGE if "window" in c else 0
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
        s["pool"] = pool = mk.Pool(layers, c["hq"], hkv, d, s["n8"], s["n3"], c.get("window", 1024), s["signs"], s["order"])
        pool.fp8_view().copy_(s["pages"])
        pool.fp8_scales_view().copy_(s["scales"])
        pool.tq3_view().copy_(s["tq3"])
        s["pages"], s["scales"], s["tq3"] = pool.fp8_view(), pool.fp8_scales_view(), pool.tq3_view()
    s["sign"] = torch.from_numpy(s["signs"]).cuda()


def _lists(c, seed, lens):
    """Pages as a selection leaves them: the first ones, the last ones and some between, ascending."""
    out = np.full((len(lens), c["hkv"], c["pages"]), -1, np.int32)
    cnt = np.zeros((len(lens), c["hkv"]), np.int32)
    g = _np(seed, "lists")
    for r, n in enumerate(lens):
        np_, k = _pages(n), min(_pages(n), c["pages"])
        cnt[r] = k
        for h in range(c["hkv"]):
            if np_ <= c["pages"]:
                out[r, h, :k] = np.arange(k)
            else:
                mid = c["first"] + g.choice(np_ - c["first"] - c["last"], size=k - c["first"] - c["last"], replace=False)
                out[r, h] = np.concatenate([np.arange(c["first"]), np.sort(mid), np.arange(np_ - c["last"], np_)])
    return _i32(out), _i32(cnt)


def prepare(case, seed):
    c = case
    lens = _spread(c["n_req"], c["lo"], c["hi"])
    hq, hkv, d, n_req, kind = c["hq"], c["hkv"], c["d"], c["n_req"], c["kind"]
    s = {"case": c, "seed": int(seed)}
    if "rot" in c:
        freq, axis = _turn(c)
        s["freq"], s["axis"] = torch.from_numpy(freq).cuda(), torch.from_numpy(axis).cuda().long()
        if own:
            import paper_2608_23834_amd as mk
            s["rope"] = mk.Rope(d, freq, axis, c["axes"], interleaved=c["pairs"] == "neighbours", scale=1.0)
    if kind == "rope":
        n = sum(lens)
        s["pos"] = _positions(c, _np(seed, "at").integers(0, 1000, n_req), lens)
        rows = _rows(seed, "q", n, hq + 2 * hkv if c["packed"] else hq, d)
        s["x"] = rows[:, :hq]
        s["out"] = torch.zeros((n, hq, d), dtype=torch.bfloat16, device="cuda")
    elif kind == "append":
        held = _spread(n_req, c["start"] // 30, c["start"])
        _cache(s, c, seed, held, [a + b for a, b in zip(held, lens)], c["layers"])
        n = sum(lens)
        s["before"], s["cu"], s["pos"] = _i32(held), _i32(_cum(lens)), _positions(c, held, lens)
        s["touch"] = max(_pages(a + b) - a // PAGE for a, b in zip(held, lens))
        s["k"] = torch.stack([_rows(seed, "k%d" % l, n, hkv, d) for l in range(c["layers"])])
        s["v"] = torch.stack([_rows(seed, "v%d" % l, n, hkv, d) for l in range(c["layers"])])
    elif kind == "step":
        _cache(s, c, seed, lens, [n + 1 for n in lens], 1)
        s["before"], s["cu"] = _i32(lens), _i32(_cum([1] * n_req))
        s["pos"], s["touch"] = _positions(c, lens, [1] * n_req), 1
        s["q"] = _rows(seed, "q", n_req, hq, d)
        s["k"], s["v"] = _rows(seed, "k0", n_req, hkv, d)[None], _rows(seed, "v0", n_req, hkv, d)[None]
    elif kind == "bounds":
        _cache(s, c, seed, lens, lens, c["layers"])
        s["from"] = _i32([max(0, n - c["new"]) if c["new"] else 0 for n in lens])
        s["seq"] = _i32(lens)
        s["touch"] = max(_pages(n) - (max(0, n - c["new"]) if c["new"] else 0) // PAGE for n in lens)
    if kind in ("bounds", "select"):
        layers, mp = c.get("layers", 1), _pages(max(lens))
        shape = (layers, n_req, hkv, mp)
        if kind == "bounds":
            s["codes"] = torch.zeros((*shape, 2, d), dtype=torch.uint8, device="cuda")
            s["bscale"] = torch.zeros(shape, device="cuda")
        else:
            mid = torch.randn((*shape, d), generator=_gen(seed, "mid"), device="cuda") * 40.0
            half = torch.rand((*shape, d), generator=_gen(seed, "half"), device="cuda") * 100.0 + 60.0
            s["codes"] = torch.stack([mid + half, mid - half], 4).clamp(-448, 448).to(E4M3).view(torch.uint8)
            s["bscale"] = torch.rand(shape, generator=_gen(seed, "bs"), device="cuda") * 0.004 + 0.006
            s["mp"], s["seq"], s["layers"] = mp, _i32(lens), 1
            s["q"] = _rows(seed, "q", n_req, hq, d)
            s["sel"] = torch.zeros((n_req, hkv, c["pages"]), dtype=torch.int32, device="cuda")
            s["count"] = torch.zeros((n_req, hkv), dtype=torch.int32, device="cuda")
        if own:  # the same values in the framework's own holder
            import paper_2608_23834_amd as mk
            if kind == "select":
                s["pool"] = mk.Pool(1, hq, hkv, d, 1, 1, 1024, np.ones(d, np.int8))
                s["ws"] = mk.select_workspace(s["pool"], n_req, mp)
            s["bounds"] = b = mk.PageBounds(s["pool"], n_req, mp)
            b.codes.copy_(s["codes"])
            b.scales.copy_(s["bscale"])
            s["codes"], s["bscale"] = b.codes, b.scales
    elif kind == "sparse":
        _cache(s, c, seed, lens, lens, 1)
        s["seq"], s["q"] = _i32(lens), _rows(seed, "q", n_req, hq, d)
        s["sel"], s["count"] = _lists(c, seed, lens)
    if kind in ("step", "sparse"):
        s["out"] = torch.zeros((n_req, hq, d), device="cuda")
        s["lse"] = torch.zeros((n_req, hq), device="cuda")
        if own:
            import paper_2608_23834_amd as mk
            s["ws"] = mk.workspace(s["pool"], n_req, c["pages"] if kind == "sparse" else s["mp"])
    return s


# ---------------------------------------------------------------- one pass

def _bits(t):
    return t.view(torch.int16)


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        import paper_2608_23834_amd as mk
        if kind == "rope":
            mk.kv_rope_apply(s["rope"], _bits(s["x"]), s["pos"], _bits(s["out"]))
        elif kind == "append":
            mk.kv_append_fp8_rope(s["pool"], s["rope"], -1, s["bt"], s["tags"], s["before"], s["cu"], s["pos"],
                                  _bits(s["k"]), _bits(s["v"]))
        elif kind == "step":
            mk.paged_attn_decode_append_rope(s["pool"], s["rope"], 0, _bits(s["q"]), _bits(s["k"]), _bits(s["v"]),
                                             s["pos"], s["bt"], s["tags"], s["before"], s["out"], s["lse"], s["ws"])
        elif kind == "bounds":
            mk.kv_page_bounds_update(s["pool"], -1, s["bt"], s["tags"], s["from"], s["seq"], s["bounds"])
        elif kind == "select":
            mk.paged_attn_select_pages(s["pool"], 0, _bits(s["q"]), s["seq"], s["bounds"], s["case"]["first"],
                                       s["case"]["last"], s["sel"], s["count"], s["ws"])
        else:
            mk.paged_attn_decode_sparse(s["pool"], 0, _bits(s["q"]), s["bt"], s["tags"], s["seq"], s["sel"],
                                        s["count"], s["out"], s["lse"], s["ws"])
    elif kind == "rope":
        s["out"] = _rotate(s, s["x"])
    elif kind == "append":
        _append(s)
    elif kind == "step":
        _append(s)
        n = _pages_of(s["before"].long() + 1)
        listed_ = torch.arange(s["mp"], device="cuda").expand(len(n), s["case"]["hkv"], s["mp"])
        s["out"], s["lse"] = _attend(s, _rotate(s, s["q"]), listed_, listed_ < n[:, None, None], s["before"] + 1)
    elif kind == "bounds":
        _bounds(s)
    elif kind == "select":
        s["sel"], s["count"] = _select(s)
    else:
        there = torch.arange(s["sel"].shape[2], device="cuda") < s["count"][:, :, None]
        s["out"], s["lse"] = _attend(s, s["q"], s["sel"].long().clamp(min=0), there, s["seq"])
    if kind == "rope":
        return {"out": s["out"]}
    if kind in ("append", "step"):
        got = {"codes": s["pages"][:, :-1].view(E4M3), "scales": s["scales"][:, :-1], "table": s["bt"], "tags": s["tags"]}
        return got if kind == "append" else {**got, "out": s["out"], "lse": s["lse"]}
    if kind == "bounds":
        return {"codes": s["codes"].view(E4M3), "scales": s["bscale"]}
    if kind == "select":
        return {"pages": s["sel"], "count": s["count"]}
    return {"out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------- the plain forms

def _pages_of(n):
    return (n + PAGE - 1) // PAGE


def _bf16(y):
    """float64 to bfloat16 in one rounding, to nearest even."""
    u = y.view(torch.int64)
    u = (u + (0xFFFFFFFFFFF + ((u >> 45) & 1))) & ~0x1FFFFFFFFFFF
    return u.view(torch.float64).to(torch.bfloat16)


def _rotate(s, x):
    """Rows [..., n, heads, d] rotated by the n tokens' positions; angles and products in 64 bits."""
    c = s["case"]
    ang = s["pos"].double()[s["axis"]].t() * s["freq"]  # [n][rot / 2]
    co, si = ang.cos()[:, None], ang.sin()[:, None]
    rot = c["rot"]
    xd = x[..., :rot].double()
    if c["pairs"] == "halves":
        a, b = xd[..., :rot // 2], xd[..., rot // 2:]
        y = torch.cat([a * co - b * si, b * co + a * si], -1)
    else:
        a, b = xd[..., 0::2], xd[..., 1::2]
        y = torch.stack([a * co - b * si, b * co + a * si], -1).flatten(-2)
    return torch.cat([_bf16(y), x[..., rot:]], -1)


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
    x = torch.stack([_rotate(s, s["k"]), s["v"]], 1).float()[:, :, row]  # [layer][K, V][r][j][slot][head][d]
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


def _attend(s, q, pages, there, seq):
    """Attention of one query per request over the logical pages pages[r][h][:] where `there`."""
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    n_req, _, n_pg = pages.shape
    r = torch.arange(n_req, device="cuda")[:, None, None]
    h = torch.arange(hkv, device="cuda")[None, :, None]
    pages = torch.where(there, pages, 0)
    ids, stale = s["bt"].long()[r, pages], s["tags"][r, pages] == TAG_S
    i8, i3 = torch.where(stale, 0, ids).clamp(min=0), torch.where(stale, ids, 0)
    k8, v8 = _dense8(s["pages"][0][i8, h], s["scales"][0][i8, h], d)
    k3, v3 = _dense3(s["tq3"][0][i3, h], s["sign"], d)
    st = stale[..., None, None]
    k, v = torch.where(st, k3, k8).flatten(2, 3), torch.where(st, v3, v8).flatten(2, 3)  # [r][h][token][d]
    at = pages[..., None] * PAGE + torch.arange(PAGE, device="cuda")
    ok = (there[..., None] & (at < seq[:, None, None, None])).flatten(2)[:, :, None]
    sc = (q.float().view(n_req, hkv, hq // hkv, d) @ k.transpose(2, 3)) / math.sqrt(d)
    sc = torch.where(ok, sc, -math.inf)
    top = sc.amax(3, keepdim=True)
    w = torch.exp(sc - top)
    total = w.sum(3, keepdim=True)
    return ((w @ v) / total).reshape(n_req, hq, d), (top + total.log()).reshape(n_req, hq)


def _bounds(s):
    c = s["case"]
    d, n_req = c["d"], len(s["seq"])
    p = s["from"].long()[:, None] // PAGE + torch.arange(s["touch"], device="cuda")
    there = p < _pages_of(s["seq"].long())[:, None]
    p = torch.where(there, p, s["from"].long()[:, None] // PAGE)  # (a padding entry repeats the first page)
    r = torch.arange(n_req, device="cuda")[:, None].expand_as(p)
    ids = s["bt"].long()[r, p]
    k = s["pages"][:, ids, :, :PAGE * d].contiguous().view(E4M3).float().unflatten(-1, (PAGE, d))  # [l][r][j][h][t][d]
    held = (p[:, :, None] * PAGE + torch.arange(PAGE, device="cuda") < s["seq"][:, None, None])[None, :, :, None, :, None]
    hi = torch.where(held, k, -math.inf).amax(4)
    lo = torch.where(held, k, math.inf).amin(4)
    # [l][r][h][p]: the first two indexes of the assignment are (r, p)
    both = torch.stack([hi, lo], 4).to(E4M3).view(torch.uint8)
    s["codes"].permute(1, 3, 0, 2, 4, 5)[r, p] = both.permute(1, 2, 0, 3, 4, 5)
    s["bscale"].permute(1, 3, 0, 2)[r, p] = s["scales"][:, ids, :, 0].permute(1, 2, 0, 3)


def _select(s):
    c = s["case"]
    hq, hkv, d, n_req, mp, k = c["hq"], c["hkv"], c["d"], len(s["seq"]), s["mp"], c["pages"]
    b = s["codes"][0].view(E4M3).float().double()  # [r][h][p][hi, lo][d]
    q = s["q"].double().view(n_req, hkv, hq // hkv, d)
    # (64 bits: which page is in and which is out hangs on the last of them)
    score = q.clamp(min=0) @ b[..., 0, :].transpose(2, 3) + q.clamp(max=0) @ b[..., 1, :].transpose(2, 3)
    score = score.amax(2) * s["bscale"][0].double()
    n = _pages_of(s["seq"].long())[:, None, None]
    p = torch.arange(mp, device="cuda")
    score = torch.where((p < c["first"]) | (p >= n - c["last"]), math.inf, score)
    score = torch.where(p < n, score, -math.inf)
    best = score.sort(dim=2, descending=True, stable=True).indices[..., :k]
    count = n.clamp(max=k).expand(n_req, hkv, 1)
    best = torch.where(torch.arange(best.shape[2], device="cuda") < count, best, 1 << 40).sort(2).values
    sel = torch.full((n_req, hkv, k), -1, dtype=torch.int32, device="cuda")
    sel[..., :best.shape[2]] = torch.where(best < 1 << 40, best, -1)
    return sel, count[..., 0].int()


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    lens = _spread(c["n_req"], c["lo"], c["hi"])
    hq, hkv, d, kind, n = c["hq"], c["hkv"], c["d"], c["kind"], sum(lens)
    group = hq // hkv
    if kind == "rope":
        return {"bytes": n * (4 * hq * d + 4 * c["axes"]), "flops": n * hq * c["rot"] * 3}
    if kind == "append":
        return {"bytes": c["layers"] * n * hkv * d * 6 + 4 * n * c["axes"],
                "flops": c["layers"] * n * hkv * (c["rot"] * 3 + 2 * d)}
    if kind == "bounds":
        new = [min(c["new"], m) if c["new"] else m for m in lens]
        pages = sum(_pages(m) - (m - k) // PAGE for m, k in zip(lens, new))
        held = sum(m - (m - k) // PAGE * PAGE for m, k in zip(lens, new))
        return {"bytes": c["layers"] * hkv * (held * d + pages * (2 * d + 8)), "flops": c["layers"] * hkv * held * d * 2}
    if kind == "select":
        pages = sum(_pages(m) for m in lens if _pages(m) > c["pages"])
        return {"bytes": hkv * pages * (2 * d + 4) + 2 * hq * d * len(lens) + 4 * hkv * c["pages"] * len(lens),
                "flops": hkv * pages * 4 * group * d}
    b8, b3, rows = 2 * PAGE * d + 8, 16 * d + 32, len(lens) * hq * 6 * d
    if kind == "step":
        old = [max(0, m - c["window"]) // PAGE for m in lens]
        pages = sum(_pages(m + 1) * b8 - o * (b8 - b3) for m, o in zip(lens, old))
        return {"bytes": hkv * pages + rows + len(lens) * hkv * d * 6, "flops": sum(4 * hq * d * (m + 1) for m in lens)}
    bytes_, flops = rows, 0
    for m in lens:  # the old pages' share of those between the first and last
        np_, k = _pages(m), min(_pages(m), c["pages"])
        new = min(k, np_ - max(0, m - c["window"]) // PAGE)
        bytes_ += hkv * (new * b8 + (k - new) * b3)
        flops += 4 * hq * d * k * PAGE
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------- from the definition, in 64 bits

def _turned(s, x):
    """Rotated rows, unrounded: every pair as a complex number times e^(i angle)."""
    c = s["case"]
    m = c["rot"] // 2
    freq, axis = _turn(c)
    pos = s["pos"].cpu().numpy().astype(np.float64)
    ang = torch.from_numpy(pos[axis].T * freq).cuda()
    y = x.double().clone()
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
    if kind == "rope":
        return {"out": _turned(s, s["x"])}
    if kind == "select":
        return None
    if kind == "bounds":
        return _exact_bounds(s)
    if kind in ("append", "step"):
        codes, scales = _exact_append(s)
        got = {"codes": codes[:, :-1] if kind == "append" else None, "scales": scales[:, :-1], "table": None, "tags": None}
        if kind == "append":
            return got
        run(s)  # (the pages that the attention then reads)
    q = _bf16(_turned(s, s["q"])).double() if kind == "step" else s["q"].double()
    seq = [x + 1 for x in s["before"].tolist()] if kind == "step" else s["seq"].tolist()
    out = torch.zeros((len(seq), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((len(seq), hq), dtype=torch.float64, device="cuda")
    for r, n in enumerate(seq):
        np_ = _pages(n)
        k = torch.zeros((np_, hkv, PAGE, d), dtype=torch.float64, device="cuda")
        v = torch.zeros_like(k)
        for tag in (TAG_R, TAG_S):
            i = (s["tags"][r, :np_] == tag).nonzero()[:, 0]
            if len(i):
                k[i], v[i] = _k_v(s, s["bt"][r, i].long(), tag, 0)
        for h in range(hkv):
            p = torch.arange(np_, device="cuda") if kind == "step" else s["sel"][r, h, :int(s["count"][r, h])].long()
            kk, vv = k[p, h].reshape(-1, d), v[p, h].reshape(-1, d)
            ok = (p[:, None] * PAGE + torch.arange(PAGE, device="cuda") < n).flatten()
            g = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            sc = q[r, g] @ kk[ok].T / math.sqrt(d)
            lse[r, g] = torch.logsumexp(sc, 1)
            out[r, g] = torch.softmax(sc, 1) @ vv[ok]
    return {**got, "out": out, "lse": lse} if kind == "step" else {"out": out, "lse": lse}


def _exact_append(s):
    """The pages' values over their scales before E4M3's rounding, and the scales, request by request."""
    d, layers = s["case"]["d"], s["k"].shape[0]
    hkv = s["case"]["hkv"]
    codes = s["pages"].view(E4M3).double()
    scales = s["scales"].double()
    k, v = _bf16(_turned(s, s["k"])).double(), s["v"].double()
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


def _exact_bounds(s):
    d = s["case"]["d"]
    codes = s["codes"].view(E4M3).double()
    scales = s["bscale"].double()
    for r, (a, n) in enumerate(zip(s["from"].tolist(), s["seq"].tolist())):
        p = torch.arange(a // PAGE, _pages(n), device="cuda")
        id_ = s["bt"][r, p].long()
        k = s["pages"][:, id_, :, :PAGE * d].contiguous().view(E4M3).double().view(-1, len(p), s["case"]["hkv"], PAGE, d)
        last = n - int(p[-1]) * PAGE
        top, low = k.amax(3), k.amin(3)
        top[:, -1], low[:, -1] = k[:, -1, :, :last].amax(2), k[:, -1, :, :last].amin(2)
        codes[:, r, :, p, 0], codes[:, r, :, p, 1] = top.transpose(1, 2), low.transpose(1, 2)
        scales[:, r, :, p] = s["scales"][:, id_, :, 0].double().transpose(1, 2)
    return {"codes": codes, "scales": scales}
