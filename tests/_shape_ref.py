"""Attention with shaped scores in 64 bits, in numpy, with the bound on its fp32 form's error.

A score is off by e_t: d + 8 roundings of 2^-24 of sum |q k| scale and 2^-22 of it (the query's fp16
pair); the tanh 2^-22 of the capped score (2 ulp and its argument's rounding); the bias and the scale
and sum of exponents eight roundings of what they hold, 2^-21 (|s| + |bias|).  With weights w the
output then moves by at most sum_t w_t e_t |v_t - o| <= 2 max|v| sum_t w_t e_t, and rounds once per
token of its sums, (n + 64) 2^-24 max|v|; lse by sum_t w_t e_t and 2^-22 (1 + |lse|)."""
import numpy as np

PAGE = 16


def visible(p, n, window=0, first=0, prefix=0):
    """Which of the tokens 0 .. n - 1 a query at position p sees."""
    t = np.arange(n)
    ok = (t <= p) | ((t < prefix) & (p < prefix))
    if window:
        ok &= t >= p - window + 1
    return ok & (t >= first)


def attend_row(q, k, v, p, scale=0.0, cap=0.0, slope=0.0, sink=None, **mask):
    """One query q [d] at position p over k, v [n][d]: out, lse and the bounds on their errors."""
    d = len(q)
    f = float(np.float32(scale)) if scale else 1 / np.sqrt(d)
    ok = visible(p, len(k), **mask)
    k, v, dist = k[ok], v[ok], np.abs(p - np.arange(len(ok))[ok])
    s = k @ q * f
    e = ((d + 8) * 2.0 ** -24 + 2.0 ** -22) * (np.abs(k) @ np.abs(q)) * f
    if cap:
        s = cap * np.tanh(s / cap)
        e = e + 2.0 ** -22 * np.abs(s)
    bias = slope * dist
    e = e + 2.0 ** -21 * (np.abs(s) + np.abs(bias))
    s = s - bias
    if sink is not None:
        s, e, v = np.r_[s, sink], np.r_[e, 2.0 ** -21 * abs(sink) if np.isfinite(sink) else 0.0], np.r_[v, np.zeros((1, d))]
    if not len(s) or s.max() == -np.inf:
        return np.zeros(d), -np.inf, 0.0, 0.0
    w = np.exp(s - s.max())
    z = w.sum()
    w = w / z
    lse = s.max() + np.log(z)
    off = (w * np.where(w > 0, e, 0.0)).sum()
    big = np.abs(v).max(initial=0.0)
    return w @ v, lse, 2 * off * big + (len(s) + 64) * 2.0 ** -24 * big, off + 2.0 ** -22 * (1 + abs(lse))


def shape_of(kw, hq, row, r):
    """Keywords of attend_row for query head hq, row `row` of request r."""
    f = dict(scale=kw.get("scale", 0.0), cap=kw.get("cap", 0.0), window=kw.get("window", 0))
    if kw.get("slopes") is not None:
        f["slope"] = float(kw["slopes"][hq])
    if kw.get("sinks") is not None:
        f["sink"] = float(kw["sinks"][hq])
    if kw.get("first_keys") is not None:
        f["first"] = int(kw["first_keys"][row])
    if kw.get("prefix_lens") is not None:
        f["prefix"] = int(kw["prefix_lens"][r])
    return f


def decode(orc, layer, q, bt, tags, lens, kw):
    """One query per request: out [r][hq][d], lse and both bounds; q float64."""
    n_req, hq, d = q.shape
    out, lse = np.zeros((n_req, hq, d)), np.full((n_req, hq), -np.inf)
    to, tl = np.zeros((n_req, hq)), np.zeros((n_req, hq))
    g = hq // orc.n_kv_heads
    for r, n in enumerate(lens):
        for h in range(orc.n_kv_heads):
            k, v = orc.reconstruct(layer, r, h, bt, tags, n)
            for j in range(h * g, (h + 1) * g):
                out[r, j], lse[r, j], to[r, j], tl[r, j] = attend_row(q[r, j], k, v, n - 1, **shape_of(kw, j, r, r))
    return out, lse, to, tl


def chunk(orc, layer, q, cu, bt, tags, lens, kw):
    """Chunk attention: out [n][hq][d] in 64 bits and a bound on the 2-norm of each row's error in bf16.

    The rotated query is held in three E4M3 terms, 2^-14 of an entry each (or of the row's largest
    entries where that is more): errors of independent signs, so a score is off by eta = 2^-14 B rms at
    most, B the largest of |s|, the root of the sum of (q k)^2 and |q| |k| / sqrt d, all times the softmax
    scale; the cap, the bias and the exponent add 2^-20 (|s| + |bias|).  The output moves by
    sqrt(sum w^2 eta^2 |v - o|^2) rms, of which three times is never reached over a row's many signs; each
    entry then rounds to bf16, 2^-8 of it, and a few weights that share all of a row are few signs:
    2^-13 max|v - o| on top.

    Weights and values are halves in their product.  A weight's 2^-12 moves the output as eta does (and
    by 2^-12 of itself where the row's sum keeps the unrounded weight), and below 2^-14 of the reference,
    2^-17 of the largest weight, it is off by 2^-25 (2^-28) whatever its size: n 2^-28 max|v - o|.  A TQ3
    value is its page's least value, added apart, and a product of scale and code, off by 2^-12 of itself;
    the tokens of a page may share that sign, the pages and channels do not: 3 2^-12 sqrt(sum over pages
    |sum over its tokens w (v - least)|^2)."""
    hq, d = q.shape[1:]
    g = hq // orc.n_kv_heads
    out, tol = np.zeros(q.shape), np.zeros(q.shape[:2])
    for r, n in enumerate(lens):
        rows = np.arange(cu[r], cu[r + 1])
        pos = n - len(rows) + np.arange(len(rows))
        for h in range(orc.n_kv_heads):
            k, v = orc.reconstruct(layer, r, h, bt, tags, n)
            whole = orc.reconstruct(layer, r, h, bt, tags, -(-n // PAGE) * PAGE)[1].reshape(-1, PAGE, d)
            part = np.zeros_like(whole).reshape(-1, d)  # scale times code
            part[:n] = v - np.repeat(whole.min(1), PAGE, 0)[:n]
            part = part.reshape(whole.shape)
            for j in range(h * g, (h + 1) * g):
                f = shape_of({**kw, "first_keys": None}, j, 0, r)
                scale = float(np.float32(f["scale"])) if f["scale"] else 1 / np.sqrt(d)
                x = q[rows, j]
                s = x @ k.T * scale
                b = np.maximum(np.abs(s), np.sqrt((x * x) @ (k * k).T) * scale)
                b = np.maximum(b, np.outer(np.linalg.norm(x, axis=1), np.linalg.norm(k, axis=1)) / np.sqrt(d) * scale)
                if f["cap"]:
                    s = f["cap"] * np.tanh(s / f["cap"])
                bias = f.get("slope", 0.0) * np.abs(pos[:, None] - np.arange(n))
                eta = 2.0 ** -14 * b + 2.0 ** -20 * (np.abs(s) + np.abs(bias))
                s = s - bias
                first = np.zeros(len(rows), int) if kw.get("first_keys") is None else np.asarray(kw["first_keys"])[rows]
                for i in range(len(rows)):
                    s[i, ~visible(pos[i], n, f["window"], int(first[i]), f.get("prefix", 0))] = -np.inf
                top = np.maximum(s.max(1), f.get("sink", -np.inf))
                top = np.where(top == -np.inf, 0.0, top)[:, None]
                w = np.exp(s - top)
                z = w.sum(1, keepdims=True) + np.exp(f.get("sink", -np.inf) - top)
                w = w / np.where(z > 0, z, 1.0)
                o = w @ v
                away2 = (v * v).sum(1) - 2 * o @ v.T + (o * o).sum(1)[:, None]  # |v - o|^2
                out[rows, j] = o
                far = np.sqrt(np.where(w > 0, away2, 0.0).max(1, initial=0.0).clip(min=0.0))
                eta = eta + 2.0 ** -12
                by_page = np.zeros((len(rows), whole.shape[0] * PAGE))
                by_page[:, :n] = w
                coded = np.zeros(len(rows))  # sum over pages of the squared norms
                for g0 in range(whole.shape[0]):
                    coded += ((by_page[:, g0 * PAGE:(g0 + 1) * PAGE] @ part[g0]) ** 2).sum(1)
                tol[rows, j] = (3 * np.sqrt((w * w * eta * eta * away2.clip(min=0.0)).sum(1))
                                + (2.0 ** -13 + n * 2.0 ** -28) * far + 3 * 2.0 ** -12 * np.sqrt(coded)
                                + (2.0 ** -8 + 2.0 ** -12) * np.linalg.norm(o, axis=1))
    return out, tol
