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
