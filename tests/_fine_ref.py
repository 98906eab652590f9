"""The error that decode attention of fp32's exactness may have, and what it would be with one of
its parts held in fewer bits: for the rotating step and sparse attention, in numpy, 64 bits.

Error sources of a score s_t (nats), all of independent signs: every entry of the rotated query,
2^-22 of it (an fp16 pair, half a step each); a rounding of the running sum per eight products, d / 8
of them; eight more roundings of scales and exponents, each 2^-24 of the score.  With
B_t = max(|s_t|, sqrt(sum_c (q_c k_tc)^2 / d), |q| |k_t| / d) over whatever they are relative to -- the
second and third being a sum of d terms of random sign in the plain and in the rotated channels --
they come to a relative error of the weight
    eta_t^2 = (2^-22 B_t)^2 + (d / 8 + 8) (2^-24 B_t)^2 + (2^-22)^2 + (2^-23)^2,
the last two the weight's own fp16 pair and its exponential.  With the normalized weights w and the
output o that makes, rms over the signs and as a 2-norm over the channels, for a query
    |do|^2 = sum_t w_t^2 eta_t^2 |v_t - o|^2
             + sum_pages (3 2^-24 w_page |V_page|)^2 + n_pages (2^-24 |o|)^2,
V_page the channelwise largest |v|: zero + scale code takes two sums of up to three times that, and
every page is added to the accumulator in fp32.  A row of d channels is many signs, so three times the
rms is never reached; tokens that share all their weight among a few are few signs, so a bias of one
rounding, 2^-22 |o|, comes on top.  lse: 3 sqrt(sum w^2 eta^2) + 2^-22 + 2^-22 |lse|."""
import numpy as np

PAGE = 16


def attend(k, v, q):
    """Weights (normalized), output and lse of one query in 64 bits."""
    s = k @ q / np.sqrt(len(q))
    w = np.exp(s - s.max())
    z = w.sum()
    return s, w / z, (w / z) @ v, s.max() + np.log(z)


def bound(k, v, q, at=None):
    """(bound on |do|, on |dlse|) of one query over rows k, v; at: the rows' positions."""
    d = len(q)
    s, w, o, lse = attend(k, v, q)
    b = np.maximum(np.abs(s), np.sqrt(((k * q) ** 2).sum(1) / d))
    b = np.maximum(b, np.linalg.norm(k, axis=1) * np.linalg.norm(q) / d)
    eta2 = (2.0 ** -22 * b) ** 2 + (d / 8 + 8) * (2.0 ** -24 * b) ** 2 + 2.0 ** -44 + 2.0 ** -46
    page = (np.arange(len(s)) if at is None else np.asarray(at)) // PAGE
    pages, first = np.unique(page, return_index=True)
    wp = np.add.reduceat(w, first)
    vp = np.linalg.norm(np.maximum.reduceat(np.abs(v), first), axis=1)
    do2 = (w ** 2 * eta2 * ((v - o) ** 2).sum(1)).sum() + ((3 * 2.0 ** -24 * wp * vp) ** 2).sum() \
        + len(pages) * (2.0 ** -24 * np.linalg.norm(o)) ** 2
    return (3 * np.sqrt(do2) + 2.0 ** -22 * np.linalg.norm(o),
            3 * np.sqrt((w ** 2 * eta2).sum()) + 2.0 ** -22 + 2.0 ** -22 * abs(lse))


def rows(orc, layer, q_bits, bt, tags, lens, pages=None, counts=None):
    """Per request and query head: (r, g, k, v, q, positions) of what it attends to, in 64 bits."""
    from _rope_ref import bf16_f64
    n_req, Hq, _ = q_bits.shape
    H = orc.n_kv_heads
    q = bf16_f64(q_bits)
    for r, n in enumerate(lens):
        for h in range(H):
            k, v = orc.reconstruct(layer, r, h, bt, tags, n)
            at = np.arange(n)
            if pages is not None:
                at = at[np.isin(at // PAGE, pages[r, h, : counts[r, h]])]
            if len(at):
                for g in range(h * (Hq // H), (h + 1) * (Hq // H)):
                    yield r, g, k[at], v[at], q[r, g], at


def check(got_out, got_lse, *args):
    """The largest error of any query over its bound: (out, lse); at most 1."""
    worst = [0.0, 0.0]
    for r, g, k, v, q, at in rows(*args):
        _, _, o, lse = attend(k, v, q)
        bo, bl = bound(k, v, q, at)
        worst[0] = max(worst[0], np.linalg.norm(got_out[r, g] - o) / bo)
        worst[1] = max(worst[1], abs(got_lse[r, g] - lse) / bl)
    return worst


# ---------------------------------------------------------------- the same with fewer bits

def fp16(x):
    with np.errstate(over="ignore"):
        return np.asarray(x, np.float32).astype(np.float16).astype(np.float64)


def pair(x):
    hi = fp16(x)
    return hi + fp16(np.asarray(x) - hi)


def e4m3_terms(x, n):
    """x as the sum of n E4M3 values."""
    import torch
    left, got = np.asarray(x, np.float64), 0.0
    for _ in range(n):
        t = torch.from_numpy(left).float().clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
        got, left = got + t, left - t
    return got


def rotated_query(q, sigma, hold):
    """q with its Hadamard rotation, scaled by a power of two (largest entry in [2^14, 2^15), or for hold
    on E4M3 [2^7, 2^8)), held as hold(x) does."""
    d = len(q)
    i = np.arange(d)
    had = 1.0 - 2.0 * (np.array([bin(x).count("1") for x in range(d)])[i[:, None] & i[None]] & 1)
    x = had @ (q * sigma) / np.sqrt(d)
    f = 2.0 ** ((15 if hold is not e4m3_3 else 8) - 1 - np.floor(np.log2(np.abs(x).max())))
    return (had @ (hold(x * f) / f)) / np.sqrt(d) * sigma


def e4m3_3(x):
    return e4m3_terms(x, 3)


def forms(k, v, q, sigma):
    """name -> output with a part held as the name says; weights against a reference 2^-7 below the largest."""
    def out(qh, hold, below=7):
        s = k @ qh / np.sqrt(len(q))
        w = np.exp(s - s.max()) * 2.0 ** below
        return hold(w) @ v / w.sum()
    same = lambda x: x  # noqa: E731
    good = rotated_query(q, sigma, pair)
    return {"pairs": out(good, pair), "query once": out(rotated_query(q, sigma, fp16), pair),
            "query in three E4M3 terms": out(rotated_query(q, sigma, e4m3_3), same), "weights once": out(good, fp16),
            "weights against the largest": out(good, pair, 0)}


# ---------------------------------------------------------------- weights that the pair's floor cuts off

FEW_TOKENS, FEW_D, FEW_GAIN = 3200, 128, 10.8


# Its own bound, relative to |o|.  bound() takes the roundings' signs as independent, but here every page
# behind a wave's first is the same, its roundings too, and values and weights are all of one sign, so they
# add up, in units of 2^-24 of the sum that is rounded (half a step):
#   22  a page's products with its values: the matrix unit adds eight products at a time to the sum, each cut
#       below 2^-24 of the largest of them and the sum: 16 products, the low parts' sum in each of the four
#       steps, half a unit for each step's result;
#   24  the additions of a wave's 25 pages to its accumulator;
#   28  the same for its sum of weights, two more inside a page and two across the lanes;
#   16  eight waves' outputs and sums of weights;  7  quotients, the chunk's merge;
#    2  the weights' pair: 3,192 times 2^-25 beside 8 * 2^7 + 3,192 * 2^-3.8.
FEW_BOUND = 99 * 2.0 ** -24


def few_large():
    """(K, V, q) bf16 bits of one head, FEW_TOKENS rows: the first token of each of the first eight pages
    outweighs every other one by about 2^11; all values alike.  Each of the waves that share the pages so
    meets a large weight first and then small ones, all the same and all rounded the same way: an fp16 pair
    that holds no less than 2^-25 of the reference loses up to 2^-14 of each of them."""
    import mkv_workloads as wl
    rng = np.random.default_rng(77)
    q = rng.standard_normal(FEW_D).astype(np.float32)
    q *= np.float32(1.01 * 4.0 / np.linalg.norm(q))
    k = np.zeros((FEW_TOKENS, FEW_D), np.float32)
    k[: 8 * PAGE: PAGE] = q * (FEW_GAIN * np.log(2) * np.sqrt(FEW_D) / 16)
    v = np.broadcast_to(rng.standard_normal(FEW_D).astype(np.float32), k.shape)
    return wl.bf16_round(k), wl.bf16_round(np.ascontiguousarray(v)), wl.bf16_round(q)
