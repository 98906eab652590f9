"""Plain 64-bit forms of the rotation, the page bounds, the page selection and attention
over listed pages, in numpy, for the tests of those operators."""
import numpy as np

PAGE = 16


def bf16_f64(bits):
    u = np.asarray(bits).view(np.uint16).astype(np.uint32) << 16
    return u.view(np.float32).astype(np.float64)


def bf16_bits(y):
    """float64 -> bf16 bits, one rounding to nearest even."""
    u = np.ascontiguousarray(y, dtype=np.float64).view(np.int64)
    nan = np.isnan(y)
    w = ((u + (0xFFFFFFFFFFF + ((u >> 45) & 1))) & ~0x1FFFFFFFFFFF).view(np.float64)
    small = np.abs(y) < 2.0 ** -126  # subnormal: steps of 2^-133
    w = np.where(small, np.rint(np.where(small, y, 0.0) * 2.0 ** 133) * 2.0 ** -133, w)
    with np.errstate(over="ignore"):
        b = (np.where(nan, 0.0, w).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return np.where(nan, np.uint16(0x7FC0), b)


def rotate(x_bits, pos, freq, axis, interleaved, scale=1.0):
    """bf16 bits [..., n, heads, d] rotated by pos [n_axes][n]."""
    m = len(freq)
    x = bf16_f64(x_bits)
    ang = np.asarray(pos, np.float64)[np.asarray(axis)].T * np.asarray(freq, np.float64)  # [n][m]
    c, s = (scale * np.cos(ang))[:, None], (scale * np.sin(ang))[:, None]
    i = np.arange(m)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + m)
    y = x.copy()
    with np.errstate(invalid="ignore", over="ignore"):
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        bits = bf16_bits(y)
    bits[..., 2 * m:] = np.asarray(x_bits).view(np.uint16)[..., 2 * m:]
    return bits


def same_bits(a, b):
    """Equal bf16 bits; any NaN equals any NaN."""
    a, b = np.asarray(a).view(np.uint16), np.asarray(b).view(np.uint16)
    return np.all((a == b) | (np.isnan(bf16_f64(a)) & np.isnan(bf16_f64(b))))


def e4m3(codes):
    c = np.asarray(codes, np.uint8).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(np.float64) - 10))
    v = np.where(c & 127 == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def bounds(fp8, scales, bt, lens, d):
    """(largest, smallest) value [L][r][H][p][2][d] and scales [L][r][H][p] of FP8 pages; 0 elsewhere."""
    L, _, H = fp8.shape[:3]
    n_req, mp = bt.shape
    out, sc = np.zeros((L, n_req, H, mp, 2, d)), np.zeros((L, n_req, H, mp), np.float32)
    for r, n in enumerate(lens):
        for p in range((n + PAGE - 1) // PAGE):
            k = e4m3(fp8[:, bt[r, p], :, : PAGE * d]).reshape(L, H, PAGE, d)[:, :, : n - p * PAGE]
            out[:, r, :, p, 0], out[:, r, :, p, 1] = k.max(2), k.min(2)
            sc[:, r, :, p] = scales[:, bt[r, p], :, 0]
    return out, sc


def scores(q_bits, vals, sc):
    """Bound of every page, [r][H][p]: q [r][Hq][d], vals [r][H][p][2][d]."""
    n_req, H = vals.shape[:2]
    q = bf16_f64(q_bits).reshape(n_req, H, -1, 1, vals.shape[-1])
    with np.errstate(invalid="ignore"):
        b = (np.maximum(q, 0) * vals[:, :, None, :, 0] + np.minimum(q, 0) * vals[:, :, None, :, 1]).sum(-1)
        b = np.where(np.isnan(b).any(2), np.nan, b.max(2))
        return b * sc


def select(score, lens, n_select, n_first, n_last):
    n_req, H, _ = score.shape
    pages, counts = np.full((n_req, H, n_select), -1, np.int32), np.zeros((n_req, H), np.int32)
    for r, n in enumerate(lens):
        npg = (n + PAGE - 1) // PAGE
        k = min(npg, n_select)
        counts[r] = k
        for h in range(H):
            if npg <= n_select:
                pages[r, h, :k] = np.arange(k)
                continue
            s = score[r, h, n_first: npg - n_last]
            s = np.where(np.isnan(s), -np.inf, s)
            nan = np.isnan(score[r, h, n_first: npg - n_last])
            order = np.lexsort((np.arange(len(s)), nan, -s))  # score, then NaN last, then the lower page
            best = n_first + order[: n_select - n_first - n_last]
            pages[r, h] = np.sort(np.r_[np.arange(n_first), best, np.arange(npg - n_last, npg)])
    return pages, counts


def attend(orc, layer, q_bits, bt, tags, lens, pages=None, counts=None):
    """Attention over listed pages (all where pages is None) of the oracle pool's reconstructed K and V.
    Returns out, lse and the bound on each query's error in units of its largest |v|: twice the error
    of a score -- d + 8 roundings of 2^-24 of sum |q k| / sqrt d -- and a rounding per token."""
    n_req, Hq, d = q_bits.shape
    H = orc.n_kv_heads
    q = bf16_f64(q_bits)
    out, lse = np.zeros((n_req, Hq, d)), np.full((n_req, Hq), -np.inf)
    tol = np.zeros((n_req, Hq))
    qerr = 2.0 ** -22  # of a query entry, as the fp16 pair of the TQ3 product holds it
    for r, n in enumerate(lens):
        for h in range(H):
            k, v = orc.reconstruct(layer, r, h, bt, tags, n)
            at = np.arange(n)
            if pages is not None:
                at = at[np.isin(at // PAGE, pages[r, h, : counts[r, h]])]
            if not len(at):
                continue
            k, v = k[at], v[at]
            for g in range(h * (Hq // H), (h + 1) * (Hq // H)):
                s = k @ q[r, g] / np.sqrt(d)
                w = np.exp(s - s.max())
                lse[r, g] = s.max() + np.log(w.sum())
                out[r, g] = w @ v / w.sum()
                es = ((d + 8) * 2.0 ** -24 + qerr) * (np.abs(k) @ np.abs(q[r, g])).max() / np.sqrt(d)
                tol[r, g] = (2 * es + (len(at) + 64) * 2.0 ** -24) * np.abs(v).max()
    return out, lse, tol
