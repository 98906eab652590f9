"""Head norms with their rotation in 64 bits, in numpy, for the tests of those operators."""
import numpy as np

import _rope_ref as ref


def normed(x_bits, w_bits=None, eps=1e-6, add=0.0):
    """bf16 bits [..., heads, d] normed and weighted (weights that broadcast to them), unrounded."""
    x = ref.bf16_f64(x_bits)
    with np.errstate(invalid="ignore", over="ignore"):
        y = x / np.sqrt((x * x).sum(-1, keepdims=True) / x.shape[-1] + eps)
        return y if w_bits is None else y * (ref.bf16_f64(w_bits) + add)


def turned(y, pos, freq, axis, interleaved, scale=1.0):
    """float64 rows [..., n, heads, d] rotated by pos [n_axes][n], unrounded; freq may be empty."""
    m = len(freq)
    y = y.copy()
    if m:
        ang = np.asarray(pos, np.float64)[np.asarray(axis)].T * np.asarray(freq, np.float64)
        c, s = (scale * np.cos(ang))[:, None], (scale * np.sin(ang))[:, None]
        i = np.arange(m)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + m)
        with np.errstate(invalid="ignore", over="ignore"):
            y[..., a], y[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    return y


def norm_rotate(x_bits, w_bits, eps, add, pos, freq, axis, interleaved, scale=1.0):
    """The same as bf16 bits, one rounding."""
    with np.errstate(over="ignore"):
        return ref.bf16_bits(turned(normed(x_bits, w_bits, eps, add), pos, freq, axis, interleaved, scale))
