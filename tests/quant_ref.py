"""Weights in 4 bits: the definition of adept_quant_pack's values, element by element, in float64."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantised(w):
    """The values that w [n, k] takes."""
    w = np.asarray(w, np.float64)
    n, k = w.shape
    out = np.empty_like(w)
    for c in range(0, k, 32):
        part = w[:, c:c + 32]
        for r in range(n):
            x = part[r]
            if not np.isfinite(x).all():
                out[r, c:c + 32] = np.nan
                continue
            e = -100
            while e < 100 and np.abs(x).max() > 7 * 2.0 ** e:
                e += 1
            y = np.abs(x) / 2.0 ** e
            far = np.abs(y[:, None] - GRID)
            # the nearest; of two as near the one with the even code
            at = [min(range(8), key=lambda i: (f[i], i % 2)) for f in far]
            out[r, c:c + 32] = np.copysign(GRID[at] * 2.0 ** e, x)
    return out


def quantised_fast(w):
    """The same of a finite matrix, by whole arrays."""
    w = np.asarray(w, np.float64)
    n, k = w.shape
    x = np.zeros((n, -(-k // 32) * 32))
    x[:, :k] = w
    x = x.reshape(n, -1, 32)
    frac, e = np.frexp(np.abs(x).max(-1) / 7)          # frac 2^e, 1/2 <= frac < 1
    e = np.clip(np.where(frac == 0.5, e - 1, e), -100, 100)
    e = np.where(frac == 0, -100, e)[..., None]
    y = np.ldexp(np.abs(x), -e)
    step = np.where(y < 2, 0.5, np.where(y < 4, 1.0, 2.0))
    y = np.minimum(np.round(y / step) * step, 6.0)     # round(): ties to even
    return np.copysign(np.ldexp(y, e), x).reshape(n, -1)[:, :k]
