"""4-bit floating point with block scales on the CPU, in 64 bits: quantisers, values, products, gated activation.

Formats as in include/cubicquant.h: "mx" (blocks of 32, power-of-two scales), "nv" (blocks of 16, e4m3 scales and an fp32 factor g).
"""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([(f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)) for e in range(16) for f in range(8)][:127])   # bytes 0 .. 126
BLOCK = {"mx": 32, "nv": 16}


def nearest_even(v, grid):
    """Index of the nearest grid value to each v >= 0, the even index on a tie, the last one above the grid."""
    hi = np.clip(np.searchsorted(grid, v, side="left"), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = v - grid[lo], grid[hi] - v
    return np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)


def quantize(x, fmt, g=1.0):
    """x float64 [..., K] (values of the input type) -> codes uint8 [..., K] (0 .. 15), scale bytes uint8 [..., K / block]."""
    x = np.asarray(x, dtype=np.float64)
    v = x.reshape(x.shape[:-1] + (-1, BLOCK[fmt]))
    bad = ~np.isfinite(v).all(axis=-1)
    v = np.where(bad[..., None], 0.0, v)
    top = np.abs(v).max(axis=-1)
    if fmt == "mx":
        e = np.where(top > 0, np.frexp(top)[1] - 1, -1000)
        b = np.clip(e - 2 + 127, 0, 254)
        u = v * np.ldexp(1.0, 127 - b)[..., None]
    else:
        r = np.float32(1.0) / np.float32(g)
        s = (top.astype(np.float32) * r).astype(np.float64) / 6.0
        b = nearest_even(np.clip(np.float32(s).astype(np.float64), 2.0 ** -9, 448.0), E4M3)
        i = (r / E4M3[b].astype(np.float32)).astype(np.float32)
        u = (v.astype(np.float32) * i[..., None]).astype(np.float64)
    c = nearest_even(np.abs(u), GRID) | (np.signbit(u).astype(np.int64) << 3)
    c = np.where(bad[..., None], 0, c)
    b = np.where(bad, 255 if fmt == "mx" else 127, b)
    return c.reshape(x.shape).astype(np.uint8), b.astype(np.uint8)


def scale_values(b, fmt):
    b = np.asarray(b).astype(np.int64)
    if fmt == "mx":
        return np.where(b == 255, np.nan, np.ldexp(1.0, b - 127))
    return np.where(b >= 127, np.nan, E4M3[np.minimum(b, 126)])


def values(c, b, fmt, g=1.0):
    """What codes and scales stand for; the scale times g is an fp32 number."""
    s = scale_values(b, fmt)
    if fmt == "nv":
        s = (s.astype(np.float32) * np.float32(g)).astype(np.float64)
    m = np.where(c & 8, -1.0, 1.0) * GRID[c & 7]
    return (m.reshape(c.shape[:-1] + (-1, BLOCK[fmt])) * s[..., None]).reshape(c.shape)


def pack(c):
    return (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)


def gated(gate, up):
    """silu(gate) * up in 64 bits, rounded to fp32 (from which a model dtype takes it)."""
    with np.errstate(over="ignore", invalid="ignore"):
        return (gate / (1.0 + np.exp(-gate)) * up).astype(np.float32)


def product(xc, xb, wc, wb, fmt, gx=1.0, gw=1.0):
    """(y, sum of the magnitudes that were added) of x W^T in 64 bits."""
    x, w = values(xc, xb, fmt), values(wc, wb, fmt)
    a = float(np.float32(gx) * np.float32(gw)) if fmt == "nv" else 1.0
    return (x @ w.T) * a, (np.abs(x) @ np.abs(w).T) * a
