"""8-bit integers with a scale for each row, written from their definition (test infrastructure)."""
import numpy as np


def quantize(x):
    """Codes int8 and fp32 scales of rows x (float64 holding fp32 or narrower values): the scale and the quotient are fp32, the rounding exact."""
    x = np.asarray(x, np.float64).astype(np.float32)
    top = np.abs(x).max(axis=-1)
    bad = ~np.isfinite(top)
    d = np.maximum(np.where(bad, np.float32(1), top), np.float32(1e-10)) / np.float32(127)
    with np.errstate(invalid="ignore", over="ignore"):
        q = (x / d[..., None]).astype(np.float64)
        c = np.clip(np.sign(q) * np.floor(np.abs(q) + 0.5), -127, 127)
    c[bad] = 0
    return c.astype(np.int8), np.where(bad, np.float32(np.nan), d).astype(np.float32)


def product(xc, xd, wc, wd):
    """(y in 64 bits, y as fp32 operations make it before the last rounding) of codes and scales; wc [N, K], xc [M, K]."""
    total = xc.astype(np.float64) @ wc.astype(np.float64).T   # whole numbers below 2^53
    with np.errstate(invalid="ignore", over="ignore"):
        return total * xd.astype(np.float64)[:, None] * wd.astype(np.float64), total.astype(np.float32) * (wd.astype(np.float32) * xd.astype(np.float32)[:, None])


def gated(gate, up):
    """silu(gate) * up in 64 bits, then fp32."""
    with np.errstate(over="ignore", invalid="ignore"):
        return (gate * up / (1.0 + np.exp(-gate))).astype(np.float32)
