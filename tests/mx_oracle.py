"""The microscaled operators from their definition, in 64 bits on the CPU (numpy): the tests' oracle."""
import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK_BYTES = {4: 16, 8: 32}


def blocks(cols):
    return -(-cols // 32)


def quantize(x, bits):
    """(codes, scales) of the rows of x (float64), block by block."""
    rows, cols = x.shape
    nb = blocks(cols)
    v = np.zeros((rows, nb * 32))
    v[:, :cols] = x
    v = v.reshape(rows, nb, 32)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(v).all(axis=2)
        v = np.where(bad[..., None], 0.0, v)
        top = np.abs(v).max(axis=2)
        e = np.frexp(top)[1] - 1 - (2 if bits == 4 else 0)
        e = np.maximum(np.where(top == 0, -127, e), -127)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    r = v / np.ldexp(1.0, e)[..., None]
    if bits == 8:
        codes = np.clip(np.rint(r * 64), -127, 127).astype(np.int8).reshape(rows, nb * 32)
        return codes, scales
    # Nearest point of the grid, ties to the even code; above the middle of 6 and 8 it is still 6.
    mid = (GRID[1:] + GRID[:-1]) / 2
    a = np.abs(r)
    up = np.searchsorted(mid, a, side="right")     # a tie counts as above
    tie = (up > 0) & (a == mid[np.maximum(up - 1, 0)])
    code = np.where(tie & (up % 2 == 1), up - 1, up)
    code = (code | (np.signbit(r) << 3)).reshape(rows, nb * 16, 2).astype(np.uint8)
    return code[..., 0] | (code[..., 1] << 4), scales


def values(codes, scales, cols):
    """float64 [rows, cols] that the codes stand for."""
    rows, nb = scales.shape
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    if codes.dtype == np.uint8:
        c = np.stack((codes & 15, codes >> 4), axis=2).reshape(rows, nb, 32)
        v = np.where(c & 8, -1.0, 1.0) * GRID[c & 7]
    else:
        v = codes.astype(np.float64).reshape(rows, nb, 32) / 64
    return (v * s[..., None]).reshape(rows, nb * 32)[:, :cols]


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def act(x, kind):
    """f(x) and f'(x)."""
    if kind == "silu":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-x))
        return x * s, s + x * s * (1 - s)
    p = 0.5 * _erfc(-x / math.sqrt(2.0)) if x.size else x.copy()
    return x * p, p + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
