"""Microscaled 4-bit rows in plain numpy, 64 bits (the checker of the 4-bit calls).

From the definition (OCP Microscaling Formats v1.0: E2M1 elements, E8M0 scales,
blocks of 32) and the row layout that include/scone.h states.
"""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def row_bytes(cols: int) -> int:
    g = -(-cols // 128)
    return -(-68 * g // 16) * 16


def quantize(x: np.ndarray) -> np.ndarray:
    """Packed rows of x [n, cols] (any float type)."""
    x = np.asarray(x)
    n, cols = x.shape
    g = -(-cols // 128)
    out = np.zeros((n, row_bytes(cols)), np.uint8)
    for r in range(n):
        for b in range(-(-cols // 32)):
            v = x[r, 32 * b:32 * b + 32].astype(np.float64)
            if not np.isfinite(v).all():
                out[r, 64 * g + b] = 255
                continue
            top = np.abs(v).max()
            e = -127 if top == 0 else max(int(np.floor(np.log2(top))) - 2, -127)
            if top > 0 and not 2.0 ** np.floor(np.log2(top)) <= top:  # log2 rounded up
                e = max(e - 1, -127)
            out[r, 64 * g + b] = e + 127
            a = np.abs(v) * 2.0 ** -e
            for i, (m, s) in enumerate(zip(a, np.signbit(v))):
                d = np.abs(GRID - m)
                near = np.flatnonzero(d == d.min())
                code = near[0] if near.size == 1 or near[0] % 2 == 0 else near[1]
                k = 32 * b + i
                out[r, k // 2] |= (int(code) | (8 if s else 0)) << (4 * (k % 2))
    return out


def values(rows: np.ndarray, cols: int) -> np.ndarray:
    """The values [n, cols] of packed rows, in 64 bits."""
    g = -(-cols // 128)
    codes = np.empty((rows.shape[0], 128 * g), np.uint8)
    codes[:, 0::2] = rows[:, :64 * g] & 15
    codes[:, 1::2] = rows[:, :64 * g] >> 4
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]
    s = rows[:, 64 * g:68 * g].astype(np.float64)
    scale = np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return (v * np.repeat(scale, 32, axis=1))[:, :cols]


def linear(x: np.ndarray, w: np.ndarray, bias=None, gelu=False, residual=None):
    """act(x w^T + bias) + residual, and sum |x| |w| (what sums round relative to)."""
    y = x @ w.T
    size = np.abs(x) @ np.abs(w).T
    if bias is not None:
        y = y + bias
        size = size + np.abs(bias)
    if gelu:
        from scipy.special import erfc
        y = 0.5 * y * erfc(-y * np.sqrt(0.5))
    if residual is not None:
        y = y + residual
    return y, size
