"""Layers in microscaled 4-bit floating point and Newton-Schulz orthogonalisation in 64 bits, on numpy arrays."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def quantize(x):
    """(codes, scales) of x (rows, cols), one code a value and one byte a block of 32 columns (0 beyond cols)."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    v = np.zeros((rows, nb, BLOCK))
    v.reshape(rows, -1)[:, :cols] = x
    top = np.abs(v).max(-1)
    bad = ~np.isfinite(v).all(-1)
    with np.errstate(invalid="ignore"):
        e = np.clip(np.frexp(np.where(bad | (top == 0), 1.0, top))[1] - 1 - 2, -127, 127)
    e = np.where(top == 0, -127, e)
    a = np.where(bad[..., None], 0.0, np.abs(v) * np.exp2(-e.astype(np.float64))[..., None])
    # the nearest grid point; between two, the one with the even code
    d = np.abs(np.minimum(a, 6.0)[..., None] - GRID)
    near = d.min(-1, keepdims=True)
    hit = d == near
    first = hit.argmax(-1)
    code = np.where((hit.sum(-1) > 1) & (first % 2 == 1), first + 1, first)
    code = code + 8 * np.signbit(v)
    return code.reshape(rows, -1)[:, :cols].astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales):
    """What codes (rows, cols) and scales (rows, blocks) stand for."""
    v = np.where(codes >= 8, -1.0, 1.0) * GRID[codes & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(s, BLOCK, axis=1)[:, :codes.shape[1]]


def linear(x, w, bias=None, relu=False):
    """act(x w^T + bias), and per element the sum of the products' magnitudes."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        y, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        y, mag = y + bias, mag + np.abs(bias)
    return (np.where(y < 0, 0.0, y) if relu else y), mag


def linear_grad(dy, x, w, y=None):
    """dx, dw, db of linear, each with its magnitudes."""
    g = np.asarray(dy, dtype=np.float64)
    if y is not None:
        g = np.where(np.asarray(y) > 0, g, 0.0)
    x, w, ag = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64), np.abs(g)
    return (g @ w, ag @ np.abs(w)), (g.T @ x, ag.T @ np.abs(x)), (g.sum(0), ag.sum(0))


def orthogonalize(g, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    a, b, c = coefficients
    x = np.asarray(g, dtype=np.float64)
    x = x / (np.linalg.norm(x) + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for _ in range(steps):
        m = x @ x.T
        x = a * x + b * (m @ x) + c * (m @ (m @ x))
    return x.T if tall else x
