"""Layers in float, dropout and the cross entropy in 64 bits, on numpy arrays."""
import numpy as np
from scipy.special import erfc

ACTS = ("none", "relu", "gelu", "silu")


def philox(ctr, key):
    """Philox 4x32-10 of counters (.., 4) and a key of two words, uint32."""
    c = [np.asarray(ctr)[..., i].astype(np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    low, half = np.uint64(0xffffffff), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [b >> half ^ c[1] ^ np.uint64(k[0]), b & low, a >> half ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(c, -1).astype(np.uint32)


def threshold(p):
    return int(np.rint(float(np.float32(p)) * 65536))


def mask(rows, cols, p, seed, offset, first_row=0):
    """Dropout's factors of rows first_row .. of a matrix."""
    groups = -(-cols // 8)
    ctr = np.zeros((rows, groups, 4), dtype=np.uint64)
    ctr[..., 0] = np.arange(groups)
    ctr[..., 1] = first_row + np.arange(rows)[:, None]
    offset %= 2 ** 64
    ctr[..., 2], ctr[..., 3] = offset % 2 ** 32, offset // 2 ** 32
    w = philox(ctr, (seed % 2 ** 32, seed // 2 ** 32))
    bits = np.stack((w & 0xffff, w >> 16), -1).reshape(rows, groups * 8)[:, :cols]
    k = threshold(p)
    return np.where(bits >= k, 65536.0 / (65536 - k), 0.0)


def dropout(x, m, residual=None):
    y = np.where(m > 0, np.asarray(x, dtype=np.float64), 0.0) * m   # (a dropped infinity is 0)
    return y if residual is None else y + residual


def act(z, name):
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "relu":
            return np.where(z < 0, 0.0, z)
        if name == "gelu":
            return 0.5 * z * erfc(-z / np.sqrt(2.0))
        if name == "silu":
            return z / (1 + np.exp(-z))
    return z


def slope(z, name):
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "relu":
            return (z > 0).astype(np.float64)
        if name == "gelu":
            return 0.5 * erfc(-z / np.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
        if name == "silu":
            s = 1 / (1 + np.exp(-z))
            return s + z * s * (1 - s)
    return np.ones_like(z)


def linear(x, w, bias=None):
    """z, and per element the sum of the products' magnitudes."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        z, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    return (z, mag) if bias is None else (z + bias, mag + np.abs(bias))


def gradients(g, x, w, add=None):
    """dx, dw, db from g, each with its magnitudes."""
    g, x, w = (np.asarray(a, dtype=np.float64) for a in (g, x, w))
    ag = np.abs(g)
    dx = (g @ w, ag @ np.abs(w)) if add is None else (g @ w + add, ag @ np.abs(w) + np.abs(add))
    return dx, (g.T @ x, ag.T @ np.abs(x)), (g.sum(0), ag.sum(0))


def cross_entropy(x, label, smoothing=0.0, lse2=0.0, mean=True, scale=1.0):
    """(total, loss, dlogits)."""
    x = np.asarray(x, dtype=np.float64)
    rows, n = x.shape
    loss, d = np.zeros(rows), np.zeros((rows, n))
    count = max(1, int((label >= 0).sum())) if mean else 1
    with np.errstate(all="ignore"):
        for r in range(rows):
            t = label[r]
            if t < 0:
                continue
            if t >= n:
                loss[r], d[r] = np.nan, np.nan
                continue
            # (by differences from the maximum: e - x_t would lose log sum beside a maximum of 2^53 or more)
            top = x[r].max()
            below = x[r] - top if np.isfinite(top) else np.full(n, np.nan)
            p = np.exp(below)
            log_sum = np.log(p.sum())
            e = top + log_sum
            loss[r] = log_sum + lse2 * e * e - ((1 - smoothing) * below[t] if smoothing < 1 else 0.0)
            if smoothing > 0:
                loss[r] -= smoothing * below.mean()
            q = (1 + 2 * lse2 * e) * p / p.sum() - smoothing / n
            q[t] -= 1 - smoothing
            d[r] = scale * q / count
    return loss.sum() / count, loss, d
