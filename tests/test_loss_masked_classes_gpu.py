"""Cross entropy on the GPU where classes are masked by large negative numbers that are neither -infinity nor the type's lowest value, and
where whole rows lie far from 0, in every way that rows are divided (vcr_cross_entropy against 64 bits).

Tolerances.  x - m is exact or rounds by 2^-24 of itself, its product with log2 e (itself off by 2^-26) by as much again, and the
exponential is within two units of its own: exp(x - m) is off by (2 |x - m| + 4) 2^-24 of itself, and is 0 where it would be less than 2^-126.  The
exponentials that count at all have |x - m| < 88; with the additions of n of them (by threads, then pairwise) their sum is off by
(2 R + 16 + sqrt(n)) 2^-24 of itself, R the largest |x - m| up to 88: `each` of the logarithm.  A loss, (m - x_t) + log sum + c e^2 with
e = m + log sum, rounds each term and addition: 8 2^-24 of the terms' magnitudes.  A gradient's exponential and its factor, 1 / sum among them, are
each off by `each` and a few roundings of the terms, the exponent's change of 1 + 2 c e, and round to the type at last."""
import numpy as np
import pytest

from oracle import dense64 as o64

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    from paper_2606_09377_amd import Ctx
    return Ctx(0)


def host(t):
    return t.double().cpu().numpy()


def check(ctx, x, label, dtype, shift=0, lse2=0.0, mean=True):
    """x (numpy) and label through the call, against the oracle."""
    import torch
    rows, n = x.shape
    t = torch.empty((rows, n + shift), dtype=getattr(torch, dtype), device="cuda")[:, shift:]
    t.copy_(torch.as_tensor(x, dtype=torch.float32))
    total, loss, d = (host(v) for v in ctx.cross_entropy(t, torch.as_tensor(label).cuda(), lse2=lse2, mean=mean))
    v = host(t)
    want_total, want, want_d = o64.cross_entropy(v, label, lse2=lse2, mean=mean)
    assert np.isfinite(want).all() and np.isfinite(want_d).all()
    top = v.max(1)
    below = top[:, None] - v
    R = np.where(below < 88, below, 0.0).max(1)
    each = (2 * R + 16 + np.sqrt(n)) * E
    logs = np.log(np.exp(-below).sum(1))
    e = np.abs(top + logs)
    off = (top - v[np.arange(rows), label]) + np.abs(logs)
    e_tol = each + 2 * E * (np.abs(top) + np.abs(logs))
    tol = 8 * E * (off + lse2 * e * e) + 2 * each + lse2 * 2 * e * e_tol
    bad = ~(np.abs(loss - want) <= tol)
    assert not bad.any(), (np.flatnonzero(bad)[:8], loss[bad][:8], want[bad][:8], tol[bad][:8])
    count = rows if mean else 1
    assert abs(float(total) - want_total) <= (tol.sum() + (8 + np.sqrt(rows)) * E * np.abs(want).sum()) / count
    hit = np.arange(n) == label[:, None]
    q = np.abs(want_d * count + hit)   # (1 + 2 c e) p
    tol = (3 * each[:, None] * q + 4 * E * (q + hit) + (2 * lse2 * e_tol)[:, None] * q + 2.0 ** -125) / count
    tol = tol + HALF[dtype] * (np.abs(want_d) + tol)
    bad = ~(np.abs(d - want_d) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], d[bad][:4], want_d[bad][:4], tol[bad][:4])


# one workgroup for everything (8 lanes a row, a wave a row), waves, workgroups of 256, 512 and 1024, rows beyond the registers, rows divided
PLANS = [(200, 30), (30, 60), (9, 200), (32, 1000), (300, 200), (40, 1000), (40, 4000), (40, 8000), (40, 16000), (40, 32000), (40, 50000), (70, 140000), (3, 100001)]
MASKS = (-1e4, -16777216.0, -1.6e7, -1e9, -2e9, -5e9, -1e10, -1e20, -1e30, -1e36, -9.9e36, -1.1e37)


def cases(n):
    """(name, f(row of normal logits) -> a row and its label)"""
    a, b = n // 4 // 8 * 8, max(n // 4 // 8 * 8 + 8, n // 2)
    for hide in MASKS:
        def stretch(x, lo, hi, at, hide=hide):
            x[lo:hi] = hide
            return x, at
        yield lambda x, s=stretch: s(x, n - max(8, n // 3), n, 1)              # padding classes, at the end
        yield lambda x, s=stretch: s(x, 0, max(8, n // 3), n - 1)              # the first ones
        yield lambda x, s=stretch: s(x, a, b, 0)                               # whole pieces in the middle
        yield lambda x, s=stretch: s(x, a, b, a)                               # the same, with a masked label
        yield lambda x, s=stretch: s(x, n // 3, n // 3 + 1, n // 2)            # a single one

        def others(x, hide=hide):
            x[1::2] = hide
            return x, n // 4 * 2
        yield others

        def all_but_one(x, hide=hide):
            x[:], x[n // 2] = hide, 0.5
            return x, n // 2
        yield all_but_one

        def whole(x, hide=hide):
            x[:] = hide
            return x, n // 3
        yield whole

        def above(x, hide=hide):   # classes far above the others
            x[[1, n // 2, n - 1]] = -hide
            return x, n // 2
        yield above


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,n", PLANS)
def test_masks_by_large_numbers(ctx, rows, n, dtype):
    rng = np.random.default_rng(rows + n)
    each = list(cases(n))
    for first in range(0, len(each), rows):
        x, label = 3 * rng.standard_normal((rows, n)), np.zeros(rows, dtype=np.int64)
        for r in range(rows):
            x[r], label[r] = each[(first + r) % len(each)](x[r])
        check(ctx, x, label, dtype, shift=first // rows % 3)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,n", PLANS)
def test_masks_beside_the_squared_sum(ctx, rows, n, dtype):
    """(without rows of large maxima, whose squares leave float32)"""
    rng = np.random.default_rng(rows * n)
    x, label = 3 * rng.standard_normal((rows, n)), rng.integers(0, n // 2, rows)
    for r in range(rows):
        x[r, n - max(8, n // 3):] = MASKS[(r * 5 + n) % len(MASKS)]
    check(ctx, x, label, dtype, lse2=1e-3, mean=False)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,n", PLANS)
def test_rows_far_from_zero(ctx, rows, n, dtype):
    """Rows of a large number and its neighbours in the type, on both sides of where the exponential changes its form."""
    rng = np.random.default_rng(3 * rows + n)
    bits = 24 if dtype == "float32" else 8
    far = [s * v for v in (1e3, 1e6, 2.0 ** 23, 2.0 ** 24 - 2, 2.0 ** 24, 2.0 ** 24 + 4, 1e8, 2.0 ** 30, 3e9, 1e10, 1e20, 1e30) for s in (1, -1)]
    for first in range(0, len(far), rows):
        x = np.empty((rows, n))
        for r in range(rows):
            v = far[(first + r) % len(far)]
            x[r] = v + rng.integers(-4, 5, n) * 2.0 ** (np.floor(np.log2(abs(v))) + 1 - bits)
        check(ctx, x, rng.integers(0, n, rows), dtype, shift=first // rows % 2, mean=first % 2 == 0)
