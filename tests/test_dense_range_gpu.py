"""Small float32 operands of the float layers' products (vcr_linear, vcr_linear_grad): exact down to 2^-110, below that each is rounded by up to 2^-134 (what a
bf16 part, a multiple of 2^-133, cannot hold).  Tolerances: those of test_dense_gpu.py, and 2^-134 times the other operand's magnitudes where values are smaller."""
import numpy as np
import pytest

from oracle import dense64 as o64
from tests.test_dense_gpu import ctx, dev, host, near, sums  # noqa: F401

pytestmark = pytest.mark.gpu


def values(rng, shape, power):
    """24 random bits each, of one binary order (below 2^-126 as many as float32 has there)."""
    return np.ldexp(rng.integers(2 ** 23, 2 ** 24, shape) * rng.choice((-1.0, 1.0), shape), power - 23).astype(np.float32)


@pytest.mark.parametrize("power", [-100, -110, -118, -126, -140])
@pytest.mark.parametrize("m,k,n", [(1, 200, 40), (40, 130, 70), (300, 200, 130)])
def test_small_operands(ctx, m, k, n, power):  # noqa: F811
    rng = np.random.default_rng(m - power)
    lost = 2.0 ** -134 if power < -110 else 0.0
    for small in (0, 1):   # the left operand of a product, the right one
        a, b = ((power, 100) if small == 0 else (100, power))
        x, w = values(rng, (m, k), a), values(rng, (n, k), b)
        z, mag = o64.linear(x, w)
        near(ctx.linear(dev(x), dev(w)), z, sums(mag, k) + lost * 2.0 ** 101 * k)
        dy, w, x = values(rng, (m, n), a), values(rng, (n, k), b), values(rng, (m, k), b)
        (dx, dx_mag), (dw, dw_mag), _ = o64.gradients(dy, x, w)
        got = ctx.linear_grad(dev(dy), dev(x), dev(w))
        near(got[0], dx, sums(dx_mag, n) + lost * 2.0 ** 101 * n)
        near(got[1], dw, sums(dw_mag, m) + lost * 2.0 ** 101 * m)
