"""Few rows of float layers whose contraction is divided among workgroups, and gradients of few rows on wide layers, against 64
bits.  Tolerances as in test_dense_gpu.py: parts are float32 sums, joined by float32 additions."""
import numpy as np
import pytest

from oracle import dense64 as o64
from tests.test_dense_gpu import ctx, dev, host, near, sums, test_linear as linear, test_linear_grad as linear_grad  # noqa: F401

pytestmark = pytest.mark.gpu


# (some in one part beside those in several; columns that end inside a group, a chunk and eight; the last part short)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,k,n", [(1, 8192, 256), (1, 9001, 40), (2, 4100, 500), (5, 70001, 16), (16, 8193, 96), (17, 2079, 33), (33, 2100, 250),
                                   (48, 6152, 700), (64, 30000, 17), (64, 2048, 2049)])
def test_few_rows_in_parts(ctx, m, k, n, dtype):  # noqa: F811
    linear(ctx, m, k, n, dtype)


@pytest.mark.parametrize("dtype,pitch", [("float32", 0), ("bfloat16", 0), ("bfloat16", 3)])
@pytest.mark.parametrize("m", [1, 16, 64])
def test_parts_over_the_residual(ctx, m, dtype, pitch):  # noqa: F811
    import torch
    rng = np.random.default_rng(m)
    k, n = 9000, 200
    x, w, r = (dev(rng.standard_normal(s), dtype, pitch) for s in ((m, k), (n, k), (m, n)))
    z, mag = o64.linear(host(x), host(w))
    want = z + host(r)
    apart = ctx.linear(x, w, residual=r)
    got = ctx.linear(x, w, residual=r, out=r)
    assert got.data_ptr() == r.data_ptr() and torch.equal(got, apart)
    near(got, want, sums(mag, k) + 2.0 ** -24 * np.abs(want), dtype)
    assert all(torch.equal(ctx.linear(x, w), ctx.linear(x, w)) for _ in range(3))


# dw beside dx in a launch, and by its own plan; narrow layers, whose dx is taken by tiles
@pytest.mark.parametrize("m,k,n", [(5, 6400, 1100), (64, 6144, 700), (33, 6143, 1200), (1, 2000, 5000), (64, 8200, 90), (40, 96, 6000), (64, 300, 4100)])
def test_gradients_of_few_rows_on_wide_layers(ctx, m, k, n):  # noqa: F811
    linear_grad(ctx, m, k, n, "float32")


def test_operands_beside_nan(ctx):  # noqa: F811
    """bf16 matrices as they are stored end inside a stage of the contraction, with NaN behind every row and after the last."""
    import torch
    rng = np.random.default_rng(5)
    for m, k, n in ((8, 72, 40), (70, 40, 136), (130, 8, 264), (300, 1032, 136), (520, 200, 520)):
        def held(r, c):
            buf = torch.full((r + 3, c + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
            t = buf[1:r + 1, 8:c + 8]
            t.copy_(torch.as_tensor(rng.standard_normal((r, c)), dtype=torch.float32).bfloat16())
            return t
        x, w, dy = held(m, k), held(n, k), held(m, n)
        z, mag = o64.linear(host(x), host(w))
        near(ctx.linear(x, w), z, sums(mag, k), "bfloat16")
        for t, (v, g), terms, o in zip(ctx.linear_grad(dy, x, w), o64.gradients(host(dy), host(x), host(w)), (n, m, m), ("bfloat16", "bfloat16", "float32")):
            near(t, v, sums(g, terms) + 2.0 ** -23 * g, o)


@pytest.mark.parametrize("n", [(1 << 22) - 8, (1 << 22) + 16])
def test_gradients_of_very_many_outputs(ctx, n):  # noqa: F811
    """g's rows written out for the tiles reach their offsets' 32 bits at 2^22 columns."""
    import torch
    g = torch.Generator("cuda").manual_seed(3)
    m, k = 3, 8
    x, dy, z = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((m, k), (m, n), (m, n)))
    _, dw, db = ctx.linear_grad(dy, x, None, z=z, act="relu", need=(False, True, True))
    at = torch.cat([torch.arange(40), torch.arange(n // 2, n // 2 + 40), torch.arange(n - 40, n)]).cuda()
    (_, (want, mag), (b, b_mag)) = o64.gradients(host(dy[:, at]) * (host(z[:, at]) > 0), host(x), np.zeros((len(at), k)))
    near(dw[at], want, sums(mag, m), "bfloat16")
    near(db[at], b, sums(b_mag, m))


@pytest.mark.parametrize("m,k,n", [(1, 200, 48), (5, 9000, 40), (16, 300, 96), (33, 130, 70), (64, 2500, 33), (300, 200, 100)])
def test_values_that_round_to_infinity_in_bf16(ctx, m, k, n):  # noqa: F811
    """Finite float32 values of more than bf16's largest take part with all their bits, beside infinite ones that reach their own results alone."""
    rng = np.random.default_rng(k)
    x, w, dy = rng.standard_normal((m, k)), 1e-20 * rng.standard_normal((n, k)), 1e-20 * rng.standard_normal((m, n))
    x[0, 3], x[m - 1, k - 1], x[m // 2, k // 2] = 3.4e38, -3.396e38, 3.4028234e38
    tx, tw = dev(x), dev(w)
    z, mag = o64.linear(host(tx), host(tw))
    near(ctx.linear(tx, tw), z, sums(mag, k))
    w = rng.standard_normal((n, k))
    w[0, 3], w[n - 1, k - 1], w[n // 2, k // 2] = 3.4e38, -3.396e38, 3.4028234e38
    tw, tg = dev(w), dev(dy)
    (want, mag), _, _ = o64.gradients(host(tg), host(tx), host(tw))
    near(ctx.linear_grad(tg, None, tw, need=(True, False, False))[0], want, sums(mag, n))
    w[n // 3, 7] = np.inf
    tw = dev(w)
    got = host(ctx.linear_grad(tg, None, tw, need=(True, False, False))[0])
    assert np.array_equal(got[:, 7], np.sign(dy[:, n // 3]) * np.inf)
    rest = np.arange(k) != 7
    assert (np.abs(got - want)[:, rest] <= (sums(mag, n) + 2.0 ** -24 * (np.abs(want) + sums(mag, n)))[:, rest]).all()


# an odd last column, one column alone, and contractions that end inside a chunk
@pytest.mark.parametrize("m,k,n", [(3, 1, 70), (3, 2, 33), (20, 3, 31), (64, 33, 1), (64, 65, 45), (7, 95, 130)])
def test_gradients_of_few_rows_of_odd_widths(ctx, m, k, n):  # noqa: F811
    linear_grad(ctx, m, k, n, "float32")
