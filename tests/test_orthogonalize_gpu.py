"""Newton-Schulz orthogonalisation on the GPU against 64 bits.

Tolerances (Frobenius norm, relative).  A step's map s -> s (a + b s^2 + c s^4) of the singular values has a slope of
at most 3.9 in [0, 1.2], so what a step's rounding adds, e of its result, grows by at most that in every
later one: five steps give e (1 + 3.9 + ... + 3.9^4) = 310 e.  float32 products leave 2^-22 (three roundings of
2^-24, and the sums); those of 16 bits 2^-16 (two factors rounded by 2^-16 at most, 2^-17 in the mean
square, which is what the norm sees); a bf16 result is rounded by 2^-9 in the mean square more."""
import numpy as np
import pytest

from oracle import layers64 as o64

pytestmark = pytest.mark.gpu

TOL = {"float32": 310 * 2.0 ** -22, "bfloat16": 310 * 2.0 ** -16 + 2.0 ** -9}


@pytest.fixture(scope="module")
def ctx():
    from paper_2606_09377_amd import Ctx
    return Ctx(0)


def host(t):
    return t.double().cpu().numpy()


def off(got, want):
    return np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300)


SHAPES = [(1, 1), (1, 40), (40, 1), (7, 31), (32, 32), (33, 65), (65, 33), (100, 784), (784, 100), (128, 128), (300, 257),
          (513, 1000), (1024, 1024), (1500, 777)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,n", SHAPES)
def test_against_64_bits(ctx, m, n, dtype):
    import torch
    rng = np.random.default_rng(m + 3 * n)
    g = torch.as_tensor(rng.standard_normal((m, n)) * 1e-3, dtype=torch.float32).to(getattr(torch, dtype)).cuda()
    out = ctx.orthogonalize(g)
    assert out.dtype == g.dtype
    assert off(host(out), o64.orthogonalize(host(g))) <= TOL[dtype]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_few_directions(ctx, dtype):
    """A gradient of a small batch: 8 directions of 300, the rest zero up to the type's rounding."""
    import torch
    rng = np.random.default_rng(8)
    g = torch.as_tensor(rng.standard_normal((300, 8)) @ rng.standard_normal((8, 500)), dtype=torch.float32)
    g = g.to(getattr(torch, dtype)).cuda()
    assert off(host(ctx.orthogonalize(g)), o64.orthogonalize(host(g))) <= TOL[dtype]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,n", [(50, 70), (70, 50), (200, 130), (2048, 2048)])
def test_batches_strides_and_base(ctx, m, n, dtype):
    import torch
    rng = np.random.default_rng(m)
    dt = getattr(torch, dtype)
    buf = torch.full((3, m + 2, n + 5), float("nan"), dtype=dt, device="cuda")
    g = buf[:, 1:m + 1, 3:n + 3]
    g.copy_(torch.as_tensor(rng.standard_normal((3, m, n)), dtype=torch.float32))
    base = torch.as_tensor(rng.standard_normal((3, m, n)), dtype=torch.float32).cuda()
    out = ctx.orthogonalize(g, gain=-0.5, base=base, keep=0.9)
    assert out.dtype == torch.float32
    alone = [ctx.orthogonalize(g[i], gain=-0.5, base=base[i], keep=0.9) for i in range(3)]
    for i in range(3 if m < 1000 else 1):
        x = o64.orthogonalize(host(g[i]))
        want = 0.9 * host(base[i]) - 0.5 * x
        tol = 0.5 * TOL["float32"] * np.linalg.norm(x) + 2.0 ** -23 * np.linalg.norm(want)
        assert np.linalg.norm(host(out[i]) - want) <= tol
        assert np.linalg.norm(host(alone[i]) - want) <= tol
    same = base.clone()
    ctx.orthogonalize(g, gain=-0.5, base=same, keep=0.9, out=same)
    assert torch.equal(same, out)


@pytest.mark.parametrize("steps", [1, 5])
def test_results_of_the_other_type(ctx, steps):
    import torch
    rng = np.random.default_rng(10 + steps)
    g = torch.as_tensor(rng.standard_normal((120, 200)), dtype=torch.float32).cuda()
    for src, dst in (("float32", "bfloat16"), ("bfloat16", "float32")):
        x = g.to(getattr(torch, src))
        out = torch.empty(g.shape, dtype=getattr(torch, dst), device="cuda")
        ctx.orthogonalize(x, steps=steps, out=out)
        assert off(host(out), o64.orthogonalize(host(x), steps)) <= TOL[dst]


@pytest.mark.parametrize("steps", [1, 2, 7])
def test_steps_and_coefficients(ctx, steps):
    import torch
    rng = np.random.default_rng(steps)
    g = torch.as_tensor(rng.standard_normal((90, 120)), dtype=torch.float32).cuda()
    co = (1.5, -0.5, 0.0)   # slope at most 1.5 in [0, 1]
    want = o64.orthogonalize(host(g), steps, co, 0.0)
    got = ctx.orthogonalize(g, steps=steps, coefficients=co, eps=0.0)
    assert off(host(got), want) <= 2.0 ** -22 * sum(1.5 ** i for i in range(steps))


def test_zero_tiny_huge_and_non_finite(ctx):
    import torch
    z = torch.zeros((40, 60), device="cuda")
    assert not ctx.orthogonalize(z).any()
    rng = np.random.default_rng(0)
    g = rng.standard_normal((40, 60)).astype(np.float32)
    want = o64.orthogonalize(g, eps=0.0)
    for s in (1e-30, 1e30):   # squares beyond float32
        assert off(host(ctx.orthogonalize(torch.as_tensor(g * np.float32(s)).cuda(), eps=0.0)), want) <= 2 * TOL["float32"]
    for v in (np.nan, np.inf):
        h = g.copy()
        h[3, 4] = v
        assert torch.isnan(ctx.orthogonalize(torch.as_tensor(h).cuda())).all()
        assert torch.isnan(ctx.orthogonalize(torch.as_tensor(h).bfloat16().cuda())).all()
    assert not ctx.orthogonalize(z.bfloat16()).any()
    for s in (1e-37, 1e-30, 1e30, 1e37):   # the norm's power of two is taken out of a bf16 update exactly
        b = torch.as_tensor(g * np.float32(s)).bfloat16().cuda()
        out = ctx.orthogonalize(b, eps=0.0, out=torch.empty((40, 60), device="cuda"))
        assert off(host(out), o64.orthogonalize(host(b), eps=0.0)) <= TOL["float32"]
