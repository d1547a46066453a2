"""Every kernel of the float layers' products, with its steady loop, contractions that end inside a stage, divided ones and tiles left to another shape, against 64
bits on the GPU (float64 library products).  tests/test_dense_launches.py checks that these calls take them all.

Tolerances: those of test_dense_gpu.py."""
import pytest

# ("linear", rows, k, n, bf16, pitch, relu, dropout, residual, z, results of the other type)
# ("grad", rows, k, n, bf16, pitch, relu, dropout, which of dx 1, dw 2 and db 4, dw of the other type)
CALLS = [
    ("grad", 6483, 8, 8, 1, 0, 1, 0, 7, 1), ("grad", 461, 1, 13490, 1, 0, 1, 1, 7, 0), ("grad", 2, 32, 7688, 1, 8, 0, 0, 7, 1),
    ("grad", 990, 3, 5456, 0, 0, 1, 1, 7, 1), ("grad", 855, 8, 752, 1, 8, 1, 1, 7, 1), ("linear", 20, 4688, 8, 1, 8, 1, 0, 0, 0, 1),
    ("grad", 2, 54688, 40, 1, 0, 0, 0, 7, 1), ("grad", 1075, 4562, 4, 1, 8, 1, 0, 7, 0), ("grad", 1, 1, 853, 1, 0, 0, 1, 7, 1),
    ("grad", 638, 16, 8576, 1, 8, 0, 1, 2, 1), ("grad", 515, 18888, 40, 0, 8, 0, 0, 7, 1), ("linear", 19, 1040, 8, 1, 0, 1, 1, 0, 0, 1),
    ("linear", 34, 872, 8, 1, 8, 1, 1, 0, 1, 1), ("linear", 68, 680, 8, 1, 0, 1, 0, 0, 1, 1), ("grad", 290, 4864, 523, 1, 0, 1, 1, 7, 0),
    ("linear", 66, 408, 5640, 1, 8, 1, 1, 0, 1, 1), ("linear", 2, 1504, 5736, 1, 0, 1, 0, 0, 1, 0), ("linear", 284, 280, 6800, 1, 8, 1, 1, 0, 1, 0),
    ("grad", 678, 4736, 256, 1, 0, 0, 0, 7, 0), ("linear", 1000, 657, 1200, 1, 3, 1, 1, 0, 0, 0), ("grad", 218, 36836, 93, 0, 0, 1, 0, 7, 1),
    ("grad", 1, 8, 2, 1, 8, 0, 1, 7, 1), ("grad", 225, 1, 1, 0, 8, 1, 1, 7, 0), ("grad", 1, 277, 9761, 0, 8, 1, 1, 7, 1),
    ("linear", 483, 664, 3416, 1, 0, 0, 0, 0, 0, 0), ("grad", 100, 8416, 848, 1, 8, 1, 1, 7, 1), ("grad", 1, 2, 2, 0, 8, 0, 1, 7, 0),
    ("grad", 18, 2, 1, 0, 3, 0, 1, 7, 1), ("grad", 2, 8, 648, 1, 0, 1, 0, 1, 1), ("grad", 757, 8, 3, 1, 0, 1, 0, 2, 1),
    ("grad", 3, 42800, 80, 0, 8, 1, 0, 7, 1), ("linear", 2101, 547, 2229, 0, 3, 0, 1, 0, 0, 1), ("grad", 173, 35151, 66, 0, 8, 0, 1, 7, 1),
    ("linear", 1, 1, 1, 1, 0, 0, 0, 1, 1, 0), ("grad", 1, 1, 1, 0, 0, 0, 0, 1, 1), ("grad", 1, 1, 1, 1, 3, 1, 0, 2, 0),
    ("linear", 1, 2, 1, 0, 8, 1, 1, 0, 1, 1), ("grad", 1, 2, 2, 0, 8, 0, 1, 1, 1), ("linear", 19, 1, 1, 1, 0, 1, 1, 1, 0, 0),
    ("linear", 24, 1, 1, 0, 8, 0, 0, 0, 1, 1), ("linear", 33, 1, 1, 0, 3, 1, 0, 1, 1, 0), ("linear", 47, 1, 1, 1, 0, 1, 0, 0, 0, 0),
    ("grad", 18, 3, 2, 0, 3, 0, 0, 1, 1), ("grad", 37, 2, 1, 0, 0, 1, 0, 7, 0), ("grad", 43, 2, 1, 0, 3, 0, 0, 1, 1),
    ("grad", 21, 2, 4, 0, 0, 0, 1, 5, 0), ("grad", 47, 2, 1, 0, 8, 0, 1, 5, 0), ("linear", 21, 8, 3, 1, 8, 1, 1, 1, 1, 0),
    ("linear", 41, 8, 1, 1, 0, 1, 0, 1, 1, 0), ("linear", 72, 8, 2, 1, 8, 1, 0, 1, 0, 1), ("linear", 1, 3805, 1, 0, 3, 1, 1, 0, 0, 0),
    ("linear", 1, 4193, 1, 1, 3, 1, 1, 1, 0, 1), ("linear", 19, 1649, 1, 0, 0, 1, 1, 1, 1, 1), ("linear", 34, 1267, 2, 0, 0, 1, 1, 0, 0, 0),
    ("linear", 21, 1889, 3, 1, 0, 0, 1, 0, 0, 0), ("grad", 1, 1, 24000, 1, 3, 0, 0, 7, 1), ("linear", 35, 1650, 3, 1, 3, 1, 0, 1, 0, 1),
    ("linear", 5, 2, 12110, 1, 0, 0, 0, 0, 1, 1), ("linear", 10, 1, 8493, 0, 0, 0, 1, 1, 1, 0), ("linear", 17, 2, 9242, 1, 8, 0, 1, 0, 0, 0),
    ("grad", 2, 8, 18472, 1, 0, 0, 1, 7, 0), ("linear", 22, 2, 8300, 0, 3, 1, 0, 1, 0, 1), ("linear", 37, 2, 9281, 1, 8, 0, 1, 1, 1, 0),
    ("linear", 44, 1, 8736, 0, 3, 1, 0, 1, 1, 1), ("linear", 4200, 40, 88, 1, 0, 0, 1, 0, 0, 0), ("linear", 17, 8, 37840, 1, 8, 0, 1, 1, 1, 0),
    ("grad", 42, 16632, 8, 1, 0, 1, 0, 5, 0), ("linear", 682, 808, 22176, 1, 8, 1, 0, 0, 0, 0), ("grad", 206, 3, 34986, 1, 8, 1, 1, 6, 0),
    ("linear", 2, 144, 58464, 1, 8, 1, 1, 1, 1, 0), ("grad", 5, 57384, 264, 1, 0, 0, 0, 7, 1), ("grad", 868, 52208, 152, 1, 0, 0, 0, 7, 0),
    ("grad", 906, 16392, 992, 1, 0, 0, 0, 7, 1), ("linear", 1073, 814, 12342, 1, 0, 1, 1, 0, 0, 0), ("linear", 2629, 531, 3145, 1, 0, 1, 1, 1, 1, 0),
    ("linear", 4625, 463, 2115, 0, 0, 0, 0, 0, 0, 1), ("linear", 181, 602, 36706, 1, 3, 1, 0, 1, 1, 0),
    ("linear", 1756, 720, 4960, 1, 8, 1, 0, 1, 1, 0), ("grad", 6954, 1256, 920, 1, 0, 1, 1, 7, 1), ("grad", 2009, 5120, 1760, 1, 0, 1, 0, 7, 1),
    ("linear", 1850, 1680, 5248, 1, 3, 1, 1, 0, 0, 0), ("linear", 3977, 1912, 2376, 1, 0, 1, 1, 0, 0, 0),
    ("grad", 1480, 5464, 1752, 1, 8, 1, 0, 7, 0), ("linear", 5556, 1874, 4752, 1, 8, 0, 1, 0, 0, 0), ("grad", 2871, 7224, 2552, 1, 0, 1, 1, 7, 0),
    ("linear", 4333, 3048, 4552, 1, 8, 0, 1, 1, 0, 0), ("linear", 4001, 4104, 4104, 1, 0, 1, 1, 1, 1, 0),
    ("grad", 4001, 4104, 4104, 1, 8, 1, 1, 7, 0), ("linear", 2500, 4099, 4100, 0, 0, 1, 1, 1, 0, 0), ("grad", 4100, 2050, 2049, 0, 3, 1, 1, 7, 0),
    ("linear", 64, 8192, 8192, 1, 0, 0, 0, 1, 0, 0), ("linear", 64, 8192, 8200, 0, 0, 1, 0, 0, 0, 0),
]
E = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    from paper_2606_09377_amd import Ctx
    return Ctx(0)


def sums(mag, K):
    return (4 + 2 * K ** 0.5) * 2.0 ** -23 * mag


def near(got, want, tol):
    import torch
    half = E if got.dtype == torch.float32 else 2.0 ** -8
    off = (got.double() - want).abs() - (tol + half * (want.abs() + tol))
    assert bool((off <= 0).all()), (float(off.max()), int((~(off <= 0)).sum()), torch.nonzero(~(off <= 0))[:4].tolist())


def product(a, b):
    """a b^T, and the same of magnitudes."""
    bt = b.t().contiguous()
    return a @ bt, a.abs() @ bt.abs()


@pytest.mark.gpu
@pytest.mark.parametrize("call", CALLS, ids=str)
def test_products(ctx, call):
    import torch
    from paper_2606_09377_amd import Dropout
    kind, m, k, n, bf16, pitch, relu, drop = call[:8]
    types = (torch.float32, torch.bfloat16)
    dt, out = types[bf16], types[bf16 ^ call[-1]]
    g = torch.Generator("cuda").manual_seed(m + 3 * k + 5 * n)

    def normal(r, c, dtype=dt, scale=1.0):
        t = torch.full((r, c + pitch), float("nan"), device="cuda", dtype=dtype)[:, :c]
        return t.copy_(torch.randn((r, c), generator=g, device="cuda") * scale)
    act, d = "relu" if relu else "none", Dropout(0.25, m * k, n) if drop else None
    mask = ctx.dropout(torch.ones((m, n), device="cuda"), d).double() if drop else 1.0
    x, w = normal(m, k), normal(n, k, scale=k ** -0.5)
    if kind == "linear":
        residual, keep_z = call[8:10]
        b, r = torch.randn(n, generator=g, device="cuda"), normal(m, n, out) if residual else None
        y = torch.full((m, n + pitch), 7.0, device="cuda", dtype=out)
        got = ctx.linear(x, w, bias=b, act=act, dropout=d, residual=r, keep_z=bool(keep_z), out=y[:, :n])
        z, mag = product(x.double(), w.double())
        z, tol = z + b.double(), sums(mag + b.double().abs(), k)
        if keep_z:
            near(got[1], z, tol)
        want = (z.clamp_min(0) if relu else z) * mask
        tol = tol * mask + 2 * E * want.abs()
        if residual:
            want = want + r.double()
            tol = tol + E * want.abs()
        near(y[:, :n], want, tol)
        assert bool((y[:, n:] == 7.0).all())
        return
    need = call[8]
    dy, z, add = normal(m, n), normal(m, n), normal(m, k) if drop else None
    dx, dw, db = ctx.linear_grad(dy, x, w, z=z if relu else None, act=act, dropout=d, add=add, need=(need & 1 > 0, need & 2 > 0, need & 4 > 0), dw_dtype=out)
    v = dy.double() * mask
    if relu:
        v = torch.where(z > 0, v, torch.zeros_like(v))
    if need & 1:
        want, mag = product(v, w.double().t())
        if drop:
            want, mag = want + add.double(), mag + add.double().abs()
        near(dx, want, sums(mag, n) + 2 * E * mag)
    if need & 2:
        want, mag = product(v.t().contiguous(), x.double().t())
        near(dw, want, sums(mag, m) + 2 * E * mag)
    if need & 4:
        near(db, v.sum(0), sums(v.abs().sum(0), m) + 2 * E * v.abs().sum(0))
