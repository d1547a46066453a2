"""Every tile shape of the products, its steady loop, divided contractions and launches of two shapes, against 64 bits on the GPU
(float64 library products).  tests/test_product_plan.py checks that these calls take them all.

Tolerances: of single products those of test_layers_gpu.py.  Orthogonalised updates by their Frobenius norm: as in
test_orthogonalize_accuracy.py with 2^-22 a step, sums being longer here.  (A wrong tile of the hundreds of one is off by far more.)"""
import numpy as np
import pytest

# ("product" | "linear" | "grad", rows, contraction, columns, bf16) and ("orthogonalize", rows, columns, bf16, count, steps, base)
CALLS = [
    ("product", 2239, 3698, 7265, True), ("product", 6455, 1623, 142, True), ("product", 5618, 825, 260, True),
    ("product", 2997, 2614, 134, False), ("product", 17, 8091, 60, True),
    ("linear", 856, 1795, 4907, True), ("linear", 3535, 990, 2322, True), ("linear", 313, 898, 3270, True),
    ("linear", 5785, 668, 134, False), ("linear", 5503, 3197, 361, False), ("linear", 525, 838, 7716, False),
    ("linear", 10, 2370, 18, True), ("linear", 6, 2519, 18, False),
    ("grad", 1759, 7742, 1149, True), ("grad", 1754, 623, 635, True), ("grad", 6, 42, 3142, True),
    ("grad", 780, 5596, 727, False), ("grad", 956, 159, 5444, False), ("grad", 239, 2181, 205, False),
    ("grad", 173, 82, 4411, False), ("grad", 1556, 38, 16, False),
    ("orthogonalize", 2858, 2964, True, 2, 1, False), ("orthogonalize", 3134, 2994, True, 1, 1, False),
    ("orthogonalize", 1450, 2113, False, 3, 1, False), ("orthogonalize", 1422, 3853, True, 1, 1, False),
    ("orthogonalize", 3774, 1113, False, 1, 2, False), ("orthogonalize", 1126, 2780, False, 3, 1, False),
    ("orthogonalize", 3125, 411, True, 3, 2, False), ("orthogonalize", 560, 2416, True, 3, 1, False),
    ("orthogonalize", 194, 1554, True, 3, 3, False), ("orthogonalize", 393, 624, True, 1, 3, False),
    ("orthogonalize", 421, 578, True, 1, 1, True), ("orthogonalize", 782, 206, True, 3, 1, False),
]


@pytest.fixture(scope="module")
def ctx():
    from paper_2606_09377_amd import Ctx
    return Ctx(0)


def near(got, want, mag, K):
    import torch
    tol = (4 + 2 * K ** 0.5) * 2.0 ** -23 * mag
    if got.dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    off = (got.double() - want).abs() - tol
    assert bool((off <= 0).all()), (float(off.max()), int((off > 0).sum()))


@pytest.mark.gpu
@pytest.mark.parametrize("call", [c for c in CALLS if c[0] != "orthogonalize"], ids=str)
def test_products(ctx, call):
    import torch
    kind, m, k, n, bf16 = call
    dt = torch.bfloat16 if bf16 else torch.float32
    g = torch.Generator("cuda").manual_seed(m + 3 * k + 5 * n)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    w = ctx.mx_quantize(normal(n, k))
    wv = ctx.mx_dequantize(w).double()
    x, b = normal(m, k).to(dt), normal(n)
    if kind == "grad":
        dy, y = normal(m, n).to(dt), normal(m, n).to(dt)
        dx, dw, db = ctx.mx_linear_grad(dy, x, w, y=y)
        d = torch.where(y > 0, dy, torch.zeros_like(dy)).double()
        dt_ = d.t().contiguous()
        near(dx, d @ wv, d.abs() @ wv.abs(), n)
        near(dw, dt_ @ x.double(), dt_.abs() @ x.double().abs(), m)
        near(db, d.sum(0), d.abs().sum(0), m)
        return
    if kind == "product":
        q = ctx.mx_quantize(x)
        x = ctx.mx_dequantize(q)
        y = ctx.mx_product(q, w, bias=b, dtype=dt)
    else:
        y = ctx.mx_linear(x, w, bias=b)
    wt = wv.t().contiguous()
    near(y, x.double() @ wt + b.double(), x.double().abs() @ wt.abs() + b.double().abs(), k)


@pytest.mark.gpu
@pytest.mark.parametrize("call", [c for c in CALLS if c[0] == "orthogonalize"], ids=str)
def test_updates(ctx, call):
    import torch
    _, m, n, bf16, count, steps, with_base = call
    A, B, C = 3.4445, -4.7750, 2.0315
    gen = torch.Generator("cuda").manual_seed(m + n)
    g = (torch.randn((count, m, n), generator=gen, device="cuda") * 1e-3).to(torch.bfloat16 if bf16 else torch.float32)
    base = torch.randn((count, m, n), generator=gen, device="cuda") if with_base else None
    out = torch.empty((count, m, n), device="cuda")
    ctx.orthogonalize(g, steps=steps, coefficients=(A, B, C), gain=0.5, base=base, keep=0.9, out=out)
    for i in range(count):
        x = g[i].double()
        x = x.t().contiguous() if m > n else x
        x = x / (x.norm() + 1e-7)
        bound = 0.0
        for s in range(steps):
            bound += 2.0 ** -22 * float(x.norm()) * A ** (steps - s)
            gram = x @ x.t().contiguous()
            x = A * x + (B * gram + C * (gram @ gram)) @ x
        want = 0.5 * (x.t() if m > n else x)
        if with_base:
            want = want + 0.9 * base[i].double()
            bound += 2.0 ** -23 * float(want.norm())
        off = (out[i].double() - want).norm()
        assert float(off) <= bound, (float(off), bound)
        # and no single element far off: a tile's share of the norm
        assert float((out[i].double() - want).abs().max()) <= bound / np.sqrt(min(m, n))


# one, two and four row blocks of weights a workgroup, several rounds of them; rows that fit LDS together, and in slices
@pytest.mark.gpu
@pytest.mark.parametrize("n", [1000, 8208, 33000, 66000])
@pytest.mark.parametrize("k", [300, 9000])
@pytest.mark.parametrize("kind,m", [("float32", 1), ("float32", 5), ("bfloat16", 1), ("bfloat16", 8), ("4 bits", 1), ("4 bits", 16)])
def test_few_rows(ctx, kind, m, k, n):
    import torch
    g = torch.Generator("cuda").manual_seed(n + k + m)
    w = ctx.mx_quantize(torch.randn((n, k), generator=g, device="cuda"))
    x, b = torch.randn((m, k), generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    if kind == "4 bits":
        q = ctx.mx_quantize(x)
        x, y = ctx.mx_dequantize(q), ctx.mx_product(q, w, bias=b)
    else:
        x = x.to(getattr(torch, kind))
        y = ctx.mx_linear(x, w, bias=b)
    wt = ctx.mx_dequantize(w).double().t().contiguous()
    near(y, x.double() @ wt + b.double(), x.double().abs() @ wt.abs() + b.double().abs(), k)
    del wt, w
    torch.cuda.empty_cache()
