"""Layers in float on the GPU (vcr_linear, vcr_linear_grad) against 64 bits.

Tolerances.  A product of bf16 values is exact in float32, of two float32 values off by at most 1.65 2^-24 of itself.  A float32
sum of K terms, in any order, each addition rounded or cut to 24 bits (2^-23), is off by about sqrt(K) 2^-23 of the sum of
magnitudes at random; (4 + 2 sqrt(K)) 2^-23 of it is allowed for z and for the gradients' sums.  What follows z:
  - an activation is off by its slope (at most 1.13) times z's, and a few roundings of its own value (16 2^-24 of |z|, which is
    no less than the value; exp and erfc are within 2 units in the last place, and each has one or two roundings around it);
  - dropout multiplies both by its factor, whose own rounding and the product's are 2 2^-24 of the value;
  - the residual's addition rounds by 2^-24 of the sum.
A slope is off by 2^-20: two terms of at most 1.13 and 0.45, each within 8 units in the last place.  With bf16 operands and a
smooth activation g is rounded to bf16: 2^-8 of itself (half a unit).  Results in bf16 round by 2^-8 of themselves."""
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


def dev(a, dtype="float32", pitch=0, shift=0):
    """a on the GPU, its rows `pitch` elements longer and shifted by `shift` elements."""
    import torch
    t = torch.as_tensor(np.ascontiguousarray(a), dtype=torch.float32).to(getattr(torch, dtype))
    buf = torch.full((t.shape[0], t.shape[1] + pitch + shift), float("nan"), dtype=t.dtype, device="cuda")
    buf[:, shift:shift + t.shape[1]] = t.cuda()
    return buf[:, shift:shift + t.shape[1]]


def vec(a):
    import torch
    return torch.as_tensor(np.asarray(a), dtype=torch.float32).cuda()


def host(t):
    return t.double().cpu().numpy()


def sums(mag, K):
    return (4 + 2 * np.sqrt(K)) * 2.0 ** -23 * mag + 1e-300


def near(got, want, tol, out="float32"):
    """Within tol before the result's rounding."""
    got = host(got)
    tol = tol + HALF[out] * (np.abs(want) + tol)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4], int(bad.sum()))


def expected(z, mag, K, act="none", m=None, residual=None):
    """y and what it may be off by."""
    tol, y = sums(mag, K), o64.act(z, act)
    if act in ("gelu", "silu"):
        tol = 1.13 * tol + 16 * E * np.abs(z)
    if m is not None:
        y, tol = o64.dropout(y, m), m * tol + 2 * E * m * np.abs(y)
    if residual is not None:
        y = y + residual
        tol = tol + E * np.abs(y)
    return y, tol


SHAPES = [(1, 1, 1), (1, 128, 16), (1, 1000, 333), (3, 200, 17), (5, 4096, 64), (8, 1500, 40), (9, 96, 130), (16, 300, 1000),
          (17, 31, 5), (33, 129, 700), (64, 512, 513), (100, 640, 100), (130, 1100, 260), (300, 256, 1030), (520, 384, 777)]
LARGE = [(2100, 160, 2304), (4000, 96, 4100), (1024, 1024, 1024)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,k,n", SHAPES + LARGE)
def test_linear(ctx, m, k, n, dtype):
    import torch
    from paper_2606_09377_amd import Dropout
    rng = np.random.default_rng(m + 11 * k + 17 * n)
    x, w, b, res = (rng.standard_normal(s) for s in ((m, k), (n, k), (n,), (m, n)))
    w /= np.sqrt(k)
    seed, offset = int(rng.integers(0, 2 ** 63)), int(rng.integers(0, 2 ** 63))
    drop = Dropout(0.3, seed, offset)
    mask = o64.mask(m, n, 0.3, seed, offset)
    tb = vec(b)
    b = host(tb)
    for (pitch, shift), act, d, r, keep_z, other in (((0, 0), "none", False, False, False, None), ((8, 8), "relu", True, True, True, None),
                                                     ((5, 3), "gelu", False, True, False, "bfloat16"), ((16, 8), "silu", True, False, True, "float32")):
        tx, tw, tr = dev(x, dtype, pitch, shift), dev(w, dtype, pitch, shift), dev(res, other or dtype, pitch, shift)
        z, mag = o64.linear(host(tx), host(tw), None if act == "none" else b)
        want, tol = expected(z, mag, k, act, mask if d else None, host(tr) if r else None)
        out = torch.full((m, n + pitch), 7.0, dtype=getattr(torch, other or dtype), device="cuda")
        got = ctx.linear(tx, tw, bias=None if act == "none" else tb, act=act, dropout=drop if d else None, residual=tr if r else None,
                         keep_z=keep_z, out=out[:, :n])
        if keep_z:
            near(got[1], z, sums(mag, k), dtype)
            got = got[0]
        assert got.data_ptr() == out.data_ptr()
        near(got, want, tol, other or dtype)
        assert bool((out[:, n:] == 7.0).all())


def g_of(dy, z, act, m, dtype):
    """g, and what it may be off by."""
    d = dy if m is None else o64.dropout(dy, m)
    if act == "none":
        return d, 2 * E * np.abs(d)
    g, tol = d * o64.slope(z, act), 2 * E * np.abs(d)
    if act != "relu":
        tol = tol + 2.0 ** -20 * np.abs(d)
        if dtype == "bfloat16":
            tol = tol + 2.0 ** -8 * np.abs(g)
    return g, tol


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,k,n", SHAPES + LARGE)
def test_linear_grad(ctx, m, k, n, dtype):
    import torch
    from paper_2606_09377_amd import Dropout
    rng = np.random.default_rng(m + 19 * k + 23 * n)
    x, w, dy, z, add = (rng.standard_normal(s) for s in ((m, k), (n, k), (m, n), (m, n), (m, k)))
    z[0] = 0.0
    seed, offset = int(rng.integers(0, 2 ** 63)), int(rng.integers(0, 2 ** 63))
    mask = o64.mask(m, n, 0.3, seed, offset)
    for (pitch, shift), act, d, a, dw_type in (((0, 0), "none", False, False, None), ((8, 0), "relu", True, True, "float32"),
                                               ((3, 2), "gelu", False, True, None), ((16, 8), "silu", True, False, "bfloat16")):
        tx, tw, tg, tz, ta = (dev(v, dtype, pitch, shift) for v in (x, w, dy, z, add))
        got = ctx.linear_grad(tg, tx, tw, z=None if act == "none" else tz, act=act, dropout=Dropout(0.3, seed, offset) if d else None,
                              add=ta if a else None, dw_dtype=None if dw_type is None else getattr(torch, dw_type))
        g, off = g_of(host(tg), host(tz), act, mask if d else None, dtype)
        want = o64.gradients(g, host(tx), host(tw), host(ta) if a else None)
        more = (off @ np.abs(host(tw)), off.T @ np.abs(host(tx)), off.sum(0))
        for t, (v, mag), e, K, o in zip(got, want, more, (n, m, m), (dtype, dw_type or dtype, "float32")):
            if o == "float32" and t.dim() == 1 and dtype == "bfloat16" and act not in ("none", "relu"):
                e = 2 * E * mag + 2.0 ** -20 * np.abs(o64.dropout(host(tg), mask) if d else host(tg)).sum(0)   # (db's g is not rounded)
            near(t, v, sums(mag, K) + e, o)
    only = ctx.linear_grad(tg, tx, tw, need=(False, False, True))
    assert only[0] is None and only[1] is None
    near(only[2], host(tg).sum(0), sums(np.abs(host(tg)).sum(0), m))


def test_gradients_are_the_differences(ctx):
    """dx, dw, db and the residual's gradient against differences of the loss sum(dy y) in 64 bits."""
    from paper_2606_09377_amd import Dropout
    m, k, n = 6, 70, 9
    for act in o64.ACTS:
        rng = np.random.default_rng(5)
        x, w, dy, r = (rng.standard_normal(s).astype(np.float32) for s in ((m, k), (n, k), (m, n), (m, n)))
        b = rng.standard_normal(n).astype(np.float32)
        drop, mask = Dropout(0.4, 9, 10), o64.mask(m, n, 0.4, 9, 10)

        def loss(x, w, b, r):
            return float((o64.dropout(o64.act(o64.linear(x, w, b)[0], act), mask, r) * dy).sum())
        _, z = ctx.linear(dev(x), dev(w), bias=vec(b), act=act, dropout=drop, residual=dev(r), keep_z=True)
        grads = [host(t) for t in ctx.linear_grad(dev(dy), dev(x), dev(w), z=z, act=act, dropout=drop)] + [dy.astype(np.float64)]
        ins = [v.astype(np.float64) for v in (x, w, b, r)]
        h = 1e-5   # no pre-activation changes its sign: they stay 1e-3 away from 0
        assert np.abs(o64.linear(ins[0], ins[1], ins[2])[0]).min() > 1e-3
        for grad, at in zip(grads, ins):
            for i in rng.integers(0, grad.size, 10):
                e = np.zeros(at.size)
                e[i] = h
                p, q = ([v + s * e.reshape(at.shape) if v is at else v for v in ins] for s in (1, -1))
                d = (loss(*p) - loss(*q)) / (2 * h)
                assert abs(d - grad.flat[i]) <= 2e-6 * max(1.0, np.abs(grad).max()), (act, i, d, grad.flat[i])


def test_relu_takes_its_own_result_for_z(ctx):
    import torch
    from paper_2606_09377_amd import Dropout
    rng = np.random.default_rng(3)
    x, w, dy = dev(rng.standard_normal((70, 90))), dev(rng.standard_normal((50, 90))), dev(rng.standard_normal((70, 50)))
    drop = Dropout(0.25, 4, 1)
    y, z = ctx.linear(x, w, act="relu", dropout=drop, keep_z=True)
    for a, b in zip(ctx.linear_grad(dy, x, w, z=z, act="relu", dropout=drop), ctx.linear_grad(dy, x, w, z=y, act="relu", dropout=drop)):
        assert torch.equal(a, b)


def test_no_rows(ctx):
    import torch
    x, w = torch.empty((0, 40), device="cuda"), torch.ones((30, 40), device="cuda")
    assert ctx.linear(x, w, act="gelu").shape == (0, 30)
    dx, dw, db = ctx.linear_grad(torch.empty((0, 30), device="cuda"), x, w)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()
    db = ctx.linear_grad(torch.empty((0, 30), device="cuda"), x, w, need=(False, False, True))[2]
    assert not db.any()


def test_in_place_and_none_of_the_padding(ctx):
    """y over the residual, dx over add; rows and columns beside them are left as they were."""
    import torch
    rng = np.random.default_rng(8)
    for m, k, n, dtype in ((1, 64, 40, "float32"), (37, 130, 75, "bfloat16"), (300, 512, 333, "float32"), (3, 520, 72, "bfloat16")):
        x, w, dy = dev(rng.standard_normal((m, k)), dtype), dev(rng.standard_normal((n, k)) / np.sqrt(k), dtype), dev(rng.standard_normal((m, n)), dtype)
        for call, cols in ((lambda r, o: ctx.linear(x, w, residual=r, out=o), n), (lambda r, o: None, k)):
            buf = torch.randn(m + 2, cols + 6, device="cuda").to(x.dtype)
            at = buf[1:-1, 3:-3]
            if cols == n:
                want = ctx.linear(x, w, residual=at.clone())
                rest = buf.clone()
                call(at, at)
                assert torch.equal(at, want)
            else:
                from paper_2606_09377_amd.vcrown import _mat
                want = ctx.linear_grad(dy, x, w, add=at.clone(), need=(True, False, False))[0]
                rest = buf.clone()
                ctx._current_stream()
                ctx._check(ctx.lib.vcr_linear_grad(ctx.h, _mat(dy), None, _mat(w), None, _mat(at), _mat(at), None, None))
                assert torch.equal(at, want)
            rest[1:-1, 3:-3] = at
            assert torch.equal(buf, rest)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m", [1, 40, 300])
def test_non_finite_operands(ctx, m, dtype):
    """Infinite and NaN operands reach the results they belong to, and no others; dropped ones reach none."""
    import torch
    from paper_2606_09377_amd import Dropout
    rng = np.random.default_rng(m)
    k, n = 200, 48
    x, w = rng.standard_normal((m, k)), rng.standard_normal((n, k))
    x[0, 3], w[5, 7], w[9, 199] = np.inf, np.nan, -np.inf
    tx, tw = dev(x, dtype), dev(w, dtype)
    want, mag = o64.linear(host(tx), host(tw))
    got = host(ctx.linear(tx, tw))
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(np.isinf(got), np.isinf(want))
    np.testing.assert_array_equal(got[np.isinf(want)], want[np.isinf(want)])
    ok = np.isfinite(want)
    assert (np.abs(got - want)[ok] <= (sums(mag, k) + HALF[dtype] * (np.abs(want) * 2))[ok]).all()
    drop, mask = Dropout(0.5, 1, m), o64.mask(m, n, 0.5, 1, m)
    y = host(ctx.linear(tx, tw, dropout=drop))
    assert not y[mask == 0].any() and np.array_equal(np.isnan(y), np.isnan(want) & (mask > 0))
    # a gradient that is infinite where the mask or the slope leaves nothing
    dy = np.where(mask > 0, rng.standard_normal((m, n)), np.inf)
    z = rng.standard_normal((m, n))
    dy[(z <= 0)] = np.nan
    clean = np.where((mask > 0) & (z > 0), np.nan_to_num(dy, posinf=0.0), 0.0)
    a = ctx.linear_grad(dev(dy, dtype), dev(np.ones((m, k)), dtype), dev(np.ones((n, k)), dtype), z=dev(z, dtype), act="relu", dropout=drop)
    b = ctx.linear_grad(dev(clean, dtype), dev(np.ones((m, k)), dtype), dev(np.ones((n, k)), dtype), z=dev(z, dtype), act="relu", dropout=drop)
    assert all(torch.equal(p, q) and bool(torch.isfinite(p).all()) for p, q in zip(a, b))


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_activations_over_their_range(ctx, act):
    """Values and slopes from -40 to 40, small ones among them: one input, identity weights."""
    import torch
    v = np.concatenate([np.linspace(-40, 40, 3001), np.geomspace(1e-30, 1, 400), -np.geomspace(1e-30, 1, 400)])[:, None]
    one = torch.ones((1, 1), device="cuda")
    t = dev(v)
    y, z = ctx.linear(t, one, act=act, keep_z=True)
    v = host(t)
    np.testing.assert_array_equal(host(z), v)
    want = o64.act(v, act)
    # relative, but for what is below float32's normal range.  (erfc's argument a = -z / sqrt 2 is rounded, and the constant in it: by
    # 2 2^-24 of itself, which changes erfc(a) by a erfc'(a) / erfc(a) times that, at most (2 a^2 + 1) 2^-23 = (z^2 + 1) 2^-23 of itself.)
    rel = 2.0 ** -18 + ((v * v + 1) * 2.0 ** -23 if act == "gelu" else 0.0)
    assert (np.abs(host(y) - want) <= rel * np.abs(want) + 2.0 ** -126).all()
    g = ctx.linear_grad(torch.ones_like(t), t, one, z=z, act=act, need=(True, False, False))[0]
    assert (np.abs(host(g) - o64.slope(v, act)) <= 2.0 ** -20).all()


@pytest.mark.parametrize("m,k,n", [(1, 40000, 40), (5, 33000, 100), (16, 20000, 56), (40, 40000, 33), (7, 104, 70000), (70, 104, 20000)])
def test_long_contractions_and_many_columns(ctx, m, k, n):
    rng = np.random.default_rng(k)
    for dtype in ("float32", "bfloat16"):
        x, w, dy = dev(rng.standard_normal((m, k)), dtype), dev(rng.standard_normal((n, k)), dtype), dev(rng.standard_normal((m, n)), dtype)
        z, mag = o64.linear(host(x), host(w))
        near(ctx.linear(x, w), z, sums(mag, k), dtype)
        for t, (v, g), K, o in zip(ctx.linear_grad(dy, x, w), o64.gradients(host(dy), host(x), host(w)), (n, m, m), (dtype, dtype, "float32")):
            near(t, v, sums(g, K) + 2 * E * g, o)


def test_few_rows_are_rows_of_many(ctx):
    """A row's result does not depend on the other rows, beyond the order of its sum."""
    rng = np.random.default_rng(6)
    k, n = 1032, 264
    for dtype in ("float32", "bfloat16"):
        x, w = dev(rng.standard_normal((70, k)), dtype), dev(rng.standard_normal((n, k)), dtype)
        z, mag = o64.linear(host(x), host(w))
        for m in (1, 2, 4, 5, 8, 9, 15, 16, 17, 32, 33, 48, 63, 64, 65):
            near(ctx.linear(x[:m], w), z[:m], sums(mag[:m], k), dtype)


def test_repeats_bit_for_bit_on_other_streams(ctx):
    import torch
    rng = np.random.default_rng(2)
    x, w, dy = dev(rng.standard_normal((200, 700)), "bfloat16"), dev(rng.standard_normal((300, 700)), "bfloat16"), dev(rng.standard_normal((200, 300)), "bfloat16")
    first = [ctx.linear(x, w), *ctx.linear_grad(dy, x, w)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append([ctx.linear(x, w), *ctx.linear_grad(dy, x, w)])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, first))


def test_offsets_beyond_32_bits(ctx):
    """x of over 2^32 bytes, and results of over 2^32 bytes: the last rows against 64 bits."""
    import torch
    g = torch.Generator("cuda").manual_seed(4)
    m, k, n = 600_000, 4096, 40
    x = torch.empty((m, k), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.randn((n, k), generator=g, device="cuda").bfloat16()
    z, mag = o64.linear(host(x[-50:]), host(w))
    near(ctx.linear(x, w)[-50:], z, sums(mag, k), "bfloat16")
    dx, dw, db = ctx.linear_grad(x[:, :n].contiguous(), x, w)
    want = o64.gradients(host(x[-50:, :n]), host(x[-50:]), host(w))
    near(dx[-50:], want[0][0], sums(want[0][1], n), "bfloat16")
    # one input's column against 64 bits
    col = x[:, -1].double()
    for j in (0, n - 1):
        t = x[:, j].double()
        v, a = float((t * col).sum()), float((t * col).abs().sum())
        assert abs(float(dw[j, -1]) - v) <= sums(a, m) + 2.0 ** -8 * abs(v) * 1.01
    del x, dx
    x = torch.randn((2, 64), generator=g, device="cuda")
    w = torch.randn((1 << 24, 64), generator=g, device="cuda")
    z, mag = o64.linear(host(x), host(w[-60:]))
    near(ctx.linear(x, w)[:, -60:], z, sums(mag, 64))
