"""Layers in 4 bits on the GPU (vcr_mx_*) against 64 bits.

Tolerances.  Quantisation is exact: equal codes and scales.  A product of 4-bit values, or of a 4-bit value and
one of three bf16 parts, is exact in float32; of two float32 values as three parts each it is off by at
most 1.65 2^-24 of itself.  A float32 sum of K terms, in any order, with each addition rounded or cut to
24 bits (2^-23), is off by about sqrt(K) 2^-23 of the sum of magnitudes at random and K 2^-23 at worst;
(4 + 2 sqrt(K)) 2^-23 of it is allowed.  bf16 results (8 significant bits) round by
2^-8 of themselves."""
import ctypes

import numpy as np
import pytest

from oracle import layers64 as o64

pytestmark = pytest.mark.gpu


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


def host(t):
    return t.double().cpu().numpy()


def near(got, want, mag, K, out="float32"):
    got = host(got)
    tol = (4 + 2 * np.sqrt(K)) * 2.0 ** -23 * mag + 1e-300
    if out == "bfloat16":
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (got[bad][:4], want[bad][:4], tol[bad][:4], int(bad.sum()))


def weights(rng, n, k, spread=3):
    """Random codes and scales in row order, their MX and values."""
    import torch
    from paper_2606_09377_amd import MX
    codes = rng.integers(0, 16, (n, k)).astype(np.uint8)
    scales = rng.integers(124 - spread, 124 + spread + 1, (n, -(-k // 32))).astype(np.uint8)
    even = np.zeros((n, -(-k // 2) * 2), dtype=np.uint8)
    even[:, :k] = codes
    packed = torch.as_tensor(even[:, ::2] | even[:, 1::2] << 4).cuda()
    return MX.pack(packed, torch.as_tensor(scales).cuda(), k), o64.values(codes, scales)


def unpacked(q):
    c, s = q.unpack()
    c = c.cpu().numpy()
    codes = np.stack((c & 15, c >> 4), -1).reshape(c.shape[0], -1)[:, :q.cols]
    return codes, s.cpu().numpy()


SHAPES = [(1, 1), (1, 33), (16, 128), (17, 129), (5, 31), (33, 1000), (100, 513), (64, 2048)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_is_exact(ctx, rows, cols, dtype):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (rows, cols)))
    for pitch, shift in ((0, 0), (8, 8), (3, 1)):
        t = dev(x, dtype, pitch, shift)
        q = ctx.mx_quantize(t)
        codes, scales = o64.quantize(host(t))
        gc, gs = unpacked(q)
        np.testing.assert_array_equal(gs, scales)
        np.testing.assert_array_equal(gc, codes)
        for out in ("float32", "bfloat16"):
            import torch
            y = ctx.mx_dequantize(q, dtype=getattr(torch, out))
            np.testing.assert_array_equal(host(y), o64.values(codes, scales))
        # padding rows and columns hold zero codes
        full = q.codes.view(-1, q.codes.shape[1], 4, 16, 16).permute(0, 3, 1, 2, 4).reshape(-1, q.codes.shape[1] * 64)
        assert not full[rows:].any() and not full[:, -(-cols // 2):].any()


def test_quantize_ties_ranges_and_non_finite(ctx):
    ties = np.array([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 6.5, 7.9375] + [4.0] * 21)
    rows = [ties, -ties, np.nextafter(ties.astype(np.float32), np.float32(9)), np.nextafter(ties.astype(np.float32), np.float32(-9))]
    x = np.stack(rows).astype(np.float32)
    # every magnitude of float32, subnormal ones, blocks of zeros
    x = np.concatenate([x] + [x * np.float32(2.0 ** e) for e in (-140, -127, -126, -124, -100, 60, 124)] + [np.zeros((1, 32), np.float32)])
    x[-2, 5] = np.inf
    x[-3, 7] = np.nan
    x[-4, 31] = -np.inf
    t = dev(x)
    q = ctx.mx_quantize(t)
    codes, scales = o64.quantize(host(t))
    gc, gs = unpacked(q)
    np.testing.assert_array_equal(gs, scales)
    ok = np.repeat(scales != 255, 32, axis=1)
    np.testing.assert_array_equal(gc[ok], codes[ok])
    y = host(ctx.mx_dequantize(q))
    assert np.isnan(y[-2]).all() and np.isnan(y[-3]).all() and np.isnan(y[-4]).all()
    np.testing.assert_array_equal(y[ok], o64.values(codes, scales)[ok])


def test_dequantize_every_code_and_scale(ctx):
    import torch
    from paper_2606_09377_amd import MX
    codes = np.tile(np.arange(16, dtype=np.uint8), (256, 2))
    scales = np.arange(256, dtype=np.uint8)[:, None]
    packed = torch.as_tensor(codes[:, ::2] | codes[:, 1::2] << 4).cuda()
    y = host(ctx.mx_dequantize(MX.pack(packed, torch.as_tensor(scales).cuda(), 32)))
    want = o64.values(codes, scales)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    np.testing.assert_array_equal(y, want)


PRODUCTS = [(1, 1, 1), (1, 128, 16), (1, 1000, 333), (3, 200, 17), (15, 4096, 64), (16, 300, 1000), (17, 31, 5),
            (33, 129, 700), (64, 512, 513), (100, 640, 100), (130, 1100, 260), (300, 256, 1030), (520, 384, 777)]
LARGE = [(2100, 160, 2300), (4000, 96, 4100)]   # enough tiles of every shape


@pytest.mark.parametrize("out", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,k,n", PRODUCTS + LARGE)
def test_product(ctx, m, k, n, out):
    import torch
    rng = np.random.default_rng(m + 7 * k + 13 * n)
    a, av = weights(rng, m, k)
    w, wv = weights(rng, n, k)
    b = rng.standard_normal(n).astype(np.float32)
    for bias, relu in ((None, False), (b, True)):
        want, mag = o64.linear(av, wv, bias, relu)
        y = ctx.mx_product(a, w, None if bias is None else torch.as_tensor(bias).cuda(), relu, dtype=getattr(torch, out))
        near(y, want, mag, k, out)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,k,n", PRODUCTS + LARGE)
def test_linear(ctx, m, k, n, dtype):
    import torch
    rng = np.random.default_rng(m + 11 * k + 17 * n)
    w, wv = weights(rng, n, k)
    b = rng.standard_normal(n).astype(np.float32)
    x = rng.standard_normal((m, k))
    for (pitch, shift), bias, relu in (((0, 0), None, False), ((5, 3), b, True), ((16, 8), b, False)):
        t = dev(x, dtype, pitch, shift)
        want, mag = o64.linear(host(t), wv, bias, relu)
        out = torch.full((m, n + pitch), 7.0, dtype=t.dtype, device="cuda")
        y = ctx.mx_linear(t, w, None if bias is None else torch.as_tensor(bias).cuda(), relu, out=out[:, :n])
        near(y, want, mag, k, dtype)
        assert bool((out[:, n:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,k,n", PRODUCTS + LARGE)
def test_linear_grad(ctx, m, k, n, dtype):
    import torch
    rng = np.random.default_rng(m + 19 * k + 23 * n)
    w, wv = weights(rng, n, k)
    x, dy, y = (rng.standard_normal(s) for s in ((m, k), (m, n), (m, n)))
    y[0] = 0.0
    for masked, (pitch, shift) in ((False, (0, 0)), (True, (3, 2)), (True, (8, 0))):
        tx, tg, ty = dev(x, dtype, pitch, shift), dev(dy, dtype, pitch, shift), dev(y, dtype, pitch, shift)
        got = ctx.mx_linear_grad(tg, tx, w, y=ty if masked else None)
        want = o64.linear_grad(host(tg), host(tx), wv, host(ty) if masked else None)
        for g, (v, mag), K, o in zip(got, want, (n, m, m), (dtype, "float32", "float32")):
            near(g, v, mag, K, o)
    only = ctx.mx_linear_grad(tg, tx, w, need=(False, False, True))
    assert only[0] is None and only[1] is None
    near(only[2], *o64.linear_grad(host(tg), host(tx), wv)[2], m)


def test_gradients_are_the_differences(ctx):
    """dx, dw and db against differences of the loss sum(dy * relu(x w^T + b)) in 64 bits."""
    import torch
    rng = np.random.default_rng(5)
    m, k, n = 6, 70, 9
    w, wv = weights(rng, n, k)
    x, dy, b = rng.standard_normal((m, k)).astype(np.float32), rng.standard_normal((m, n)).astype(np.float32), rng.standard_normal(n).astype(np.float32)

    def loss(x, w, b):
        return float((o64.linear(x, w, b, True)[0] * dy).sum())
    y = ctx.mx_linear(dev(x), w, torch.as_tensor(b).cuda(), relu=True)
    dx, dw, db = (host(t) for t in ctx.mx_linear_grad(dev(dy), dev(x), w, y=y))
    x, b = x.astype(np.float64), b.astype(np.float64)
    h = 1e-5   # no pre-activation changes its sign: they stay 1e-3 away from 0
    assert np.abs(o64.linear(x, wv, b)[0]).min() > 1e-3
    for grad, at in ((dx, x), (dw, wv), (db, b)):
        for i in rng.integers(0, grad.size, 12):
            e = np.zeros(at.size)
            e[i] = h
            p, q = ([v + s * e.reshape(at.shape) if v is at else v for v in (x, wv, b)] for s in (1, -1))
            d = (loss(*p) - loss(*q)) / (2 * h)
            assert abs(d - grad.flat[i]) <= 1e-6 * max(1.0, np.abs(grad).max()), (i, d, grad.flat[i])


@pytest.mark.parametrize("m,k,n", [(1, 40000, 40), (5, 33000, 100), (8, 20000, 50), (40, 40000, 33), (7, 100, 70000)])
def test_long_contractions_and_many_columns(ctx, m, k, n):
    """Contractions that do not fit LDS together, or are divided among workgroups; columns in many rounds."""
    rng = np.random.default_rng(k)
    w, wv = weights(rng, n, k)
    for dtype in ("float32", "bfloat16"):
        x = dev(rng.standard_normal((m, k)), dtype)
        near(ctx.mx_linear(x, w), *o64.linear(host(x), wv), k, dtype)
    q = ctx.mx_quantize(x)
    near(ctx.mx_product(q, w), *o64.linear(host(ctx.mx_dequantize(q)), wv), k)
    dy = dev(rng.standard_normal((m, n)))
    near(ctx.mx_linear_grad(dy, None, w, need=(True, False, False))[0], host(dy) @ wv, np.abs(host(dy)) @ np.abs(wv), n)


def test_large_gradients(ctx):
    rng = np.random.default_rng(77)
    m, k, n = 130, 2200, 2300
    w, wv = weights(rng, n, k)
    x, dy = dev(rng.standard_normal((m, k))), dev(rng.standard_normal((m, n)))
    for got, (want, mag), K in zip(ctx.mx_linear_grad(dy, x, w), o64.linear_grad(host(dy), host(x), wv), (n, m, m)):
        near(got, want, mag, K)


@pytest.mark.parametrize("m", [1, 40, 300])
def test_non_finite_and_extreme_operands(ctx, m):
    """Infinite, NaN, huge and tiny float32 rows give what float32 products give."""
    rng = np.random.default_rng(m)
    k, n = 200, 50
    w, wv = weights(rng, n, k)
    x = rng.standard_normal((m, k)).astype(np.float32)
    x[0, 3], x[0, 100] = np.inf, 1.0
    t = dev(x)
    got = host(ctx.mx_linear(t, w))
    with np.errstate(invalid="ignore"):
        want = np.where(wv[:, 3] == 0, np.nan, np.sign(wv[:, 3]) * np.inf)
    np.testing.assert_array_equal(got[0], want)
    if m > 1:
        near(ctx.mx_linear(t, w)[1:], *o64.linear(x[1:], wv), k)
    x[0, 3] = np.nan
    assert np.isnan(host(ctx.mx_linear(dev(x), w))[0]).all()
    for f in (np.float32(3.4e38), np.float32(2.0 ** -120)):   # the largest part alone rounds to infinity
        y = np.zeros((m, k), np.float32)
        y[:, 5], y[:, 6] = f, -f
        want, mag = o64.linear(y, wv)
        # a product beyond float32 makes a float32 sum infinite or NaN, whatever the other one takes away
        over = np.maximum(np.abs(y[:, 5:6] * wv[:, 5].astype(np.float64)), np.abs(y[:, 6:7] * wv[:, 6].astype(np.float64))) >= 2.0 ** 128
        got = host(ctx.mx_linear(dev(y), w))
        assert not np.isfinite(got[over]).any()
        tol = 32 * 2.0 ** -23 * mag + 2.0 ** -133
        sure = mag < 2.0 ** 127   # (between, the order of the sum decides)
        assert (np.abs(got - want) <= tol)[sure].all() and sure.any()
    # a NaN block of weights reaches its row of results only
    c, s = w.unpack()
    s[7, 2] = 255
    from paper_2606_09377_amd import MX
    wn = MX.pack(c, s, k)
    z = dev(rng.standard_normal((m, k)))
    for got in (ctx.mx_linear(z, wn), ctx.mx_product(ctx.mx_quantize(z), wn)):
        assert np.isnan(host(got)[:, 7]).all() and np.isfinite(np.delete(host(got), 7, 1)).all()


def test_no_rows(ctx):
    import torch
    rng = np.random.default_rng(3)
    w, _ = weights(rng, 20, 40)
    x = torch.empty((0, 40), device="cuda")
    assert ctx.mx_linear(x, w).shape == (0, 20)
    q = ctx.mx_quantize(x)
    assert ctx.mx_product(q, w).shape == (0, 20) and ctx.mx_dequantize(q).shape == (0, 40)
    dx, dw, db = ctx.mx_linear_grad(torch.empty((0, 20), device="cuda"), x, w)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()


def test_rows_do_not_mix_and_calls_repeat(ctx):
    """The same call gives the same bits, on another stream too, with larger calls in between."""
    import torch
    rng = np.random.default_rng(9)
    w, wv = weights(rng, 300, 700)
    w2, _ = weights(rng, 1500, 900)
    x = dev(rng.standard_normal((21, 700)))
    a = ctx.mx_linear(x, w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        b = ctx.mx_linear(x, w)
        big = ctx.mx_linear(dev(rng.standard_normal((500, 900))), w2)
    c = ctx.mx_linear(x, w)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c) and torch.isfinite(big).all()
    near(a, *o64.linear(host(x), wv), 700)


def test_calls_are_recorded_into_a_graph(ctx):
    import torch
    from paper_2606_09377_amd import VcrError
    rng = np.random.default_rng(12)
    m, k, n = 24, 1000, 500
    w, wv = weights(rng, n, k)
    x, dy = dev(rng.standard_normal((m, k))), dev(rng.standard_normal((m, n)))
    y, q = torch.empty((m, n), device="cuda"), ctx.mx_quantize(x)

    def calls():
        ctx.mx_quantize(x, out=q)
        ctx.mx_linear(x, w, relu=True, out=y)
        return (ctx.mx_product(q, w), *ctx.mx_linear_grad(dy, x, w, y=y), ctx.orthogonalize(x))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        outs = calls()
    for seed in range(3):
        x.copy_(dev(np.random.default_rng(seed).standard_normal((m, k))))
        want = [t.clone() for t in calls()] + [y.clone()]
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        ctx.mx_linear(dev(rng.standard_normal((200, k))), w)   # the program's own work in between
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(list(outs) + [y], want))
    # without a call before there is no workspace to record
    fresh = torch.cuda.Stream()
    g2 = torch.cuda.CUDAGraph()
    with pytest.raises(VcrError):
        with torch.cuda.graph(g2, stream=fresh):
            ctx.mx_linear(x, w)
    torch.cuda.synchronize()
    near(ctx.mx_linear(x, w), *o64.linear(host(x), wv), k)


def test_workspace_cap_and_statistics():
    import torch
    from paper_2606_09377_amd import Ctx, VcrError
    from paper_2606_09377_amd.vcrown import OPT_WORKSPACE_CAP_BYTES, VCR_ERR_OOM
    ctx = Ctx(0)
    rng = np.random.default_rng(1)
    w, wv = weights(rng, 640, 640)
    x = dev(rng.standard_normal((600, 640)))
    ctx.set_option(OPT_WORKSPACE_CAP_BYTES, 1 << 16)
    with pytest.raises(VcrError) as e:
        ctx.mx_linear(x, w)
    assert e.value.status == VCR_ERR_OOM
    ctx.set_option(OPT_WORKSPACE_CAP_BYTES, 0)
    near(ctx.mx_linear(x, w), *o64.linear(host(x), wv), 640)
    torch.cuda.synchronize()
    s = ctx.stats()
    assert s["workspace_bytes"] > 0 and s["peak_workspace_bytes"] >= s["workspace_bytes"]


def test_bounds_are_left_alone(ctx):
    """Calls on layers between bounds calls do not change the bounds or the layer bounds kept."""
    import torch
    from paper_2606_09377_amd import Ctx
    from workloads import random_mlp
    wl = random_mlp(7, [40, 150, 130, 10], 3, 0.05)
    c = Ctx(0)
    c.load_net(wl.net)
    x0, C = torch.from_numpy(wl.x0).cuda(), torch.from_numpy(wl.C).cuda()
    lb, ub = c.crown_bounds(x0, wl.eps, C)
    l, u = c.layer_bounds(1, 3)
    rng = np.random.default_rng(2)
    w, _ = weights(rng, 640, 640)
    c.mx_linear(torch.full((600, 640), float("nan"), device="cuda"), w)
    c.orthogonalize(torch.full((300, 640), float("nan"), device="cuda"))
    l2, u2 = c.layer_bounds(1, 3)
    lb2, ub2 = c.crown_bounds(x0, wl.eps, C)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in ((l, l2), (u, u2), (lb, lb2), (ub, ub2)))


def test_offsets_beyond_32_bits(ctx):
    """Weights of over 2^32 values' bytes in float32: the last rows against 64 bits."""
    import torch
    from paper_2606_09377_amd import MX
    n, k = 270336, 4096
    g = torch.Generator("cuda").manual_seed(4)
    q = MX.empty(n, k)
    q.codes.random_(0, 256, generator=g)
    q.scales.fill_(120)
    x = dev(np.random.default_rng(1).standard_normal((2, k)))
    y = host(ctx.mx_linear(x, q)[:, -100:])
    tail = MX(q.codes[-7:].contiguous(), q.scales[-7:].contiguous(), 112, k)
    codes, scales = unpacked(tail)
    want, mag = o64.linear(host(x), o64.values(codes, scales)[-100:])
    assert (np.abs(y - want) <= (4 + 2 * np.sqrt(k)) * 2.0 ** -23 * mag).all()
    v = ctx.mx_dequantize(q)
    assert n * k * 4 > 2 ** 32
    np.testing.assert_array_equal(host(v[-112:]), o64.values(codes, scales))
    v2 = ctx.mx_quantize(v)
    assert torch.equal(ctx.mx_dequantize(v2), v)
