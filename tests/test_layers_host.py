"""What the calls on layers' weights refuse, on a validation-only context, and the oracle's own checks."""
import ctypes

import numpy as np
import pytest

from oracle import layers64 as o64


@pytest.fixture(scope="module")
def vc():
    import os
    import paper_2606_09377_amd.vcrown as vc
    if not os.path.exists(vc.LIB_PATH):
        from paper_2606_09377_amd import build
        build.build()
    vc.load_library()
    return vc


def _buf(n=4096):
    raw = np.zeros(n + 64, dtype=np.uint8)
    return raw[-raw.ctypes.data % 64:]


def test_refusals(vc):
    ctx = vc.Ctx(-1)
    lib, h, keep = ctx.lib, ctx.h, _buf()
    p, ref = keep.ctypes.data, ctypes.byref
    ARG, SHAPE, STATE = vc.VCR_ERR_ARG, vc.VCR_ERR_SHAPE, vc.VCR_ERR_STATE

    def mat(rows, cols, kind=0, ld=None, at=p):
        return vc.VcrMat(at, kind, rows, cols, cols if ld is None else ld)

    def mx(rows, cols, at=p, at2=p):
        return vc.VcrMx(at, at2, rows, cols)

    def quant(x, q):
        return lib.vcr_mx_quantize(h, x and ref(x), q and ref(q))
    # valid calls stop before device work
    assert quant(mat(3, 5), mx(3, 5)) == STATE and b"validation-only" in lib.vcr_last_error(h)
    assert lib.vcr_mx_quantize(None, ref(mat(3, 5)), ref(mx(3, 5))) == ARG
    for x, q, want in ((None, mx(3, 5), ARG), (mat(3, 5), None, ARG), (mat(3, 5, kind=2), mx(3, 5), ARG),
                       (mat(3, 5, kind=-1), mx(3, 5), ARG), (mat(3, 5, at=None), mx(3, 5), ARG),
                       (mat(3, 5, at=p + 2), mx(3, 5), ARG), (mat(3, 5, kind=1, at=p + 1), mx(3, 5), ARG),
                       (mat(3, 5, kind=1, at=p + 2), mx(3, 5), STATE), (mat(3, 5, ld=4), mx(3, 5), SHAPE),
                       (mat(3, 5, ld=1 << 40), mx(3, 5), SHAPE), (mat(-1, 5), mx(3, 5), SHAPE),
                       (mat(3, 0), mx(3, 5), SHAPE), (mat(1 << 31, 5), mx(3, 5), SHAPE), (mat(3, 6), mx(3, 5), SHAPE),
                       (mat(4, 5), mx(3, 5), SHAPE), (mat(3, 5), mx(3, 5, at=None), ARG),
                       (mat(3, 5), mx(3, 5, at2=p + 8), ARG), (mat(3, 5), mx(3, -1), SHAPE),
                       (mat(0, 5, at=None), mx(0, 5, None, None), STATE)):
        assert quant(x, q) == want, lib.vcr_last_error(h)
        y = lib.vcr_mx_dequantize(h, q and ref(q), x and ref(x))
        assert y == want
    n64 = ctypes.c_uint64
    a, b = n64(), n64()
    assert lib.vcr_mx_bytes(17, 129, ref(a), ref(b)) == 0 and (a.value, b.value) == (2 * 2 * 1024, 2 * 256)
    assert lib.vcr_mx_bytes(-1, 4, ref(a), ref(b)) == ARG and lib.vcr_mx_bytes(4, 4, None, ref(b)) == ARG

    def product(x, w, y, bias=None, relu=0):
        return lib.vcr_mx_product(h, ref(x), ref(w), bias, relu, ref(y))

    def linear(x, w, y, bias=None, relu=0):
        return lib.vcr_mx_linear(h, ref(x), ref(w), bias, relu, ref(y))
    for call, x in ((product, mx), (linear, mat)):
        assert call(x(3, 40), mx(7, 40), mat(3, 7), p, 1) == STATE
        assert call(x(0, 40), mx(7, 40), mat(0, 7)) == STATE
        assert call(x(3, 41), mx(7, 40), mat(3, 7)) == SHAPE
        assert call(x(3, 40), mx(7, 40), mat(3, 8)) == SHAPE
        assert call(x(3, 40), mx(7, 40), mat(4, 7)) == SHAPE
        assert call(x(3, 40), mx(0, 40), mat(3, 7)) == SHAPE
        assert call(x(3, 40), mx(7, 40), mat(3, 7), p + 2) == ARG

        far = vc.VCR_ERR_UNSUPPORTED   # longer contractions than the kernels address
        assert call(x(3, 1 << 21), mx(7, 1 << 21), mat(3, 7)) == STATE
        assert call(x(3, (1 << 21) + 1), mx(7, (1 << 21) + 1), mat(3, 7)) == far

    def grad(dy, y, x, w, dx, dw, db=p):
        r = lambda v: None if v is None else ref(v)  # noqa: E731
        return lib.vcr_mx_linear_grad(h, r(dy), r(y), r(x), r(w), r(dx), r(dw), db)
    ok = (mat(3, 7), mat(3, 7), mat(3, 40), mx(7, 40), mat(3, 40), mat(7, 40))
    assert grad(*ok) == STATE and grad(*ok, None) == STATE
    assert grad(ok[0], None, None, None, None, None) == STATE
    for i, bad, want in ((0, None, ARG), (1, mat(3, 8), SHAPE), (1, mat(3, 7, kind=1), ARG), (2, None, ARG), (3, None, ARG),
                         (2, mat(4, 40), SHAPE), (2, mat(3, 40, kind=1), ARG), (3, mx(8, 40), SHAPE),
                         (4, mat(3, 41), SHAPE), (5, mat(7, 41), SHAPE), (5, mat(8, 40), SHAPE)):
        assert grad(*ok[:i], bad, *ok[i + 1:]) == want, (i, lib.vcr_last_error(h))

    n = (1 << 21) + 1
    assert grad(mat(3, n), None, None, mx(n, 40), mat(3, 40), None) == far
    assert grad(mat(n, 3), None, mat(n, 40), None, None, mat(3, 40)) == far
    assert grad(mat(n, 3), None, None, None, None, None) == STATE

    def orth(g, o, base=None, out=None, count=1, gs=0, bs=0, os_=0):
        r = lambda v: None if v is None else ref(v)  # noqa: E731
        return lib.vcr_orthogonalize(h, r(g), count, gs, r(o), r(base), bs, r(out or mat(5, 6)), os_)

    def opts(steps=5, a=3.4, b=-4.7, c=2.0, eps=1e-7, gain=1.0, keep=1.0):
        return vc.VcrNsOpts(steps, a, b, c, eps, gain, keep)
    assert orth(mat(5, 6), opts()) == STATE and orth(mat(5, 6), opts(), mat(5, 6, kind=1)) == STATE
    assert orth(mat(5, 6), opts(), count=2, gs=30, os_=30) == STATE
    assert orth(mat(5, 6), opts(), count=2, gs=29, os_=30) == SHAPE
    assert orth(mat(5, 6), opts(), mat(5, 6), count=2, gs=30, os_=30, bs=10) == SHAPE
    assert orth(mat(5, 6), None) == ARG and orth(None, opts()) == ARG
    for o in (opts(0), opts(101), opts(a=float("nan")), opts(eps=-1.0), opts(eps=float("inf")), opts(gain=float("nan"))):
        assert orth(mat(5, 6), o) == ARG
    assert orth(mat(5, 7), opts()) == SHAPE and orth(mat(5, 6), opts(), mat(6, 6)) == SHAPE
    assert orth(mat(5, 6), opts(), count=-1) == ARG and orth(mat(5, 6), opts(), count=70000) == ARG
    assert orth(mat(1 << 20, 1 << 20), opts(), out=mat(1 << 20, 1 << 20)) == SHAPE
    assert orth(mat(4, n), opts(), out=mat(4, n)) == far


def test_oracle_grid():
    """The oracle's own rounding: every value of the grid is its own, midpoints go to even codes."""
    x = np.concatenate([o64.GRID, -o64.GRID, np.full(16, 4.0)])[None]
    codes, scales = o64.quantize(x)
    assert scales[0, 0] == 127
    np.testing.assert_array_equal(o64.values(codes, scales), x)
    mid = np.concatenate([(o64.GRID[1:] + o64.GRID[:-1]) / 2, np.full(25, 4.0)])[None]
    codes, _ = o64.quantize(mid)
    assert (codes % 2 == 0).all()


def test_oracle_orthogonalize():
    g = np.random.default_rng(0).standard_normal((20, 30))
    s = np.linalg.svd(o64.orthogonalize(g), compute_uv=False)
    assert 0.6 < s.min() and s.max() < 1.3
    np.testing.assert_allclose(o64.orthogonalize(g.T), o64.orthogonalize(g).T, atol=1e-12)


def test_gradients_of_one_layer(vc):
    """x and w of different widths are not one layer's."""
    ctx = vc.Ctx(-1)
    keep = _buf()
    p, ref = keep.ctypes.data, ctypes.byref

    def mat(rows, cols):
        return vc.VcrMat(p, 0, rows, cols, cols)

    def grad(x, w):
        return ctx.lib.vcr_mx_linear_grad(ctx.h, ref(mat(3, 7)), None, ref(mat(3, x)), ref(vc.VcrMx(p, p, 7, w)), ref(mat(3, w)),
                                          ref(mat(7, x)), p)
    assert grad(40, 40) == vc.VCR_ERR_STATE
    assert grad(41, 40) == vc.VCR_ERR_SHAPE and b"w" in ctx.lib.vcr_last_error(ctx.h)


def test_calls_follow_the_stream_of_their_own_device(vc, monkeypatch):
    """Where torch's current device is another one than the context's, the context's device's current stream is taken."""
    import types
    import torch
    current = {0: 0x1000, 1: 0x2000}   # device: handle of its current stream
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: current[d], raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: types.SimpleNamespace(cuda_stream=current[1 if d is None else d]))
    given = []
    ctx = vc.Ctx.__new__(vc.Ctx)
    ctx.h, ctx.device, ctx._raw_stream = None, 0, 0   # (no library handle: nothing to destroy)
    ctx.lib = types.SimpleNamespace(vcr_set_stream=lambda h, s: given.append(s.value) or 0)
    ctx._current_stream()
    ctx._current_stream()
    ctx._stream_sync()
    current[0] = 0x3000
    ctx._current_stream()
    assert given == [0x1000, 0x1000, 0x3000]
