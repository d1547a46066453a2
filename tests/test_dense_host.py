"""What the calls on float layers, dropout and the loss refuse, on a validation-only context, and the oracle's own checks."""
import ctypes

import numpy as np
import pytest

from oracle import dense64 as o64


@pytest.fixture(scope="module")
def vc():
    import os
    import paper_2606_09377_amd.vcrown as vc
    if not os.path.exists(vc.LIB_PATH):
        from paper_2606_09377_amd import build
        build.build()
    vc.load_library()
    return vc


@pytest.fixture(scope="module")
def at():
    raw = np.zeros(4096 + 64, dtype=np.uint8)
    buf = raw[-raw.ctypes.data % 64:]
    yield buf.ctypes.data
    assert not buf.any()


def ref(v):
    return None if v is None else ctypes.byref(v)


def make_mat(vc, at):
    def mat(rows, cols, kind=0, ld=None, p=at):
        return vc.VcrMat(p, kind, rows, cols, cols if ld is None else ld)
    return mat


def test_packed_structures(vc):
    d = vc.Dropout(0.25, 2 ** 64 - 3, -1)
    s = vc.VcrDrop.from_buffer_copy(d._c)
    assert (s.p, s.seed, s.offset, s.step) == (0.25, 2 ** 64 - 3, 2 ** 64 - 1, None)
    o = vc.VcrLinearOpts.from_buffer_copy(vc._LINEAR.pack(16, 2, 32, 48, 64))
    assert (o.bias, o.act, o.drop, o.residual, o.z) == (16, 2, 32, 48, 64)
    o = vc.VcrLossOpts.from_buffer_copy(vc._LOSS.pack(0.5, 0.25, 1, -2.0))
    assert (o.smoothing, o.lse2, o.mean, o.scale) == (0.5, 0.25, 1, -2.0)
    with pytest.raises(ValueError):
        vc._linear_opts(None, "tanh", None, None, None)
    with pytest.raises(ValueError):
        vc.Dropout(0.1, step=np.zeros(1))


def test_dropout_refusals(vc, at):
    ctx, mat = vc.Ctx(-1), make_mat(vc, at)
    ARG, SHAPE, STATE = vc.VCR_ERR_ARG, vc.VCR_ERR_SHAPE, vc.VCR_ERR_STATE

    def drop(x, d, res, y):
        return ctx.lib.vcr_dropout(ctx.h, ref(x), ref(d), ref(res), ref(y))
    D = vc.VcrDrop
    ok = D(0.5, 1, 2, None)
    assert drop(mat(3, 5), ok, None, mat(3, 5, 1)) == STATE
    assert drop(mat(0, 5, p=None), ok, None, mat(0, 5, p=None)) == STATE
    assert drop(mat(3, 5), ok, mat(3, 5, 1, 8), mat(3, 5)) == STATE
    assert ctx.lib.vcr_dropout(None, ref(mat(3, 5)), ref(ok), None, ref(mat(3, 5))) == ARG
    for p, want in ((0.0, STATE), (65535 / 65536, STATE), (1 - 2 ** -17, ARG), (1.0, ARG), (-0.1, ARG), (float("nan"), ARG),
                    (float("inf"), ARG)):
        assert drop(mat(3, 5), D(p, 0, 0, None), None, mat(3, 5)) == want
    assert drop(mat(3, 5), D(0.5, 0, 0, at + 4), None, mat(3, 5)) == ARG
    assert drop(mat(3, 5), D(0.5, 0, 0, at + 8), None, mat(3, 5)) == STATE
    for x, res, y, want in ((None, None, mat(3, 5), ARG), (mat(3, 5), None, None, ARG), (mat(3, 5), None, mat(3, 6), SHAPE),
                            (mat(3, 5), mat(4, 5), mat(3, 5), SHAPE), (mat(3, 5, 2), None, mat(3, 5), ARG),
                            (mat(3, 5, p=None), None, mat(3, 5), ARG), (mat(3, 5, p=at + 2), None, mat(3, 5), ARG),
                            (mat(3, 5, ld=4), None, mat(3, 5), SHAPE)):
        assert drop(x, ok, res, y) == want
    assert drop(mat(3, 5), None, None, mat(3, 5)) == ARG


def test_linear_refusals(vc, at):
    ctx, mat = vc.Ctx(-1), make_mat(vc, at)
    ARG, SHAPE, STATE, FAR = vc.VCR_ERR_ARG, vc.VCR_ERR_SHAPE, vc.VCR_ERR_STATE, vc.VCR_ERR_UNSUPPORTED

    def linear(x, w, y, bias=None, act=0, drop=None, res=None, z=None):
        adr = [None if v is None else ctypes.addressof(v) for v in (drop, res, z)]
        o = vc.VcrLinearOpts(bias, act, *adr)
        return ctx.lib.vcr_linear(ctx.h, ref(x), ref(w), ref(o), ref(y))
    good = (mat(3, 40), mat(7, 40), mat(3, 7))
    assert linear(*good) == STATE and b"validation-only" in ctx.lib.vcr_last_error(ctx.h)
    assert ctx.lib.vcr_linear(ctx.h, ref(good[0]), ref(good[1]), None, ref(good[2])) == STATE
    assert ctx.lib.vcr_linear(None, ref(good[0]), ref(good[1]), None, ref(good[2])) == ARG
    assert linear(mat(3, 40, 1), mat(7, 40, 1), mat(3, 7), at, 3, vc.VcrDrop(0.1, 1, 1, None), mat(3, 7, 1), mat(3, 7, 1)) == STATE
    assert linear(mat(0, 40, p=None), mat(7, 40), mat(0, 7, p=None)) == STATE
    for x, w, y, want in ((None, good[1], good[2], ARG), (good[0], None, good[2], ARG), (good[0], good[1], None, ARG),
                          (mat(3, 40, 1), good[1], good[2], ARG), (mat(3, 41), good[1], good[2], SHAPE),
                          (good[0], good[1], mat(3, 8), SHAPE), (good[0], good[1], mat(4, 7), SHAPE),
                          (good[0], mat(0, 40), mat(3, 7), SHAPE), (mat(3, 1 << 21), mat(7, 1 << 21), good[2], STATE),
                          (mat(3, (1 << 21) + 1), mat(7, (1 << 21) + 1), good[2], FAR),
                          (mat((1 << 24) + 1, 40), good[1], mat((1 << 24) + 1, 7), FAR),
                          (good[0], mat((1 << 24) + 1, 40), mat(3, (1 << 24) + 1), FAR)):
        assert linear(x, w, y) == want, ctx.lib.vcr_last_error(ctx.h)
    assert linear(*good, bias=at + 2) == ARG
    assert linear(*good, act=4) == ARG and linear(*good, act=-1) == ARG
    assert linear(*good, drop=vc.VcrDrop(1.5, 0, 0, None)) == ARG
    assert linear(*good, res=mat(3, 8)) == SHAPE and linear(*good, z=mat(2, 7)) == SHAPE
    assert linear(*good, res=mat(3, 7, 5)) == ARG and linear(*good, z=mat(3, 7, p=None)) == ARG


def test_linear_grad_refusals(vc, at):
    ctx, mat = vc.Ctx(-1), make_mat(vc, at)
    ARG, SHAPE, STATE, FAR = vc.VCR_ERR_ARG, vc.VCR_ERR_SHAPE, vc.VCR_ERR_STATE, vc.VCR_ERR_UNSUPPORTED

    def grad(dy=mat(3, 7), x=mat(3, 40), w=mat(7, 40), add=None, dx=mat(3, 40), dw=mat(7, 40), db=at, act=0, z=None, drop=None):
        o = vc.VcrLinearOpts(None, act, drop and ctypes.addressof(drop), None, z and ctypes.addressof(z))
        return ctx.lib.vcr_linear_grad(ctx.h, ref(dy), ref(x), ref(w), ref(o), ref(add), ref(dx), ref(dw), db)
    assert grad() == STATE and grad(act=2, z=mat(3, 7, 1), drop=vc.VcrDrop(0.5, 0, 0, None), add=mat(3, 40, 1)) == STATE
    assert grad(x=None, dw=None) == STATE and grad(w=None, dx=None) == STATE and grad(None) == ARG
    assert grad(dx=None, dw=None, db=None) == STATE
    assert ctx.lib.vcr_linear_grad(ctx.h, ref(mat(3, 7)), None, None, None, None, None, None, at) == STATE
    assert ctx.lib.vcr_linear_grad(None, ref(mat(3, 7)), None, None, None, None, None, None, at) == ARG
    assert grad(x=None) == ARG and grad(w=None) == ARG
    assert grad(act=1) == ARG and grad(act=1, z=mat(3, 8)) == SHAPE and grad(act=9, z=mat(3, 7)) == ARG
    assert grad(x=mat(3, 40, 1)) == ARG and grad(w=mat(7, 40, 1)) == ARG
    assert grad(x=mat(4, 40)) == SHAPE and grad(w=mat(8, 40)) == SHAPE and grad(x=mat(3, 41), dw=mat(7, 41)) == SHAPE
    assert grad(dx=mat(3, 41)) == SHAPE and grad(dw=mat(7, 41)) == SHAPE and grad(add=mat(3, 39)) == SHAPE
    assert grad(db=at + 1) == ARG and grad(drop=vc.VcrDrop(-1.0, 0, 0, None)) == ARG
    n = (1 << 21) + 1
    assert grad(dy=mat(3, n), w=mat(n, 40), dw=mat(n, 40)) == FAR
    assert grad(dy=mat(n, 7), x=mat(n, 40), dx=mat(n, 40)) == FAR
    n = (1 << 24) + 1
    assert grad(dy=mat(n, 7), x=mat(n, 40), dx=mat(n, 40), dw=None) == FAR
    assert grad(dy=mat(n, 7), x=mat(n, 40), dx=None, dw=None) == FAR


def test_cross_entropy_refusals(vc, at):
    ctx, mat = vc.Ctx(-1), make_mat(vc, at)
    ARG, SHAPE, STATE = vc.VCR_ERR_ARG, vc.VCR_ERR_SHAPE, vc.VCR_ERR_STATE

    def loss(x=mat(3, 7), label=at, o=(0.0, 0.0, 1, 1.0), each=at, total=at, d=mat(3, 7)):
        o = None if o is None else vc.VcrLossOpts(*o)
        return ctx.lib.vcr_cross_entropy(ctx.h, ref(x), label, ref(o), each, total, ref(d))
    assert loss() == STATE and loss(each=None, total=None, d=None) == STATE and loss(mat(3, 7, 1, 9), d=mat(3, 7, 0, 11)) == STATE
    assert loss(mat(0, 7, p=None), None, d=mat(0, 7, p=None)) == STATE
    nan, inf = float("nan"), float("inf")
    for o, want in (((1.0, 1e-4, 0, -3.0), STATE), ((-0.1, 0.0, 1, 1.0), ARG), ((1.1, 0.0, 1, 1.0), ARG), ((nan, 0.0, 1, 1.0), ARG),
                    ((0.0, -1.0, 1, 1.0), ARG), ((0.0, nan, 1, 1.0), ARG), ((0.0, inf, 1, 1.0), ARG), ((0.0, 0.0, 1, inf), ARG),
                    ((0.0, 0.0, 1, nan), ARG), (None, ARG)):
        assert loss(o=o) == want
    assert loss(None) == ARG and loss(label=None) == ARG and loss(label=at + 4) == ARG
    assert loss(each=at + 2) == ARG and loss(total=at + 1) == ARG and loss(d=mat(3, 8)) == SHAPE and loss(d=mat(2, 7)) == SHAPE


# ---- the oracle ------------------------------------------------------------------------------
def test_oracle_philox():
    """Known answers, published with the method (the words of pi among them)."""
    full = 0xffffffff
    for ctr, key, want in (((0, 0, 0, 0), (0, 0), "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
                           ((full,) * 4, (full, full), "408f276d 41c83b0e a20bc7c6 6d5451fd"),
                           ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
                            "d16cfe09 94fdcceb 5001e420 24126ea1")):
        assert " ".join("%08x" % w for w in o64.philox(np.array(ctr), key)) == want


def test_oracle_mask():
    m = o64.mask(400, 999, 0.3, 1 << 40, 5)
    k = o64.threshold(0.3)
    assert k == 19661 and set(np.unique(m)) == {0.0, 65536 / (65536 - k)}
    kept = (m > 0).mean()   # of n places: within five standard deviations
    assert abs(kept - (1 - k / 65536)) < 5 * np.sqrt(0.3 * 0.7 / m.size)
    # rows, columns, offsets and seeds differ; a part is the part of the whole
    np.testing.assert_array_equal(o64.mask(10, 50, 0.3, 1 << 40, 5, first_row=7), m[7:17, :50])
    for other in (o64.mask(400, 999, 0.3, 1 << 40, 6), o64.mask(400, 999, 0.3, 1, 5), np.roll(m, 1, 0), np.roll(m, 8, 1)):
        assert abs(((other > 0) == (m > 0)).mean() - 0.58) < 0.01   # as of independent ones
    assert (o64.mask(5, 9, 0.0, 1, 2) == 1.0).all()


@pytest.mark.parametrize("name", o64.ACTS)
def test_oracle_slopes_are_differences(name):
    z = np.random.default_rng(0).standard_normal(200) * 3
    z = z[np.abs(z) > 1e-3]
    h = 1e-5
    np.testing.assert_allclose((o64.act(z + h, name) - o64.act(z - h, name)) / (2 * h), o64.slope(z, name), atol=1e-8)


@pytest.mark.parametrize("smoothing,lse2", [(0.0, 0.0), (0.1, 0.0), (1.0, 0.3), (0.2, 0.01)])
def test_oracle_loss_gradient_is_the_differences(smoothing, lse2):
    rng = np.random.default_rng(1)
    x, t = rng.standard_normal((5, 7)) * 2, np.array([0, 6, -1, 3, 3])
    total, loss, d = o64.cross_entropy(x, t, smoothing, lse2)
    assert loss[2] == 0 and not d[2].any() and total == loss.sum() / 4
    h = 1e-5
    for r in range(5):
        for c in range(7):
            e = np.zeros_like(x)
            e[r, c] = h
            diff = (o64.cross_entropy(x + e, t, smoothing, lse2)[0] - o64.cross_entropy(x - e, t, smoothing, lse2)[0]) / (2 * h)
            assert abs(diff - d[r, c]) < 1e-8


def test_a_dropout_does_not_change(vc):
    d = vc.Dropout(0.25, 7, 9)
    packed = d._c
    for name, value in (("p", 0.5), ("seed", 8), ("offset", 10), ("step", None)):
        with pytest.raises(AttributeError):
            setattr(d, name, value)
    assert (d.p, d.seed, d.offset, d.step) == (0.25, 7, 9, None) and d._c == packed
