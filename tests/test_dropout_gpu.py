"""Dropout on the GPU (vcr_dropout) against 64 bits and the published generator.  A kept value is multiplied by a
float32 factor (itself rounded) and rounded to the result's type, and a residual's addition rounds once before that."""
import numpy as np
import pytest

from oracle import dense64 as o64

pytestmark = pytest.mark.gpu
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    from paper_2606_09377_amd import Ctx
    return Ctx(0)


def host(t):
    return t.double().cpu().numpy()


def view(rows, cols, dtype, pitch, shift, g):
    import torch
    buf = torch.randn((rows, cols + pitch + shift), generator=g, device="cuda").to(getattr(torch, dtype))
    return buf[:, shift:shift + cols], buf


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (7, 13), (64, 1000), (333, 257), (1500, 4096), (3, 100003)])
def test_dropout(ctx, rows, cols):
    import torch
    from paper_2606_09377_amd import Dropout
    g = torch.Generator("cuda").manual_seed(rows + cols)
    for src, dst, p, pitch, shift in (("float32", "float32", 0.5, 0, 0), ("bfloat16", "bfloat16", 0.1, 8, 8), ("float32", "bfloat16", 0.9, 3, 1),
                                      ("bfloat16", "float32", 0.0, 0, 0), ("float32", "float32", 1e-3, 4, 4)):
        x, _ = view(rows, cols, src, pitch, shift, g)
        res, _ = view(rows, cols, "bfloat16", shift, pitch, g)
        out, buf = view(rows, cols, dst, pitch, shift, g)
        before = buf.clone()
        seed, offset = int(torch.randint(0, 2 ** 62, (1,))), int(torch.randint(0, 2 ** 62, (1,)))
        m = o64.mask(rows, cols, p, seed, offset)
        drop = Dropout(p, seed, offset)
        y = host(ctx.dropout(x, drop, out=out))
        want = o64.dropout(host(x), m)
        assert (np.abs(y - want) <= (2 * 2.0 ** -24 + HALF[dst]) * 1.01 * np.abs(want)).all() and not y[m == 0].any()
        before[:, shift:shift + cols] = out
        assert torch.equal(before, buf)
        y = host(ctx.dropout(x, drop, residual=res, dtype=getattr(torch, dst)))
        both = want + host(res)
        assert (np.abs(y - both) <= 3 * 2.0 ** -24 * np.abs(want) + (2.0 ** -24 + HALF[dst]) * 1.01 * np.abs(both)).all()
        # over the inputs
        for over in (x.clone(), res.to(x.dtype)):
            r = over if over.data_ptr() != x.data_ptr() and over.shape == res.shape else None
            a = ctx.dropout(x, drop, residual=res.to(x.dtype))
            t = x.clone()
            assert torch.equal(ctx.dropout(t, drop, residual=res.to(x.dtype), out=t), a)
            t = res.to(x.dtype)
            assert torch.equal(ctx.dropout(x, drop, residual=t, out=t), a)
            del r


def test_step_moves_the_mask(ctx):
    """offset + step, modulo 2^64, is what counts."""
    import torch
    from paper_2606_09377_amd import Dropout
    x = torch.ones((40, 100), device="cuda")
    step = torch.tensor([0], device="cuda")
    d = Dropout(0.5, 77, 2 ** 64 - 2, step)
    for i in range(4):
        y = host(ctx.dropout(x, d))
        np.testing.assert_array_equal(y, o64.mask(40, 100, 0.5, 77, (2 ** 64 - 2 + i) % 2 ** 64))
        step += 1
    step.fill_(-5)
    np.testing.assert_array_equal(host(ctx.dropout(x, d)), o64.mask(40, 100, 0.5, 77, 2 ** 64 - 7))


def test_dropped_values_are_zero_whatever_they_were(ctx):
    import torch
    from paper_2606_09377_amd import Dropout
    m = o64.mask(50, 70, 0.5, 3, 4)
    x = torch.full((50, 70), float("nan"), device="cuda")
    y = host(ctx.dropout(x, Dropout(0.5, 3, 4)))
    assert np.isnan(y[m > 0]).all() and not y[m == 0].any()


def test_no_rows_and_many(ctx):
    """A matrix of no rows; one of more than 2^32 elements, whose last rows are its own."""
    import torch
    from paper_2606_09377_amd import Dropout
    assert ctx.dropout(torch.empty((0, 5), device="cuda"), Dropout(0.5)).shape == (0, 5)
    rows, cols = 540_001, 8000
    x = torch.ones((rows, cols), dtype=torch.bfloat16, device="cuda")
    ctx.dropout(x, Dropout(0.25, 6, 7), out=x)
    want = o64.mask(40, cols, 0.25, 6, 7, first_row=rows - 40)
    np.testing.assert_allclose(host(x[-40:]), want, rtol=2.0 ** -8)
    assert abs(float((x[::1000] > 0).float().mean()) - 0.75) < 5 * (0.75 * 0.25 / (541 * cols)) ** 0.5


def test_refusals_of_the_binding(ctx):
    import torch
    from paper_2606_09377_amd import Dropout, VcrError
    x = torch.ones((4, 6), device="cuda")
    with pytest.raises(VcrError):
        ctx.dropout(x, Dropout(1.0))
    for bad in (x.double(), x[0], x.t(), x.cpu()):
        with pytest.raises(ValueError):
            ctx.dropout(bad, Dropout(0.5))
    with pytest.raises(VcrError):
        ctx.dropout(x, Dropout(0.5), residual=x[:3])
