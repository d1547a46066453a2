"""Layers in 4 bits on the GPU where calls go wrong most easily: nothing to do."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2606_09377_amd import Ctx
    return Ctx(0)


@pytest.mark.parametrize("need", [(False, False, True), (True, False, True), (False, True, False), (True, True, True),
                                  (True, False, False)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradients_of_no_rows(ctx, dtype, need):
    """Sums over an empty batch are zero, whichever of them are asked for."""
    import torch
    dt = getattr(torch, dtype)
    w = ctx.mx_quantize(torch.randn((150, 40), device="cuda"))
    x, dy = torch.empty((0, 40), dtype=dt, device="cuda"), torch.empty((0, 150), dtype=dt, device="cuda")
    dirt = [torch.full(s, float("nan"), device="cuda") for s in ((150,), (150, 40))]
    del dirt   # (what the outputs are allocated from)
    for y in (None, dy):
        dx, dw, db = ctx.mx_linear_grad(dy, x, w, y=y, need=need)
        torch.cuda.synchronize()
        assert (dx is not None, dw is not None, db is not None) == need
        assert dx is None or dx.shape == (0, 40)
        assert dw is None or (dw.shape == (150, 40) and not dw.any())
        assert db is None or (db.shape == (150,) and not db.any())
