"""A product whose tiles have more than 2^32 threads, on the GPU: all of its 2^36 results.

Tolerance: sums of 64 products of float32 values, here and in float32 by the library, are each off by at most (4 + 2 sqrt(64)) 2^-23 of the sum of
magnitudes (test_dense_gpu.py), which is at most 64 times the largest of x and w; the residual's addition rounds by 2^-24 and the result to bf16 by 2^-8 of
itself."""
import pytest

pytestmark = pytest.mark.gpu


def test_more_tiles_than_a_launch_counts():
    import torch
    from paper_2606_09377_amd import Ctx
    m, k, n = 10443640, 64, 6600
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 190e9:
        pytest.skip("needs 190 GB of device memory")
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.rand((m, k), generator=g, device="cuda") - 0.5
    w = torch.rand((n, k), generator=g, device="cuda") - 0.5
    y = torch.full((m, n), 0.25, dtype=torch.bfloat16, device="cuda")
    ctx = Ctx(0)
    ctx.linear(x, w, act="relu", residual=y, out=y)
    wt = w.t().contiguous()
    sums = 2 * (4 + 2 * 8) * 2.0 ** -23 * 64 * 0.25
    for i in range(0, m, 300_000):
        want = torch.mm(x[i:i + 300_000], wt).relu_().add_(0.25)
        off = (y[i:i + 300_000].float() - want).abs_()
        assert bool((off <= want.mul_(2.0 ** -8 * 1.01).add_(sums)).all()), i
    del x, y, want, off
    ctx.close()
    torch.cuda.empty_cache()
