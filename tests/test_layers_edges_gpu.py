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


def test_statistics_count_every_workspace():
    """The peak is at least what is held, and rooms kept for a recorded graph are held."""
    import torch
    from paper_2606_09377_amd import Ctx
    from workloads import random_mlp
    c = Ctx(0)

    def held():
        s = c.stats()
        assert s["peak_workspace_bytes"] >= s["workspace_bytes"], s
        return s["workspace_bytes"]
    w = c.mx_quantize(torch.randn((640, 640), device="cuda"))
    x = torch.randn((600, 640), device="cuda")
    c.mx_linear(x, w)
    room = held()
    assert room > 0
    wl = random_mlp(7, [40, 150, 130, 10], 3, 0.05)   # a bounds call that holds less than the layer call
    c.load_net(wl.net)
    c.crown_bounds(torch.from_numpy(wl.x0).cuda(), wl.eps, torch.from_numpy(wl.C).cuda())
    both = held()
    assert both > room
    # a room that a graph was recorded with is kept beside the larger one that takes its place
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        c.mx_linear(x, w)
    torch.cuda.synchronize()
    one = held() - both
    assert one > 0
    with torch.cuda.graph(graph, stream=side):
        c.mx_linear(x, w)
    with torch.cuda.stream(side):
        c.mx_linear(torch.randn((2000, 640), device="cuda"), w)
    torch.cuda.synchronize()
    assert held() >= both + 3 * one


def test_cap_holds_over_all_streams():
    """Rooms of other streams give way under the cap; those of recorded graphs stay."""
    import torch
    from paper_2606_09377_amd import Ctx, VcrError
    from paper_2606_09377_amd.vcrown import OPT_WORKSPACE_CAP_BYTES, VCR_ERR_OOM
    c = Ctx(0)
    w = c.mx_quantize(torch.randn((640, 640), device="cuda"))
    x = torch.randn((600, 640), device="cuda")
    want = c.mx_linear(x, w)
    torch.cuda.synchronize()
    room = c.stats()["workspace_bytes"]
    c.set_option(OPT_WORKSPACE_CAP_BYTES, room + room // 2)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(2):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(c.mx_linear(x, w))
            assert c.stats()["workspace_bytes"] <= room + room // 2
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[-1]):
        y = c.mx_linear(x, w)
    with pytest.raises(VcrError) as e:
        with torch.cuda.stream(streams[0]):
            c.mx_linear(x, w)
    assert e.value.status == VCR_ERR_OOM
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    c.set_option(OPT_WORKSPACE_CAP_BYTES, 0)
    with torch.cuda.stream(streams[0]):
        again = c.mx_linear(x, w)
    torch.cuda.synchronize()
    assert torch.equal(again, want) and c.stats()["workspace_bytes"] >= 2 * room


def test_more_rows_than_a_launch_has_threads_for(ctx):
    """2^28 rows are 2^24 workgroups of 256: more threads than one launch counts."""
    import torch
    from oracle import layers64 as o64
    rows, step = (1 << 28) + 72, 1 << 26   # a stretch of launches is 2^26 rows
    g = torch.Generator("cuda").manual_seed(6)
    x = torch.randn((rows, 3), generator=g, device="cuda")
    q = ctx.mx_quantize(x)
    y = torch.full((rows, 3), float("nan"), device="cuda")
    ctx.mx_dequantize(q, out=y)
    assert not bool(y.isnan().any())
    for at in [0] + [i * step - 300 for i in range(1, 5)] + [rows - 500]:
        part = slice(at, min(at + 600, rows))
        want = o64.values(*o64.quantize(x[part].double().cpu().numpy()))
        np.testing.assert_array_equal(y[part].double().cpu().numpy(), want)
    del x, y, q
    torch.cuda.empty_cache()


def test_more_columns_than_a_launch_has_threads_for():
    """The column sums of one row are that row, up to the largest one."""
    import torch
    from paper_2606_09377_amd import Ctx
    ctx, n = Ctx(0), 1 << 30
    dy = torch.randn((1, n), generator=torch.Generator("cuda").manual_seed(7), device="cuda")
    db = ctx.mx_linear_grad(dy, None, None, need=(False, False, True))[2]
    assert torch.equal(db, dy[0])
    del dy, db
    ctx.close()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,cols", [(0, 40), (1, 1), (17, 130)])
def test_pack_and_unpack(ctx, rows, cols):
    """Codes and scales in row order and back, no rows among them."""
    import torch
    from paper_2606_09377_amd import MX
    codes = torch.randint(0, 256, (rows, -(-cols // 2)), dtype=torch.uint8, device="cuda")
    if cols % 2:
        codes[:, -1] &= 15
    scales = torch.randint(100, 150, (rows, -(-cols // 32)), dtype=torch.uint8, device="cuda")
    q = MX.pack(codes, scales, cols)
    assert (q.rows, q.cols) == (rows, cols)
    c, s = q.unpack()
    assert torch.equal(c, codes) and torch.equal(s, scales)
    x = torch.randn((3, cols), device="cuda")
    assert ctx.mx_dequantize(q).shape == (rows, cols)
    if rows:
        assert ctx.mx_linear(x, q).shape == (3, rows)


@pytest.mark.parametrize("m", [1, 3, 40, 300])
@pytest.mark.parametrize("byte", [0, 1, 2, 252, 253, 254])
def test_scales_at_the_ends(ctx, byte, m):
    """The smallest and largest scales.  Operands are small whole numbers times powers of two: every sum is exact."""
    import torch
    from oracle import layers64 as o64
    from paper_2606_09377_amd import MX
    rng = np.random.default_rng(byte)
    k, n = 200, 50
    codes = rng.integers(0, 16, (n, k)).astype(np.uint8)
    codes[:8] &= 11   # some rows without values of 4 and 6 (and 2 and 3)
    scales = np.full((n, -(-k // 32)), byte, np.uint8)
    w = MX.pack(torch.as_tensor(codes[:, ::2] | codes[:, 1::2] << 4).cuda(), torch.as_tensor(scales).cuda(), k)
    wv = o64.values(codes, scales)
    other = 2.0 ** np.clip(127 - byte, -120, 120)
    x = rng.integers(1, 9, (m, k)) * other
    dy = rng.integers(1, 9, (m, n)) * other
    inf = np.abs(wv) >= 2.0 ** 128   # as bf16 or float32 values, though not as 4-bit ones
    for dt in (torch.float32, torch.bfloat16):
        t, g = torch.as_tensor(x, dtype=dt).cuda(), torch.as_tensor(dy, dtype=dt).cuda()
        y = ctx.mx_linear(t, w, out=torch.empty((m, n), device="cuda")).double().cpu().numpy()
        ok = ~inf.any(1)
        np.testing.assert_array_equal(y[:, ok], (x @ wv.T)[:, ok])
        assert not np.isfinite(y[:, ~ok]).any() and ok.any()
        dx = ctx.mx_linear_grad(g.float(), None, w, need=(True, False, False))[0].double().cpu().numpy()
        ok = ~inf.any(0)
        np.testing.assert_array_equal(dx[:, ok], (dy @ wv)[:, ok])
        assert not np.isfinite(dx[:, ~ok]).any()
        q = ctx.mx_quantize(t)
        p = ctx.mx_product(q, w).double().cpu().numpy()
        np.testing.assert_array_equal(p, ctx.mx_dequantize(q).double().cpu().numpy() @ wv.T)
