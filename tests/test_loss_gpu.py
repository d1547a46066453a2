"""Cross entropy on the GPU (vcr_cross_entropy) against 64 bits.

Tolerances.  x - m rounds to 2^-24 of itself and so does its product with log2 e, so exp(x - m) is off by 2 |x - m| 2^-24 of itself
and a unit or two of the instruction, the sum of such terms by that of the largest |x - m| that counts and its additions.  With |x - m| up to R
and n classes summed by threads and then pairwise, (2 R + 16 + sqrt(n)) 2^-24 of a probability is allowed, twice for its factor 1 / sum.
A loss adds terms of |m|, |x_t|, |mean x| and |log sum|, each rounded: 8 2^-24 of their magnitudes and the sum's."""
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


def host(t):
    return t.double().cpu().numpy()


def check(ctx, x, label, dtype="float32", pitch=0, shift=0, out_type=None, **opts):
    """x (numpy) and label through the call, against the oracle."""
    import torch
    rows, n = x.shape
    buf = torch.full((rows, n + pitch + shift), 3.0, dtype=getattr(torch, dtype), device="cuda")
    t = buf[:, shift:shift + n]
    t.copy_(torch.as_tensor(x))
    lt = torch.as_tensor(label).cuda()
    out = torch.full((rows, n + pitch), 5.0, dtype=getattr(torch, out_type or dtype), device="cuda")
    total, loss, d = ctx.cross_entropy(t, lt, out=out[:, :n], **opts)
    v = host(t)
    want = o64.cross_entropy(v, label, **opts)
    s, c, scale = opts.get("smoothing", 0.0), opts.get("lse2", 0.0), opts.get("scale", 1.0)
    count = max(1, int((label >= 0).sum())) if opts.get("mean", True) else 1
    seen = np.where((label >= 0)[:, None], v, 0.0)
    top = seen.max(1)
    R = min(100.0, np.nanmax(np.where(np.isfinite(seen), top[:, None] - seen, 0.0)))
    each = (2 * R + 16 + np.sqrt(n)) * E
    e = np.abs(seen.max(1)) + np.log(n)
    t_loss = 8 * E * (e + np.abs(seen).max(1)) + 2 * each + c * e * e * 16 * E + c * 4 * e * each
    np.testing.assert_array_equal(np.isnan(host(loss)), np.isnan(want[1]))
    assert (np.abs(host(loss) - want[1]) <= t_loss)[np.isfinite(want[1])].all(), np.abs(host(loss) - want[1]).max()
    if np.isfinite(want[0]):
        assert abs(float(total) - want[0]) <= (t_loss.sum() + (8 + np.sqrt(rows)) * E * np.abs(want[1]).sum()) / count
    else:
        assert not np.isfinite(float(total))
    q = want[2] * count / scale + (s / n + (1 - s) * (np.arange(n) == label[:, None])) * (label >= 0)[:, None]   # (1 + 2 c e) p
    tol = abs(scale) / count * (3 * each * np.abs(q) + 4 * E * (np.abs(q) + 1.0 * (np.arange(n) == label[:, None]) + s / n)
                                + c * 2 * (t_loss + 8 * E * e)[:, None] * np.abs(q)) + 2.0 ** -149
    o = out_type or dtype
    tol = tol + HALF[o] * (np.abs(want[2]) + tol)
    bad = ~(np.abs(host(d) - want[2]) <= tol) & ~(np.isnan(host(d)) & np.isnan(want[2]))
    assert not bad.any(), (np.argwhere(bad)[:3], host(d)[bad][:3], want[2][bad][:3], tol[bad][:3])
    assert bool((out[:, n:] == 5.0).all())
    return t, lt, total, loss, d


SIZES = [(1, 1), (1, 2), (64, 10), (5, 17), (100, 100), (3, 64), (2, 513), (300, 1000), (33, 2048), (7, 2049), (5, 4100), (3, 8192),
         (4, 16385), (2, 33000), (3, 65537), (2, 100001), (1, 131080), (2, 262144), (1, 300007), (600, 5000), (1300, 9)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,n", SIZES)
def test_cross_entropy(ctx, rows, n, dtype):
    rng = np.random.default_rng(rows * 7 + n)
    x = 3 * rng.standard_normal((rows, n))
    label = rng.integers(0, n, rows)
    label[rng.random(rows) < 0.1] = -1
    for (pitch, shift), out, opts in (((0, 0), None, {}), ((8, 8), None, dict(smoothing=0.1, mean=False, scale=0.5)),
                                      ((3, 1), "float32", dict(lse2=1e-3, scale=-2.0)), ((31, 0), "bfloat16", dict(smoothing=1.0, lse2=0.01))):
        check(ctx, x, label, dtype, pitch, shift, out, **opts)


@pytest.mark.parametrize("rows,n", [(3, 9), (4, 700), (3, 5000), (2, 40000), (3, 270000)])
def test_masked_labels_logits_and_wrong_labels(ctx, rows, n):
    import torch
    rng = np.random.default_rng(n)
    lowest = float(np.finfo(np.float32).min)
    x = rng.standard_normal((rows, n)).astype(np.float32)
    label = rng.integers(0, n, rows)
    # no row counts: nothing is read
    t, _, total, loss, d = check(ctx, np.full_like(x, np.nan), np.full(rows, -100))
    assert float(total) == 0 and not loss.any() and not d.any()
    # a row whose label is masked may hold anything
    y = x.copy()
    y[0] = np.nan
    lab = label.copy()
    lab[0] = -1
    check(ctx, np.nan_to_num(y, nan=0.0), lab)
    _, loss, d = ctx.cross_entropy(torch.as_tensor(y).cuda(), torch.as_tensor(lab).cuda())
    assert float(loss[0]) == 0 and not d[0].any() and bool(torch.isfinite(d).all())
    # -infinity and the type's lowest value as masks of classes
    for hide in (-np.inf, lowest):
        y = x.copy()
        y[:, 1::2] = hide
        y[1, :] = hide
        y[1, n - 1] = 0.5   # one class left
        lab = label // 2 * 2
        lab[1] = n - 1
        got = ctx.cross_entropy(torch.as_tensor(y).cuda(), torch.as_tensor(lab).cuda())
        want = o64.cross_entropy(y, lab)
        np.testing.assert_allclose(host(got[1]), want[1], rtol=1e-5, atol=1e-6)
        np.testing.assert_allclose(host(got[2]), want[2], rtol=2e-5, atol=1e-7)
    # a row of the lowest value alone is uniform; of -infinity alone, NaN; +infinity and NaN, NaN
    y = np.full_like(x, lowest)
    loss, d = (host(v) for v in ctx.cross_entropy(torch.as_tensor(y).cuda(), torch.as_tensor(label).cuda(), mean=False)[1:])
    np.testing.assert_allclose(loss, np.log(n), rtol=1e-6)
    np.testing.assert_allclose(d[0], 1 / n - (np.arange(n) == label[0]), rtol=1e-5)
    for v in (-np.inf, np.inf, np.nan):
        y = x.copy()
        y[0, :] = v
        y[1, n // 2] = v
        total, loss, d = (host(v) for v in ctx.cross_entropy(torch.as_tensor(y).cuda(), torch.as_tensor(label).cuda()))
        assert np.isnan(loss[0]) and np.isnan(d[0]).all() and np.isnan(total) and np.isfinite(loss[2:]).all()
        assert np.isfinite(d[1]).all() if v == -np.inf else np.isnan(d[1]).all()
    # a label beyond the classes: NaN, for its row alone
    lab = label.copy()
    lab[0] = n
    check(ctx, x, lab)
    lab[0] = 2 ** 40
    check(ctx, x, lab)


def test_infinite_loss(ctx):
    """A label whose logit is -infinity, and smoothing over such a logit."""
    import torch
    x = torch.zeros((2, 40), device="cuda")
    x[0, 3] = x[1, 5] = -float("inf")
    t = torch.tensor([3, 4], device="cuda")
    total, loss, d = ctx.cross_entropy(x, t)
    assert float(loss[0]) == float("inf") and float(total) == float("inf") and bool(torch.isfinite(d).all()) and bool(torch.isfinite(loss[1]))
    _, loss, d = ctx.cross_entropy(x, t, smoothing=0.1)
    assert bool((loss == float("inf")).all()) and bool(torch.isfinite(d).all())
    x[1, 5] = 0.0
    _, loss, _ = ctx.cross_entropy(x, t, smoothing=1.0)
    assert float(loss[0]) == float("inf") and abs(float(loss[1]) - np.log(40)) < 1e-5


def test_large_logits(ctx):
    """Values near float32's ends give what 64 bits give."""
    import torch
    x = np.array([[3e38, 2.9e38, -3e38, 0], [-3e38, -3.2e38, -3.4e38, -3.1e38], [1e-38, -1e-40, 0, 1e-45], [88, -88, 700, 699.5]], dtype=np.float32)
    label = np.array([0, 0, 1, 3])
    _, loss, d = ctx.cross_entropy(torch.as_tensor(x).cuda(), torch.as_tensor(label).cuda(), mean=False)
    want = o64.cross_entropy(x, label, mean=False)
    np.testing.assert_allclose(host(loss), want[1], rtol=1e-6, atol=1e-6)
    np.testing.assert_allclose(host(d), want[2], rtol=1e-4, atol=1e-7)   # (e^-200 and less are 0 in float32)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,n", [(9, 30), (5, 3000), (3, 20000), (2, 150000), (1, 262144)])
def test_in_place_and_outputs_left_out(ctx, rows, n, dtype):
    import torch
    from paper_2606_09377_amd.vcrown import _LOSS, _mat
    rng = np.random.default_rng(n)
    x = torch.as_tensor(rng.standard_normal((rows, n))).to(getattr(torch, dtype)).cuda()
    t = torch.as_tensor(rng.integers(-1, n, rows)).cuda()
    total, loss, d = ctx.cross_entropy(x, t, smoothing=0.1, lse2=1e-3)
    y = x.clone()
    got = ctx.cross_entropy(y, t, smoothing=0.1, lse2=1e-3, out=y)
    assert got[2].data_ptr() == y.data_ptr() and all(torch.equal(a, b) for a, b in zip(got, (total, loss, d)))
    t2, l2, none = ctx.cross_entropy(x, t, smoothing=0.1, lse2=1e-3, grad=False)
    assert none is None and torch.equal(t2, total) and torch.equal(l2, loss)
    alone = torch.full((3,), 9.0, device="cuda")
    for each, tot, dl in ((0, alone.data_ptr(), None), (0, 0, _mat(y)), (0, 0, None)):
        y.fill_(4.0)
        ctx._check(ctx.lib.vcr_cross_entropy(ctx.h, _mat(x), t.data_ptr(), _LOSS.pack(0.1, 1e-3, 1, 1.0), each, tot, dl))
        assert (float(alone[0]) == float(total)) and float(alone[1]) == 9.0
        assert torch.equal(y, d) if dl else bool((y == 4.0).all())


def test_gradient_is_the_differences(ctx):
    """Of the loss in 64 bits, at float32's logits."""
    import torch
    rng = np.random.default_rng(0)
    x, label = rng.standard_normal((6, 50)).astype(np.float32), np.array([3, -1, 49, 0, 7, 7])
    d = host(ctx.cross_entropy(torch.as_tensor(x).cuda(), torch.as_tensor(label).cuda(), smoothing=0.05, lse2=0.02, scale=3.0)[2])
    h = 1e-5
    for r, c in [(0, 3), (0, 4), (1, 2), (2, 49), (5, 7), (5, 8), (3, 30)]:
        e = np.zeros(x.shape)
        e[r, c] = h
        v = [o64.cross_entropy(x + s * e, label, 0.05, 0.02)[0] for s in (1, -1)]
        assert abs(3.0 * (v[0] - v[1]) / (2 * h) - d[r, c]) <= 1e-6


def test_repeats_no_rows_and_refusals(ctx):
    import torch
    from paper_2606_09377_amd import VcrError
    g = torch.Generator("cuda").manual_seed(0)
    x, t = torch.randn((700, 3001), generator=g, device="cuda"), torch.randint(-1, 3001, (700,), generator=g, device="cuda")
    first = ctx.cross_entropy(x, t)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for s in streams * 3:
        with torch.cuda.stream(s):
            got.append(ctx.cross_entropy(x, t))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for r in got for a, b in zip(r, first))
    total, loss, d = ctx.cross_entropy(x[:0], t[:0])
    assert float(total) == 0 and loss.shape == (0,) and d.shape == (0, 3001)
    for args in ((x, t.int()), (x, t[:-1]), (x, t.cpu()), (x.t(), t), (x.double(), t), (x, t[::2])):
        with pytest.raises(ValueError):
            ctx.cross_entropy(*args)
    with pytest.raises(VcrError):
        ctx.cross_entropy(x, t, smoothing=1.5)
    with pytest.raises(VcrError):
        ctx.cross_entropy(x, t, out=torch.empty((700, 3000), device="cuda"))


def test_offsets_beyond_32_bits(ctx):
    """Logits of over 2^32 elements: the last row is its own."""
    import torch
    rows, n = 16400, 262144
    x = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    x[-1].normal_(generator=torch.Generator("cuda").manual_seed(1))
    last = x[-1:].clone()
    t = torch.full((rows,), 5, device="cuda")
    total, loss, d = ctx.cross_entropy(x, t, mean=False, out=x)
    _, one, g = ctx.cross_entropy(last, t[:1], mean=False)
    assert abs(float(loss[0]) - np.log(n)) < 1e-5 and abs(float(loss[-1]) - float(one[0])) < 1e-5
    assert torch.equal(d[0], d[-2]) and torch.allclose(d[-1].float(), g[0].float(), rtol=2.0 ** -7, atol=0)
