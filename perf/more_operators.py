"""The operators that train and run a network's layers in float, beside those in 4 bits, as they are measured: the
product with its bias, activation, dropout and residual in one call and its gradients, dropout whose mask is never
stored, and the loss of the answers with its gradient.

A case is one call on inputs drawn from the seed.  With `own` the calls go through `paper_2606_09377_amd.Ctx`; otherwise the same
is computed by elementary torch operations in float32.

Dropout keeps the value in column c of row r where the 16 random bits of that place are at least k = round(65536 p), and
multiplies it by 65536 / (65536 - k).  The bits are half h = c % 8 (the low half of word h / 2 where h is even) of the Philox 4x32-10 output
(Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011) for the counter (c / 8, r, offset's low word, offset's high
word) and the key (seed's low word, seed's high word).
"""
import math

import numpy as np
import torch

own = False

KINDS = ("linear", "grad", "dropout", "loss")
ACTS = ("none", "relu", "gelu", "silu")
LARGEST = 4096 * 8192 * 8192     # multiply-adds of one product
LARGEST_LOSS = 2048 * 262144


# ---- the cases ------------------------------------------------------------------------------
def listed():
    return [
        # one input through the first layer of the 784-1024x6 MLP: the smallest call
        dict(name="linear f32 1x784x1024", kind="linear", type="float32", rows=1, inner=784, cols=1024, act="relu",
             p=0.0, residual=False, keep_z=False),
        # one query through a wide layer, onto the residual it came from
        dict(name="linear bf16 1x8192x8192", kind="linear", type="bfloat16", rows=1, inner=8192, cols=8192, act="none",
             p=0.0, residual=True, keep_z=False),
        # a serving batch through a wide layer
        dict(name="linear bf16 48x8192x8192", kind="linear", type="bfloat16", rows=48, inner=8192, cols=8192,
             act="gelu", p=0.0, residual=False, keep_z=False),
        # an evaluation batch on widths that are no multiple of a tile
        dict(name="linear f32 2001x1000x1500", kind="linear", type="float32", rows=2001, inner=1000, cols=1500,
             act="relu", p=0.0, residual=True, keep_z=False),
        # a training batch through a layer of the wide MLP, with all that the epilogue does
        dict(name="linear bf16 4096x8192x8192", kind="linear", type="bfloat16", rows=4096, inner=8192, cols=8192,
             act="relu", p=0.1, residual=True, keep_z=True),
        # a training batch on a layer of the 784-1024x6 MLP
        dict(name="grad f32 64x1024x1024", kind="grad", type="float32", rows=64, inner=1024, cols=1024, act="relu",
             p=0.0, add=False),
        # a training batch on a layer of the wide MLP
        dict(name="grad bf16 4096x8192x8192", kind="grad", type="bfloat16", rows=4096, inner=8192, cols=8192,
             act="relu", p=0.1, add=True),
        # a small batch of odd width, on its own
        dict(name="dropout f32 777x1001", kind="dropout", type="float32", rows=777, cols=1001, p=0.5, residual=False),
        # a training batch of the wide MLP, onto its residual
        dict(name="dropout bf16 4096x8192", kind="dropout", type="bfloat16", rows=4096, cols=8192, p=0.1,
             residual=True),
        # a training batch of a classifier of ten classes: the smallest loss
        dict(name="loss f32 64x10", kind="loss", type="float32", rows=64, cols=10, pitch=0, smoothing=0.0, lse2=0.0),
        # a few answers over many classes, whose rows are longer than the classes
        dict(name="loss f32 5x100001", kind="loss", type="float32", rows=5, cols=100001, pitch=31, smoothing=0.1,
             lse2=0.0),
        # a training batch over as many classes as the widest layer has neurons
        dict(name="loss bf16 2048x262144", kind="loss", type="bfloat16", rows=2048, cols=262144, pitch=0,
             smoothing=0.0, lse2=1e-4),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm, of any remainder; a multiple of 64 a third of the
    time, as widths mostly are."""
    n = max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))
    return -(-n // 64) * 64 if hi % 64 == 0 and n > 64 and rng.random() < 0.33 else n


def draw(rng):
    kind = rng.choice(KINDS)
    case = dict(kind=kind, type=rng.choice(("float32", "bfloat16")))
    if kind == "loss":
        case |= dict(rows=_log(rng, 1, 8192), cols=_log(rng, 2, 262144), pitch=rng.choice((0, 0, 8, 31)),
                     smoothing=rng.choice((0.0, 0.1)), lse2=rng.choice((0.0, 1e-4)))
        limit = LARGEST_LOSS // (2 if case["type"] == "float32" else 1)
        if case["rows"] * (case["cols"] + case["pitch"]) > limit:
            case["rows"] = limit // (case["cols"] + case["pitch"])
        return case
    p = rng.choice((0.0, 0.1, 0.2, 0.5))
    if kind == "dropout":
        return {**case, "rows": _log(rng, 1, 4096), "cols": _log(rng, 10, 8192), "p": p or 0.3,
                "residual": rng.random() < 0.5}
    case |= dict(rows=_log(rng, 1, 4096), inner=_log(rng, 64, 8192), cols=_log(rng, 10, 8192), act=rng.choice(ACTS), p=p)
    limit = LARGEST // (4 if case["type"] == "float32" else 1)
    if case["rows"] * case["inner"] * case["cols"] > limit:
        case["rows"] = max(1, limit // (case["inner"] * case["cols"]))
    if kind == "grad":
        return {**case, "add": rng.random() < 0.5}
    return {**case, "residual": rng.random() < 0.5, "keep_z": rng.random() < 0.3}


# ---- inputs ---------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    kind, dt = case["kind"], getattr(torch, case["type"])
    s = {"case": case, "dtype": dt}
    m, n = case["rows"], case["cols"]
    if kind == "loss":
        # logits of a model that has learnt something: the label's is raised; one label in twenty is masked
        wide = torch.empty(m, n + case["pitch"], device="cuda", dtype=dt).normal_(0.0, 2.0, generator=g)
        logits = wide[:, :n]
        label = torch.randint(0, n, (m,), generator=g, device="cuda")
        logits[torch.arange(m, device="cuda"), label] += 4.0
        hidden = torch.rand(m, generator=g, device="cuda") < 0.05
        s["logits"], s["label"] = logits, torch.where(hidden, torch.full_like(label, -1), label)
        return s
    # (a program draws its generator's seed once and counts the calls)
    s["seed"], s["offset"] = 0x9E3779B97F4A7C15 * (seed + 1) % 2 ** 64, (seed << 20) + 7
    if kind == "dropout":
        s["x"] = normal(m, n).to(dt)
        s["residual"] = normal(m, n).to(dt) if case["residual"] else None
        return s
    k = case["inner"]
    s["w"] = (normal(n, k) * (2.0 / k) ** 0.5).to(dt)
    s["x"] = normal(m, k).relu_().to(dt)   # activations of the layer before
    if kind == "grad":
        s["dy"] = (normal(m, n) / m).to(dt)
        s["z"] = normal(m, n).to(dt) if case["act"] != "none" else None
        s["add"] = (normal(m, k) / m).to(dt) if case["add"] else None
        return s
    s["bias"] = normal(n) * 0.01
    s["residual"] = normal(m, n).to(dt) if case["residual"] else None
    return s


# ---- the plain forms ------------------------------------------------------------------------
def _times(a, b):
    """The high and low words of the products of a 32-bit constant and 32-bit words (held as int64)."""
    low = a * (b & 0xffff)
    mid = a * (b >> 16) + (low >> 16)
    return mid >> 16, ((mid & 0xffff) << 16) | (low & 0xffff)


def _kept(s, rows, cols):
    """Which values dropout keeps, and its factor."""
    k = round(65536 * s["case"]["p"])
    c0 = torch.arange(-(-cols // 8), device="cuda")[None].expand(rows, -1)
    c1 = torch.arange(rows, device="cuda")[:, None].expand_as(c0)
    c2 = torch.full_like(c0, s["offset"] & 0xffffffff)
    c3 = torch.full_like(c0, s["offset"] >> 32)
    k0, k1 = s["seed"] & 0xffffffff, s["seed"] >> 32
    for _ in range(10):
        h0, l0 = _times(0xD2511F53, c0)
        h1, l1 = _times(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    words = torch.stack((c0, c1, c2, c3), -1)
    bits = torch.stack((words & 0xffff, words >> 16), -1).view(rows, -1)[:, :cols]
    return bits >= k, 65536.0 / (65536 - k)


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(z * -math.sqrt(0.5))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.special.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    sig = 1 / (1 + torch.exp(-z))
    return sig * (1 + z * (1 - sig))


def _plain(s):
    case, dt = s["case"], s["dtype"]
    kind = case["kind"]
    if kind == "dropout":
        keep, factor = _kept(s, case["rows"], case["cols"])
        y = torch.where(keep, s["x"].float() * factor, 0.0)
        return (y if s["residual"] is None else y + s["residual"].float()).to(dt)
    if kind == "loss":
        x, t = s["logits"].float(), s["label"]
        n, sm, zc = case["cols"], case["smoothing"], case["lse2"]
        counted = t >= 0
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        total = e.sum(1, keepdim=True)
        lse = (top + total.log())[:, 0]
        at = t.clamp_min(0)[:, None]
        loss = lse - (1 - sm) * x.gather(1, at)[:, 0]
        if sm:
            loss = loss - sm * x.mean(1)
        if zc:
            loss = loss + zc * lse * lse
        loss = torch.where(counted, loss, 0.0)
        count = counted.sum().clamp_min(1)
        d = e * ((1 + 2 * zc * lse)[:, None] / total)
        if sm:
            d = d - sm / n
        d = d.scatter_add(1, at, torch.full_like(at, -(1 - sm), dtype=torch.float32))
        d = d * (counted / count)[:, None]
        return {"total": loss.sum() / count, "loss": loss, "dlogits": d.to(dt)}
    x, w = s["x"].float(), s["w"].float()
    if kind == "grad":
        g = s["dy"].float()
        if case["p"]:
            keep, factor = _kept(s, case["rows"], case["cols"])
            g = torch.where(keep, g * factor, 0.0)
        if s["z"] is not None:
            g = g * _slope(s["z"].float(), case["act"])
        dx = g @ w
        return {"dx": (dx if s["add"] is None else dx + s["add"].float()).to(dt), "dw": (g.T @ x).to(dt), "db": g.sum(0)}
    z = x @ w.T + s["bias"]
    y = _act(z, case["act"])
    if case["p"]:
        keep, factor = _kept(s, case["rows"], case["cols"])
        y = torch.where(keep, y * factor, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(dt), "z": z.to(dt)} if case["keep_z"] else {"y": y.to(dt)}


# ---- the framework's calls ------------------------------------------------------------------
_context = []


def _ctx():
    if not _context:
        from paper_2606_09377_amd import Ctx
        _context.append(Ctx(0))
    return _context[0]


def _own(s):
    from paper_2606_09377_amd import Dropout
    ctx, case = _ctx(), s["case"]
    kind = case["kind"]
    if kind == "loss":
        total, loss, dlogits = ctx.cross_entropy(s["logits"], s["label"], smoothing=case["smoothing"], lse2=case["lse2"])
        return {"total": total, "loss": loss, "dlogits": dlogits}
    drop = Dropout(case["p"], s["seed"], s["offset"]) if case["p"] else None
    if kind == "dropout":
        return ctx.dropout(s["x"], drop, residual=s["residual"])
    if kind == "grad":
        dx, dw, db = ctx.linear_grad(s["dy"], s["x"], s["w"], z=s["z"], act=case["act"], dropout=drop, add=s["add"])
        return {"dx": dx, "dw": dw, "db": db}
    y = ctx.linear(s["x"], s["w"], bias=s["bias"], act=case["act"], dropout=drop, residual=s["residual"],
                   keep_z=case["keep_z"])
    return {"y": y[0], "z": y[1]} if case["keep_z"] else {"y": y}


def run(state):
    return _own(state) if own else _plain(state)


# ---- floors and 64 bits ---------------------------------------------------------------------
def work(case):
    t = 4 if case["type"] == "float32" else 2
    kind, m, n = case["kind"], case["rows"], case["cols"]
    if kind == "dropout":
        return {"bytes": m * n * t * (3 if case["residual"] else 2), "flops": 0}
    if kind == "loss":
        return {"bytes": m * n * 2 * t + 12 * m, "flops": 0}
    k = case["inner"]
    if kind == "grad":
        each = 2 if case["act"] != "none" else 1
        return {"bytes": t * (m * n * each + m * k * (3 if case["add"] else 2) + 2 * n * k) + 4 * n, "flops": 4 * m * n * k}
    outs = 1 + case["residual"] + case["keep_z"]
    return {"bytes": t * (m * k + n * k + m * n * outs) + 4 * n, "flops": 2 * m * n * k}


def _mask64(case, s):
    """Dropout's factors in 64 bits, by numpy's 64-bit products."""
    rows, cols = case["rows"], case["cols"]
    word = np.uint64(0xffffffff)
    groups = (cols + 7) // 8
    ctr = [np.tile(np.arange(groups, dtype=np.uint64), rows), np.repeat(np.arange(rows, dtype=np.uint64), groups),
           np.full(rows * groups, s["offset"] % 2 ** 32, dtype=np.uint64), np.full(rows * groups, s["offset"] // 2 ** 32, dtype=np.uint64)]
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
    for r in range(10):
        a, b = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        kr = [np.uint64((key[0] + r * 0x9E3779B9) % 2 ** 32), np.uint64((key[1] + r * 0xBB67AE85) % 2 ** 32)]
        ctr = [(b >> np.uint64(32)) ^ ctr[1] ^ kr[0], b & word, (a >> np.uint64(32)) ^ ctr[3] ^ kr[1], a & word]
    halves = np.stack([c.astype(np.uint32) for c in ctr], 1).view("<u2").reshape(rows, groups * 8)[:, :cols]
    k = int(round(case["p"] * 65536))
    return torch.as_tensor(np.where(halves < k, 0.0, 65536.0 / (65536.0 - k))).cuda()


def exact(case, seed):
    """run()'s outputs from the operators' definitions in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "loss":
        count = max(1, int((s["label"] >= 0).sum()))
        n, sm, zc = case["cols"], case["smoothing"], case["lse2"]
        loss = torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
        d = torch.zeros(case["rows"], n, dtype=torch.float64, device="cuda")
        step = max(1, 2 ** 26 // n)
        for i in range(0, case["rows"], step):
            x, t = s["logits"][i:i + step].double(), s["label"][i:i + step]
            want = torch.full_like(x, sm / n)
            here = torch.nonzero(t >= 0)[:, 0]
            want[here, t[here]] += 1 - sm
            lse = torch.logsumexp(x, 1)
            each = (want * (lse[:, None] - x)).sum(1) + zc * lse ** 2
            loss[i + here] = each[here]
            q = (1 + 2 * zc * lse)[:, None] * torch.softmax(x, 1) - want
            d[i + here] = q[here] / count
        return {"total": loss.sum() / count, "loss": loss, "dlogits": d}
    mask = _mask64(case, s) if case["p"] else 1.0
    if kind == "dropout":
        y = mask * s["x"].double()
        return y if s["residual"] is None else y + s["residual"].double()
    x, w = s["x"].double(), s["w"].double()
    act = case["act"]
    if kind == "grad":
        g = mask * s["dy"].double()
        if act != "none":
            z = s["z"].double().requires_grad_()
            with torch.enable_grad():
                f = {"relu": torch.nn.functional.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[act]
                slope, = torch.autograd.grad(f(z).sum(), z)
            g = g * slope
        dx = torch.matmul(g, w)
        return {"dx": dx if s["add"] is None else dx + s["add"].double(), "dw": torch.matmul(g.t().contiguous(), x), "db": g.sum(0)}
    z = torch.matmul(x, w.t()) + s["bias"].double()
    y = z
    if act == "relu":
        y = z.clamp_min(0)
    elif act == "gelu":   # z Phi(z)
        y = z * torch.exp(torch.special.log_ndtr(z))
    elif act == "silu":
        y = z * torch.sigmoid(z)
    y = mask * y
    if s["residual"] is not None:
        y = y + s["residual"].double()
    return {"y": y, "z": z} if case["keep_z"] else {"y": y}
