"""Train a small classifier through 4-bit weights, store it in 4 bits, answer with it and verify it as stored.

    python examples/train_store_verify.py [--steps 60] [--eps 0.01]

Every step quantises the weights, runs the layers with them (vcr_mx_linear), takes the gradients through them
(vcr_mx_linear_grad) and moves the float32 weights by orthogonalised momentum (vcr_orthogonalize).  The network
that answers then holds 4-bit weights only; the same weights, read back, are loaded into the verifier, so that its
bounds are of the network that answers.  Synthetic data: inputs around two centres in the unit box for each of 4 classes.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_09377_amd import Ctx  # noqa: E402
from workloads import Net, Node  # noqa: E402

DIMS = (64, 200, 200, 4)


def data(g, n):
    """Inputs near one of 8 centres of [0, 1]^64, two a class."""
    centres = torch.rand(8, DIMS[0], generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    which = torch.randint(0, 8, (n,), generator=g, device="cuda")
    x = centres[which] + 0.1 * torch.randn(n, DIMS[0], generator=g, device="cuda")
    return x.clamp_(0, 1), which % DIMS[-1]


def forward(ctx, x, stored, biases):
    """Every layer's output; the last one's are the answers."""
    h = [x]
    for i, (w, b) in enumerate(zip(stored, biases)):
        h.append(ctx.mx_linear(h[-1], w, bias=b, relu=i + 1 < len(stored)))
    return h


def train(ctx, steps, batch=256, lr=0.1, momentum=0.9):
    g = torch.Generator("cuda").manual_seed(0)
    weights = [torch.randn(n, k, generator=g, device="cuda") * (2.0 / k) ** 0.5 for k, n in zip(DIMS, DIMS[1:])]
    biases = [torch.zeros(n, device="cuda") for n in DIMS[1:]]
    moved = [torch.zeros_like(w) for w in weights]
    losses = []
    for step in range(steps):
        x, label = data(g, batch)
        stored = [ctx.mx_quantize(w) for w in weights]
        h = forward(ctx, x, stored, biases)
        p = torch.softmax(h[-1], 1)
        losses.append(-p.gather(1, label[:, None]).clamp_min(1e-30).log().mean())
        dy = p.scatter_add(1, label[:, None], torch.full((batch, 1), -1.0, device="cuda")) / batch
        rate = lr * (1 - step / steps)
        for i in reversed(range(len(weights))):
            last = i + 1 == len(weights)
            dy_in, dw, db = ctx.mx_linear_grad(dy, h[i], stored[i], y=None if last else h[i + 1], need=(i > 0, True, True))
            moved[i].mul_(momentum).add_(dw)
            ctx.orthogonalize(moved[i], gain=-rate, base=weights[i], out=weights[i])
            biases[i].sub_(db, alpha=rate)
            dy = dy_in
    return [ctx.mx_quantize(w) for w in weights], biases, torch.stack(losses).tolist()


def network(ctx, stored, biases):
    """The stored network as the verifier takes it."""
    nodes = []
    for i, (w, b) in enumerate(zip(stored, biases)):
        nodes.append(Node("dense", 2 * i - 1, W=ctx.mx_dequantize(w).cpu().numpy(), b=b.cpu().numpy()))
        if i + 1 < len(stored):
            nodes.append(Node("relu", 2 * i))
    return Net((DIMS[0],), nodes)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--eps", type=float, default=0.01)
    ap.add_argument("--inputs", type=int, default=64)
    a = ap.parse_args(argv)
    ctx = Ctx(0)
    stored, biases, losses = train(ctx, a.steps)
    x, label = data(torch.Generator("cuda").manual_seed(2), a.inputs)
    answers = forward(ctx, x, stored, biases)[-1]
    # the same in 4 bits throughout: each layer's input quantised too
    h = x
    for i, (w, b) in enumerate(zip(stored, biases)):
        h = ctx.mx_product(ctx.mx_quantize(h), w, bias=b, relu=i + 1 < len(stored))
    # margins of the answered class over the others
    ctx.load_net(network(ctx, stored, biases))
    top = answers.argmax(1)
    eye = torch.eye(DIMS[-1], device="cuda")
    others = torch.stack([torch.tensor([j for j in range(DIMS[-1]) if j != c], device="cuda") for c in top.tolist()])
    spec = (eye[top][:, None] - eye[others]).contiguous()
    lb, ub = ctx.crown_bounds(x, a.eps, spec)
    margins = (spec @ answers[:, :, None])[:, :, 0]
    # an attack beside the bounds: one signed step against the smallest margin, through the stored weights
    worst = margins.argmin(1)
    dy = -spec[torch.arange(a.inputs, device="cuda"), worst].contiguous()
    hs = forward(ctx, x, stored, biases)
    for i in reversed(range(len(stored))):
        dy = ctx.mx_linear_grad(dy, None, stored[i], y=hs[i + 1] if i + 1 < len(stored) else None, need=(True, False, False))[0]
    moved = forward(ctx, (x + a.eps * dy.sign()).clamp(0, 1), stored, biases)[-1]
    attacked = (spec @ moved[:, :, None])[:, :, 0]
    slack = 1e-4 * (1 + margins.abs().max())
    result = {
        "loss": (losses[0], losses[-1]),
        "accuracy": float((top == label).float().mean()),
        "accuracy in 4 bits throughout": float((h.argmax(1) == label).float().mean()),
        "verified": float((lb.amin(1) > 0).float().mean()),
        "attacked": float((attacked.amin(1) <= 0).float().mean()),
        "bounds hold": bool(((lb <= margins + slack) & (margins <= ub + slack) & (lb <= attacked + slack) &
                             (attacked <= ub + slack)).all()),
        "spectral norms": [float(np.linalg.norm(n.W, 2)) for n in network(ctx, stored, biases).nodes if n.op == "dense"],
    }
    for k, v in result.items():
        print(f"{k}: {v}", flush=True)
    return result


if __name__ == "__main__":
    main()
