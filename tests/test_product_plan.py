"""Every tile shape that is built is one that some call takes."""
import random

from tests import product_plan as pp


def test_every_shape_is_taken_by_some_size():
    rng = random.Random(3)

    def size(lo, hi):
        return max(lo, round(lo * (hi / lo) ** rng.random()))
    calls = []
    for _ in range(4000):
        m, k, n, bf16 = size(17, 16384), size(32, 16384), size(16, 16384), rng.random() < 0.5
        calls += pp.product(m, k, n) + pp.linear(m, k, n, bf16) + pp.grad_dx(m, k, n, bf16) + pp.grad_dw(m, k, n, bf16)
        calls += pp.orthogonalize(m, n, bf16, rng.choice((1, 1, 3)), steps=2)
    taken = {(p[0], s[0]) for p, (_, launches) in zip(calls, pp.plans(calls)) for s in launches}
    built = {(c, i) for c, n in pp.shapes().items() for i in range(n)}
    assert taken == built, sorted(built - taken)
