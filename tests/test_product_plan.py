"""Every tile shape that is built is one that some call takes, and one that the tests on the GPU run."""
import random

from tests import product_plan as pp
from tests.test_layers_tiles_gpu import CALLS


def test_every_shape_is_taken_by_some_size():
    rng = random.Random(3)
    calls = [p for _ in range(12000) for p in pp.products_of(pp.any_call(rng)[0])]
    taken = {f[1:3] for f in pp.covered(calls) if isinstance(f[2], int)}
    built = {(c, i) for c, n in pp.shapes().items() for i in range(n)}
    assert taken == built, sorted(built - taken)


def test_calls_on_the_gpu_take_what_random_ones_do():
    rng = random.Random(4)
    reached = pp.covered([p for _ in range(20000) for p in pp.products_of(pp.any_call(rng)[0])])
    run = pp.covered([p for c in CALLS for p in pp.products_of(c)])
    assert reached <= run, sorted(reached - run, key=str)
    assert ("gram", "1x1", "rest") in run and ("gram", "3x3", "rest") in run   # (triangles in two shapes)
