"""The launches of calls on float layers, dropout and the loss, without a GPU: legal sizes up to the largest give grids that the device takes, tiles and parts that
cover the results and the contraction, and buffers inside the workspace and apart from each other (tests/host/dense_launches.cpp checks each)."""
import random

from tests import dense_launches as dl
from tests.test_dense_tiles_gpu import CALLS
from tests.test_loss_gpu import SIZES
from tests.test_loss_masked_classes_gpu import PLANS


def test_legal_sizes():
    assert "all checks passed" in dl.run("random", "400000")


def test_legal_sizes_under_asan_and_ubsan():
    """The plans' and workspaces' arithmetic under the sanitizers."""
    assert "all checks passed" in dl.run("random", "60000", sanitize=True)


def test_results_of_more_tiles_than_a_launch_counts():
    """float32 rows onto bf16 results of more than 2^36, 137 GB: tiles of more than 2^32 threads, in two launches."""
    calls = [("linear", 10443640, 64, n, 0, 0, 1, 0, 1, 0, 1) for n in (6600, 6500)]
    products = [[g for name, g, _ in each if name.startswith("k_nt<")] for each in dl.launches(calls)]
    assert [len(p) for p in products] == [2, 1], products
    assert products[0][0][0] + products[0][1][0] == -(-10443640 // 64) * -(-6600 // 64)


def test_calls_on_the_gpu_take_what_random_ones_do():
    rng = random.Random(4)
    reached = set().union(*(dl.covered(each) for each in dl.launches([dl.any_call(rng)[0] for _ in range(20000)])))
    run = set().union(*(dl.covered(each) for each in dl.launches(CALLS)))
    assert len(reached) > 200 and reached <= run, sorted(reached - run, key=str)


def test_losses_on_the_gpu_take_every_kernel():
    rng = random.Random(5)

    def reached(calls):
        return {kernel for each in dl.launches(calls) for kernel, _, _ in each}

    def size(hi):
        return max(1, round(hi ** rng.random()))
    anyone = reached([("loss", size(20000), size(2 ** 20), rng.randrange(2), 0, rng.randrange(2)) for _ in range(5000)])
    assert len(anyone) > 40
    assert anyone <= reached([("loss", m, n, t, 0, other) for m, n in SIZES + PLANS for t in (0, 1) for other in (0, 1)])
    same = {k for k in anyone if "Row<true,false>" not in k and "Row<false,true>" not in k}
    assert same <= reached([("loss", m, n, t, 0, 0) for m, n in PLANS for t in (0, 1)]) | {"k_loss_count"}
