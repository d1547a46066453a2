"""The launches of calls on float layers, dropout and the loss, without a GPU: legal sizes up to the largest give grids that the device takes, tiles and parts that
cover the results and the contraction, and buffers inside the workspace and apart from each other (tests/host/dense_launches.cpp checks each)."""
from tests import dense_launches as dl


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
