"""The few-row kernels of dense.hip hold their loops' operands and sums in registers: a spilled one in a loop would wait for the loads in flight with every use.
Compile the source for gfx950 to assembly (code built here) and check that no loop of products of k_dense_rows or k_dense_few reaches scratch memory."""
import re

from tests.test_layers_isa import _functions, _loops


def test_loops_of_few_rows_reach_no_scratch_memory():
    checked = loops = 0
    for name, body in _functions("dense.hip").items():
        if not re.search(r"12k_dense_rowsI|11k_dense_fewI", name):
            continue
        checked += 1
        for a, b in _loops(body):
            loops += 1
            assert not any(x.startswith(("scratch_", "buffer_store_dword", "buffer_load_dword ")) for x in body[a:b]), name
    assert checked == 15 and loops >= checked, (checked, loops)
