"""The loads into LDS of dense.hip set M0 in inline assembly and leave it changed, which is correct only while nothing else uses
M0; a register spilled in a loop of products would wait for the loads in flight with every use.  Compile the source for gfx950 to assembly (code
built here) and check both, and that the loops' waits leave the later stages' loads in flight where there are more than two stages."""
import re

import pytest

from tests.test_layers_isa import _functions, _loops

SRC = "dense.hip"
TILE = r"NtTileILi(\d)ELi(\d+)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)E"


def _code(body):
    return [l for l in body if l and not l.startswith((";", ".")) and not l.endswith(":")]


def test_m0_only_feeds_the_lds_loads():
    checked = 0
    for name, body in _functions(SRC).items():
        code = _code(body)
        if not any(l.startswith("global_load_lds") for l in code):
            continue
        checked += 1
        for i, l in enumerate(code):
            if "m0" not in l.split(";")[0]:
                continue
            assert re.match(r"s_mov_b32 m0, (s\d+|vcc_lo|vcc_hi)$", l), f"{name}: other use of M0: {l}"
            assert code[i + 1] == "s_nop 0" and re.match(r"global_load_lds_dword(x4)? ", code[i + 2]), name
    assert checked >= 30


def test_product_loops_spill_nothing_and_keep_loads_in_flight():
    checked = 0
    for name, body in _functions(SRC).items():
        m = re.search(r"k_ntINS_6" + TILE, name)
        if not m:
            continue
        stages = int(m.group(10))
        steady = [body[a:b] for a, b in _loops(body) if not any(re.match(r"^\.LBB\w+:", x) for x in body[a + 1:b])]
        loading = [l for l in steady if any(x.startswith("global_load_lds") for x in l)]
        assert len(loading) == 1, (name, len(loading))
        for loop in steady:
            assert not any(x.startswith(("scratch_", "buffer_store_dword", "buffer_load_dword ")) for x in loop), name
        waits = [int(v) for x in loading[0] for v in re.findall(r"^s_waitcnt.*vmcnt\((\d+)\)", x)]
        assert waits and (stages == 2 or min(waits) > 0), (name, waits)
        checked += 1
    assert checked >= 30


@pytest.mark.parametrize("src", ["dense.hip", "dropout.hip", "loss.hip"])
def test_no_packed_float_instructions(src):
    for name, body in _functions(src).items():
        assert not any(re.match(r"v_pk_(add|mul|fma)_f32", l) for l in body), name
