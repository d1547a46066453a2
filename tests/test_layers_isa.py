"""The loads into LDS of layers.hip and orthogonalize.hip set M0 in inline assembly and leave it changed, which is
correct only while nothing else uses M0.  Compile both for gfx950 to assembly (code built here) and check, in
every function that issues such a load, that M0 is written by the load sequence alone (M0 write, one wait state, the
load) and read by nothing else; that no kernel of products spills registers in its loop; and that the loop's one wait
for loads leaves the later stages' in flight where there are more than two stages."""
import functools
import os
import re
import shutil
import subprocess
import tempfile

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_09377_amd", "csrc")


def _hipcc():
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    pytest.skip("hipcc not found")


@functools.lru_cache(maxsize=None)
def _functions(src):
    """{name: body lines} of the kernels of a source."""
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "k.s")
        subprocess.run([_hipcc(), "-O3", "-std=c++17", "--offload-arch=gfx950", "--offload-device-only", "-S", "-Xclang",
                        "-target-feature", "-Xclang", "-packed-fp32-ops", "-x", "hip", os.path.join(CSRC, src), "-o", out],
                       check=True, capture_output=True)
        asm = open(out).read()
    found, name, body = {}, None, []
    for line in asm.splitlines():
        m = re.match(r"^(_Z\S+):", line)
        if m:
            name, body = m.group(1), []
        elif name is not None:
            if line.startswith(".Lfunc_end"):
                found[name] = body
                name = None
            else:
                body.append(line.strip())
    return found


SOURCES = ["layers.hip", "orthogonalize.hip"]


@pytest.mark.parametrize("src", SOURCES)
def test_m0_only_feeds_the_lds_loads(src):
    checked = 0
    for name, body in _functions(src).items():
        code = [l for l in body if l and not l.startswith((";", ".")) and not l.endswith(":")]
        if not any(l.startswith("global_load_lds") for l in code):
            continue
        checked += 1
        for i, l in enumerate(code):
            if "m0" not in l.split(";")[0]:
                continue
            assert re.match(r"s_mov_b32 m0, s\d+$", l), f"{name}: other use of M0: {l}"
            assert code[i + 1] == "s_nop 0" and re.match(r"global_load_lds_dword(x4)? ", code[i + 2]), name
    assert checked >= 20


def _loops(body):
    """Lines between a label and a later branch back to it, innermost loops with matrix instructions."""
    at = {l.split(":")[0]: i for i, l in enumerate(body) if re.match(r"^\.LBB\w+:", l)}
    spans = []
    for i, l in enumerate(body):
        m = re.match(r"s_c?branch\w* (\.LBB\w+)", l)
        if m and at.get(m.group(1), i) < i:
            spans.append((at[m.group(1)], i))
    spans = [s for s in spans if any(x.startswith("v_mfma") for x in body[s[0]:s[1]])]
    return [s for s in spans if not any(t != s and s[0] <= t[0] and t[1] <= s[1] for t in spans)]


@pytest.mark.parametrize("src", SOURCES)
def test_steady_loops_keep_loads_in_flight(src):
    checked = 0
    for name, body in _functions(src).items():
        m = re.search(r"k_ntINS_6NtTileILi(\d)ELi(\d+)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)E", name)
        if not m:
            continue
        stages = int(m.group(10))
        # the steady loop: the one whose matrix instructions are in one block (no other label inside)
        steady = [body[a:b] for a, b in _loops(body) if not any(re.match(r"^\.LBB\w+:", x) for x in body[a + 1:b])]
        assert len(steady) == 1, (name, len(steady))
        loop = steady[0]
        checked += 1
        assert not any(x.startswith(("scratch_", "buffer_store_dword", "buffer_load_dword ")) for x in loop), name
        waits = [int(v) for x in loop for v in re.findall(r"^s_waitcnt.*vmcnt\((\d+)\)", x)]
        assert waits and (stages == 2 or min(waits) > 0), (name, waits)
    assert checked >= 20
