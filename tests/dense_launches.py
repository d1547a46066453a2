"""What calls on float layers launch, from tests/host/dense_launches.cpp (the entry points' own host code, launches recorded)."""
import functools
import os
import shutil
import subprocess
import tempfile

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_09377_amd", "csrc")
SANITIZE = [f for s in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all") for f in ("-Xarch_host", s)]


@functools.lru_cache(maxsize=None)
def program(sanitize=False):
    """(what keeps it, path)"""
    hipcc = next((c for c in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc") if c and os.path.exists(c)), None)
    if hipcc is None:
        pytest.skip("hipcc not found")
    d = tempfile.TemporaryDirectory()
    exe = os.path.join(d.name, "launches")
    b = subprocess.run([hipcc, "-O1", "-g", "-std=c++17", "--offload-host-only", "-fuse-cuid=none", "-rdynamic", "-I", CSRC, *(SANITIZE if sanitize else ()),
                        "-x", "hip", os.path.join(HERE, "host", "dense_launches.cpp"), "-o", exe, "-ldl"], capture_output=True, text=True)
    assert b.returncode == 0, b.stderr[-3000:]
    return d, exe


def run(*args, text="", sanitize=False):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([program(sanitize)[1], *args], input=text, capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-3000:])
    return r.stdout


def launches(calls):
    """For each call (kind and numbers, as the program reads them) its launches: (kernel, (x, y) of its grid, notes)."""
    out = run(text="".join(" ".join(str(v) for v in c) + "\n" for c in calls)).splitlines()
    assert len(out) == len(calls)
    each = []
    for line in out:
        status, *rest = line.split("  ")
        assert status == "0", line
        each.append([(f[0], tuple(int(v) for v in f[1].split("x")), f[2:]) for f in (l.split(" ") for l in rest)])
    return each
