"""What calls on float layers launch, from tests/host/dense_launches.cpp (the entry points' own host code, launches recorded)."""
import functools
import os
import re
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


def covered(each):
    """What of the kernels these launches run: every kernel with its template's arguments and whatever it was told to do beside its work, and of a product's tiles
    also "loop" (stages enough for the steady loop), "ragged" (the contraction ends inside a stage), "short" (fewer stages than LDS holds), "empty" (a part
    without a share) and "rest" (tiles that another shape left)."""
    seen = set()
    for kernel, _, notes in each:
        tiles = re.findall(r"NtTile<([\d,]+)>", kernel)
        products = re.findall(r"chunks=(\d+) z=(\d+) cols=(\d+) first=(\d+)", " ".join(notes))
        name = re.sub(r",EpiOut<.*?>>", ">", kernel)
        told = tuple(n for n in notes if "=" not in n and n != "empty")
        seen.add((name, *told))
        if name.startswith("k_dense_few") and "along" in told:
            tiles = ["0,2,2,2,4,1,3,3,1,2"]   # FewTile
        for tile, (chunks, z, cols, first) in zip(tiles, products):
            kind, *_, ks, stages = (int(v) for v in tile.split(","))
            chunks, z, cols = int(chunks), int(z), int(cols)
            at = (name, tile)
            counts = [-(-(min(chunks, a + z) - a) // ks) for a in range(0, chunks, z)]
            rows = kind >= 3
            ragged = cols % (32 * ks) != 0 if rows else chunks % ks != 0
            last = counts[-1] - (1 if ragged else 0)
            if any(c > stages + (1 if rows else 2) for c in counts[:-1] + [last if rows else counts[-1]]):
                seen.add((*at, "loop"))
                if ragged:
                    seen.add((*at, "loop", "ragged"))
            if ragged:
                seen.add((*at, "ragged"))
            if min(counts) < stages:
                seen.add((*at, "short"))
            if "empty" in notes:
                seen.add((*at, "empty"))
            if int(first) > 0:
                seen.add((*at, "rest"))
    return seen


def any_call(rng, largest=8192):
    """A random call of linear or grad as the program reads it, whose work is at most that of 4096 x 8192 x 4096, and that work."""
    def size(hi):
        return max(1, min(hi, round(hi ** rng.random())))
    while True:
        m, k, n, bf16 = size(largest), size(rng.choice((largest, 65536))), size(rng.choice((largest, 65536))), rng.randrange(2)
        if rng.random() < 0.5:
            k, n = -(-k // 8) * 8, -(-n // 8) * 8
        if m * k * n > 2 ** 37 or max(m * k, n * k, m * n) > 2 ** 27:
            continue
        pitch, act, drop, other = rng.choice((0, 8, 3)), rng.randrange(2), rng.randrange(2), rng.randrange(2)
        if rng.random() < 0.5:
            return ("linear", m, k, n, bf16, pitch, act, drop, rng.randrange(2), rng.randrange(2), other), m * k * n
        return ("grad", m, k, n, bf16, pitch, act, drop, rng.choice((7, 7, 7, 1, 2, 5, 6)), other), 2 * m * k * n
