"""The tiles that calls on layers take, from tests/host/product_plan.cpp (nt.h's own choice, compiled for the host)."""
import functools
import os
import shutil
import subprocess
import tempfile

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_09377_amd", "csrc")


@functools.lru_cache(maxsize=None)
def _program():
    hipcc = next((c for c in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc") if c and os.path.exists(c)), None)
    if hipcc is None:
        pytest.skip("hipcc not found")
    d = tempfile.TemporaryDirectory()
    exe = os.path.join(d.name, "plan")
    subprocess.run([hipcc, "-O1", "-std=c++17", "--offload-host-only", "-I", CSRC, "-x", "hip",
                    os.path.join(HERE, "host", "product_plan.cpp"), "-o", exe], check=True, capture_output=True)
    return d, exe


def shapes():
    """{class: number of shapes}"""
    out = subprocess.run([_program()[1], "shapes"], check=True, capture_output=True, text=True).stdout
    return {l.split()[0]: int(l.split()[1]) for l in out.splitlines()}


def plans(products):
    """For each (class, rows, columns, chunks, batch, tri, bytes of an output, may be divided): (parts, [(shape, stages of the contraction,
    stages in LDS) of each launch])."""
    text = "".join(" ".join(str(v) for v in p) + "\n" for p in products)
    out = subprocess.run([_program()[1]], input=text, check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(out) == len(products)
    return [(int(l.split()[0]), [tuple(int(v) for v in t.split(":")) for t in l.split()[1:]]) for l in out]


def blocks(n, b):
    return -(-n // b)


def product(m, k, n, out_bytes=4):
    return [("4x4", m, n, blocks(k, 128), 1, 0, out_bytes, 1)] if m > 16 else []


def linear(m, k, n, bf16):
    if m <= (8 if bf16 else 5):
        return []
    return [("1x4" if bf16 else "3x4", m, n, 4 * blocks(k, 128), 1, 0, 2 if bf16 else 4, 1)]


def grad_dx(m, k, n, bf16):
    return [("1x1" if bf16 else "3x1", m, k, blocks(n, 32), 1, 0, 2 if bf16 else 4, 1)]


def grad_dw(m, k, n, bf16):
    return [("1x1" if bf16 else "3x3", n, k, blocks(m, 32), 1, 0, 4, 1)]


def orthogonalize(m, n, bf16, count=1, steps=5, base=False):
    m, n = sorted((blocks(m, 32) * 32, blocks(n, 32) * 32))
    out = []
    for i in range(steps):
        first, last = bf16 and i == 0, i + 1 == steps
        out += [("1x1" if first else "3x3", m, m, n // 32, count, 1, 12, 0), ("3x3", m, m, m // 32, count, 1, 12, 0),
                ("3x1" if first else "3x3", m, n, m // 32, count, 0, (8 if base else 4) if last else 12, 0)]
    return out
