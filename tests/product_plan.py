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
    """For each (kind, (class, rows, columns, chunks, batch, tri, bytes of an output, may be divided)): the number of parts, and (shape, stages
    of the contraction, stages in LDS) of each launch."""
    text = "".join(" ".join(str(v) for v in p) + "\n" for _, p in products)
    out = subprocess.run([_program()[1]], input=text, check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(out) == len(products)
    return [(int(l.split()[0]), [tuple(int(v) for v in t.split(":")) for t in l.split()[1:]]) for l in out]


def covered(products):
    """What of the kernels of products these run: (kind, class, shape) of a launch, with "loop" where it has stages enough for the steady
    loop, (kind, class, "parts") of a divided contraction and (kind, class, "rest") of whole rounds and a rest in another shape."""
    seen = set()
    for (kind, p), (parts, launches) in zip(products, plans(products)):
        if parts > 1:
            seen.add((kind, p[0], "parts"))
        if len(launches) > 1:
            seen.add((kind, p[0], "rest"))
        for shape, stages, in_lds in launches:
            if parts == 1:
                seen.add((kind, p[0], shape))
                if stages > in_lds + 2:
                    seen.add((kind, p[0], shape, "loop"))
    return seen


def blocks(n, b):
    return -(-n // b)


def product(m, k, n, bf16=False):
    return [("product", ("4x4", m, n, blocks(k, 128), 1, 0, 2 if bf16 else 4, 1))] if m > 16 else []


def linear(m, k, n, bf16):
    if m <= (8 if bf16 else 5):
        return []
    return [("linear", ("1x4" if bf16 else "3x4", m, n, 4 * blocks(k, 128), 1, 0, 2 if bf16 else 4, 1))]


def grad(m, k, n, bf16):
    return [("gradient", ("1x1" if bf16 else "3x1", m, k, blocks(n, 32), 1, 0, 2 if bf16 else 4, 1)),
            ("gradient", ("1x1" if bf16 else "3x3", n, k, blocks(m, 32), 1, 0, 4, 1))]


def orthogonalize(m, n, bf16, count, steps, base=False, out_bf16=False):
    m, n = sorted((blocks(m, 32) * 32, blocks(n, 32) * 32))
    out = []
    for i in range(steps):
        first, last = bf16 and i == 0, i + 1 == steps
        out += [("gram", ("1x1" if first else "3x3", m, m, n // 32, count, 1, 12, 0)),
                ("polynomial", ("3x3", m, m, m // 32, count, 1, 12, 0)),
                ("result" if last else "update",
                 ("3x1" if first else "3x3", m, n, m // 32, count, 0, (8 if base else 4) if last else 12, 0))]
    return out


CALLS = {"product": product, "linear": linear, "grad": grad, "orthogonalize": orthogonalize}


def products_of(call):
    """("linear", m, k, n, bf16) and so on, as its products."""
    return CALLS[call[0]](*call[1:])


def any_call(rng, largest=8192):
    """A random call whose work is at most that of a product of 4096 x 8192 x 4096."""
    def size(lo, hi):
        return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))
    while True:
        kind, bf16 = rng.choice(list(CALLS)), rng.random() < 0.5
        m, k, n = size(6, largest), size(32, largest), size(16, largest)
        if kind == "orthogonalize":
            call = (kind, m, n, bf16, rng.choice((1, 1, 2, 3)), rng.choice((1, 2, 3)), rng.random() < 0.3)
            work = call[4] * call[5] * 4 * min(m, n) ** 2 * max(m, n)
        else:
            call = (kind, m, k, n, bf16)
            work = m * k * n
        if work <= 2 ** 37:
            return call, work
