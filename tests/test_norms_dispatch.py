"""Which kernels the calls of the layer norm and of the weights' update take, as a program sees it from the host: the device
runtime's launch call is replaced in a client program (tests/norms_client.cpp).  No GPU, and no pointer is followed.  What the GPU
tests run is listed there by size; here every compiled kernel is found among what those sizes take."""
import re
import shutil
import subprocess
from pathlib import Path

import pytest

import test_gpu_norms as G
import test_gpu_update as A
from test_products8_dispatch import compiled, sizes

ROOT = Path(__file__).resolve().parent.parent
LIB = ROOT / "paper_2206_01299_amd" / "libaqsgd.so"
TYPES = {"f32": 0, "f16": 1, "bf16": 2}
MOST_LANES = 2 ** 32


@pytest.fixture(scope="module")
def client(tmp_path_factory):
    gxx = shutil.which("g++")
    assert gxx, "g++ is part of the image"
    exe = tmp_path_factory.mktemp("norms") / "client"
    subprocess.run([gxx, "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{ROOT / 'include'}",
                    str(ROOT / "tests" / "norms_client.cpp"), str(LIB), f"-Wl,-rpath,{LIB.parent}",
                    "-Wl,-rpath,/opt/rocm/lib", "-ldl", "-o", str(exe)], check=True)

    def run(*calls):
        """For each call its launches, as (workgroups, lanes, kernel with its constants)."""
        out = subprocess.run([str(exe), *(",".join(str(x) for x in c) for c in calls)], check=True, capture_output=True, text=True)
        made, launches = [], []
        for line in out.stdout.splitlines():
            word = line.split(maxsplit=6)
            if word[0] == "call":
                assert int(word[1]) == 0, calls[len(made)]
                made.append(launches)
                launches = []
            else:
                kernel = re.search(r"(\w+(?:<[^>]*>)?)\(", word[6])
                launches.append((int(word[1]) * int(word[2]) * int(word[3]), int(word[5]), kernel.group(1) if kernel else word[6]))
                assert launches[-1][0] * launches[-1][1] < MOST_LANES
        assert len(made) == len(calls)
        return made

    return run


def taken(made):
    return {k for launches in made for _, _, k in launches}


def by_pieces(pairs, name):
    """Rows and columns of a type's sizes given in pieces, whole ones and others."""
    return [(rows, pieces * G.PIECES[name] - less) for pieces, rows in pairs for less in (0, 1)]


def test_every_kernel_of_the_norm_runs_in_the_gpu_tests(client):
    rows = sizes(G.test_layernorm, "rows,cols")
    made = taken(client(*(("n", t, 0, r, c) for n, t in TYPES.items() for r, c in rows + by_pieces(G.NORMS, n))))
    for name in ("layernorm_kernel", "layernorm_wide_kernel", "layernorm_narrow_kernel"):
        assert compiled(name) and compiled(name) <= made, compiled(name) - made


def test_every_kernel_of_the_gradient_runs_in_the_gpu_tests(client):
    rows = sizes(G.test_layernorm_grad, "rows,cols") + sizes(G.test_layernorm_grad_by_rows, "rows,cols")
    made = taken(client(*(("g", t, which, r, c) for n, t in TYPES.items() for r, c in rows + by_pieces(G.GRADS, n) for which in (0, 1, 3))))
    for name in ("layernorm_grad_kernel", "layernorm_grad_few_kernel", "layernorm_grad_wide_kernel", "layernorm_grad_narrow_kernel",
                 "layernorm_grad_narrow_columns_kernel"):
        assert compiled(name) and compiled(name) <= made, compiled(name) - made


def test_every_kernel_of_the_update_runs_in_the_gpu_tests(client):
    kinds = [(TYPES[d], TYPES[g] + (0 if bits == 32 else 4) + 8 * rounding) for d, g in A.TYPES for bits, rounding in A.KINDS]
    made = taken(client(*(("a", d, kind, n, 1) for d, kind in kinds for n in A.SIZES)))
    assert compiled("adamw_kernel") and compiled("adamw_kernel") <= made, compiled("adamw_kernel") - made


def test_launches_of_many_tensors(client):
    """64 tensors to a launch; a norm has one launch more, a small one of up to 64 tensors just one; none for tensors of no elements."""
    made = client(("a", 0, 0, 100, 64), ("a", 0, 0, 100, 65), ("a", 0, 0, 100, 200), ("a", 0, 0, 0, 200), ("r", 1, 0, 513, 64), ("r", 1, 0, 100, 65),
                  ("r", 1, 0, 0, 3), ("a", 0, 0, 1 << 34, 3), ("r", 1, 0, 512, 64), ("r", 0, 0, 16384, 1), ("r", 0, 0, 16385, 1))
    assert [len(m) for m in made] == [1, 2, 4, 0, 2, 3, 1, 3, 1, 1, 2]


def test_launches_of_the_gradient(client):
    """One launch for few rows, two where dx takes dy's place, two for many rows, one without sums."""
    made = client(("g", 1, 1, 1024, 1600), ("g", 1, 3, 1024, 1600), ("g", 1, 1, 1409, 1600), ("g", 1, 3, 1409, 1600), ("g", 1, 0, 100000, 1600),
                  ("g", 1, 2, 100000, 1600), ("g", 1, 1, 0, 1600), ("g", 1, 1, 5000, 16384), ("g", 1, 1, 100, 3), ("g", 1, 1, 100, 70001),
                  ("g", 1, 0, 100, 70001))
    assert [len(m) for m in made] == [1, 2, 2, 2, 1, 1, 1, 1, 2, 2, 1]


def test_the_largest_calls_stay_within_a_grid(client):
    """2^30 rows and 2^24 columns, where the launches are asserted to be below 2^32 lanes."""
    client(*((what, t, 1, r, c) for what in "ng" for t in TYPES.values() for r, c in ((1 << 30, 1), (1 << 30, 8), (1 << 30, 3000 + 8), (1 << 30, 16384),
                                                                                      (1 << 30, 70001), (1, 1 << 24), (1 << 30, 1 << 24))))
