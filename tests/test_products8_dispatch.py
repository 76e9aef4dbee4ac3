"""Which kernels the 8-bit operators' calls take, as a program sees it from the host: the device runtime's launch call is
replaced in a client program (tests/products8_client.cpp).  No GPU, and no pointer is followed.  What the GPU tests run is
listed there by size; here every compiled kernel is found among what those sizes take."""
import re
import shutil
import subprocess
from pathlib import Path

import pytest

import test_gpu_products8 as T
import test_gpu_products8_columns as C
import test_gpu_products8_pipeline as L

ROOT = Path(__file__).resolve().parent.parent
LIB = ROOT / "paper_2206_01299_amd" / "libaqsgd.so"
TYPES = {"f32": 0, "f16": 1, "bf16": 2}


@pytest.fixture(scope="module")
def client(tmp_path_factory):
    gxx = shutil.which("g++")
    assert gxx, "g++ is part of the image"
    exe = tmp_path_factory.mktemp("dispatch8") / "client"
    subprocess.run([gxx, "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{ROOT / 'include'}",
                    str(ROOT / "tests" / "products8_client.cpp"), str(LIB), f"-Wl,-rpath,{LIB.parent}",
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
                kernel = re.search(r"(\w+<[^>]*>)\(", word[6])
                launches.append((int(word[1]) * int(word[2]), int(word[5]), kernel.group(1) if kernel else word[6]))
        assert len(made) == len(calls)
        return made

    return run


def compiled(name):
    """The library's kernels of this name, with their constants."""
    nm = subprocess.run(["nm", "-D", "-C", "--defined-only", str(LIB)], check=True, capture_output=True, text=True).stdout
    return set(re.findall(rf"\b{name}<[^>]*>(?=\()", nm))


def sizes(test, names):
    """What a test is run for."""
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == names)


def tile(kernel):
    """(columns of a tile, of the narrower ones behind it) of a large product's kernel."""
    _, _, _, tn, _, wn, narrow = (int(x) for x in re.search(r"product_tile_kernel<(.*)>", kernel).group(1).split(", "))
    return 16 * tn * wn, 16 * narrow * wn


@pytest.mark.parametrize("what,kinds,loops", [("m", (0, 1), L.LOOPS), ("f", (0,), L.LOOPS), ("f", (1,), L.GATED_LOOPS)])
def test_the_sizes_of_several_steps_take_the_tiles_they_are_listed_for(client, what, kinds, loops):
    for cols, narrow, m, n, k in loops:
        steps = -(-(-(-k // 64)) // 2)
        assert steps >= 4
        for kind in kinds:
            for dtype in TYPES.values():
                launches, = client((what, dtype, kind, m, n, k))
                assert len(launches) == 1 and tile(launches[0][2]) == (cols, narrow), (what, kind, m, n, k, launches)
    for each in {loop[:2] for loop in loops}:
        halves = {-(-loop[4] // 64) for loop in loops if loop[:2] == each}
        assert {h % 2 for h in halves} == {0, 1} and {-(-h // 2) % 2 for h in halves} == {0, 1}, each


def test_every_product_kernel_is_taken_by_a_size_that_the_gpu_tests_run(client):
    """By every type: the choice goes by sizes alone."""
    plain = T.PRODUCTS + T.TILES + sizes(T.test_long_sums_in_slices, "m,n,k") + [loop[2:] for loop in L.LOOPS]
    message = sizes(T.test_matmul8_of_a_message, "m,n,k") + T.TILES + [loop[2:] for loop in L.LOOPS] + \
        sizes(T.test_long_sums_in_slices, "m,n,k")
    act = sizes(T.test_ffn8, "m,f,k") + T.TILES + [loop[2:] for loop in L.LOOPS]
    gated = sizes(T.test_ffn8, "m,f,k") + T.GATED + [loop[2:] for loop in L.GATED_LOOPS]
    calls = [(what, dtype, kind, *size) for dtype in TYPES.values()
             for what, kind, of in (("m", 0, plain), ("m", 1, message), ("f", 0, act), ("f", 1, gated)) for size in of]
    taken = {kernel for launches in client(*calls) for _, _, kernel in launches}
    for name in ("product_tile_kernel", "product_split_kernel", "product_join_kernel"):
        here = compiled(name)
        assert len(here) > 1
        missing = here - taken
        assert not missing, f"{len(missing)} of {len(here)} without a size: {sorted(missing)[:5]}"


ROWS, COLS, SUMS, DRAWS = 1, 2, 4, 8


def test_the_wide_matrices_take_whole_tiles_of_128_rows(client):
    """Several spans of columns, one tile and two to a workgroup."""
    for (rows, cols), each in zip(C.WIDE, (1, 2)):
        for which in (ROWS | COLS | SUMS, COLS | SUMS, ROWS | COLS | DRAWS):
            launches, = client(("q", 0, which, rows, cols, cols))
            assert len(launches) == 2 and re.match(rf"quant8_tiles_kernel<0, {which >> 3}, {'true' if which & ROWS else 'false'}, 2>", launches[1][2])
            assert launches[1][0] == -(-cols // 128) * -(-rows // (128 * each)) and cols > 256


def test_every_kernel_of_the_quantiser_is_taken_by_a_size_that_the_gpu_tests_run(client):
    runs = {which: T.SIZES + sizes(T.test_quant8_of_many_rows, "rows,cols") for which in (ROWS | COLS | SUMS, ROWS, COLS)}
    runs[ROWS | COLS | SUMS] = runs[ROWS | COLS | SUMS] + C.WIDE + C.SUMS
    runs[COLS | SUMS] = runs[ROWS | SUMS] = runs[SUMS] = C.SUMS
    runs[ROWS | COLS] = C.WIDE
    runs[ROWS | COLS | DRAWS] = sizes(T.test_quant8_stochastic, "rows,cols") + C.WIDE
    runs[COLS | DRAWS] = [(300, 150)] + [s for s in sizes(T.test_quant8_of_many_rows, "rows,cols") if s[1] == 3]
    runs[ROWS | DRAWS] = [(5, cols) for cols in (40, 200, 900, 1500, 5001, 12000, 20000)]
    calls = [("q", dtype, which, r, c, c) for dtype in TYPES.values() for which, of in runs.items() for r, c in of]
    taken = {kernel for launches in client(*calls) for _, _, kernel in launches}
    for name in ("quant8_rows_kernel", "quant8_short_kernel", "quant8_maxima_kernel", "quant8_tiles_kernel"):
        here = compiled(name)
        assert len(here) > 1
        missing = here - taken
        assert not missing, f"{len(missing)} of {len(here)} without a size: {sorted(missing)[:5]}"
