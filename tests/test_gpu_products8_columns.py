"""quant8 of matrices of many rows and columns: tiles of 128 rows that are whole, several to a workgroup, maxima of rows
from several spans of columns; sums of columns that binary32 holds exactly, so that every row and every block counts."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import test_gpu_products8 as T
from paper_2206_01299_amd import binding as B

# rows, columns: 561 tiles of 128 x 128 below each other, nine spans; 2145, two to a workgroup, seventeen spans
WIDE = [(4100, 2057), (8200, 4100)]
# one tile, few and many blocks of rows, both heights of tiles, workgroups of several tiles
SUMS = [(1, 5), (64, 130), (129, 130), (300, 67), (1021, 1537), (4100, 2057), (33001, 131), (65601, 3), (262200, 3), (1048700, 1),
        (8200, 4100)]


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.fail("these tests need an MI355X")
    B.lib()


@pytest.mark.parametrize("dtype", T.DTYPES)
@pytest.mark.parametrize("rows,cols", WIDE)
def test_quant8_of_many_rows_and_columns(dtype, rows, cols):
    x = T.activations(np.random.default_rng([rows, cols]), rows, cols)
    T.run_quant8(x, dtype)
    T.run_quant8(x, dtype, pad=3, sums=False)
    T.run_quant8(x, dtype, pad=28, by_rows=False, offset=1)


@pytest.mark.parametrize("dtype,rows,cols", [("f32", *WIDE[0]), ("bf16", *WIDE[0]), ("f16", *WIDE[1])])
def test_quant8_of_many_rows_and_columns_stochastic(dtype, rows, cols):
    x = T.activations(np.random.default_rng([cols, rows]), rows, cols)
    T.run_quant8(x, dtype, rounding=1, seed=rows * cols, sums=False, pad=cols % 2)


@pytest.mark.parametrize("dtype", T.DTYPES)
@pytest.mark.parametrize("rows,cols", SUMS)
def test_sums_of_columns_are_exact_where_binary32_holds_them(dtype, rows, cols):
    """Whole numbers to 8 in magnitude: every partial sum is a whole number below 2^24, in any order.  With the codes of rows,
    of columns, of both, and by themselves."""
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    whole = torch.randint(-8, 9, (rows, cols), generator=gen, device="cuda", dtype=torch.int8)
    x, want = whole.to(B.DTYPE_NAME[dtype]), whole.sum(dim=0, dtype=torch.int64)
    d = B.make_quant8_desc(rows=rows, cols=cols, dtype=dtype)
    by_rows = dict(row_codes=torch.empty((rows, T.R.stride(cols)), dtype=torch.int8, device="cuda"),
                   row_scales=torch.empty(rows, device="cuda"))
    by_cols = dict(col_codes=torch.empty((cols, T.R.stride(rows)), dtype=torch.int8, device="cuda"),
                   col_scales=torch.empty(cols, device="cuda"))
    for codes in ({}, by_rows, by_cols, {**by_rows, **by_cols}):
        sums = torch.full((cols,), float("nan"), device="cuda")
        B.quant8(d, x, **codes, col_sums=sums)
        assert torch.equal(sums.double(), want.double()), sorted(codes)
