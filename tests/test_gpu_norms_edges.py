"""Layer norm and its gradient where a rounding or an order decides: means in the middle between two binary32 numbers, deviations
that overflow, columns' sums of many rows."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import norms_reference as N
import products8_reference as R
import test_gpu_norms as G
from paper_2206_01299_amd import binding as B
from test_gpu_products8 import DTYPES


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.fail("these tests need an MI355X")
    B.lib()


def below(v, dtype):
    """The largest value of the type that is not above v (v at least 0)."""
    v = min(v, {"f16": 65504.0, "bf16": 3.0e38, "f32": 3.0e38}[dtype])
    if dtype == "f16":
        h = np.float16(v)
        return float(np.nextafter(h, np.float16(0))) if float(h) > v else float(h)
    f = np.float32(v)
    f = np.nextafter(f, np.float32(0)) if float(f) > v else f
    return float(f) if dtype == "f32" else float((f.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32))


def rows_of_totals(totals, cols, dtype, rng):
    """Rows whose elements add up to exactly these totals, in any order of a binary64 sum."""
    x = np.zeros((len(totals), cols))
    for row, left in zip(x, totals):
        for at in rng.permutation(cols):
            if left == 0.0:
                break
            row[at] = below(left, dtype)
            left -= row[at]
        assert left == 0.0
    return x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(64, 49), (5000, 49), (64, 300), (5000, 600), (40, 1502), (300, 1537), (20, 4623), (12, 9215), (5, 18430), (4, 36860)])
def test_means_in_the_middle_between_two_numbers(dtype, rows, cols):
    """The mean is a quotient rounded in binary64, and that to binary32, ties to the even one.  Here every sum is exact and every quotient lies
    in the middle, for widths whose inverse in binary64 times the sum would leave it: the mean has no other choice of bits."""
    rng = np.random.default_rng([rows, cols])
    odd = 2.0 ** 24 + 1 + 2 * rng.integers(0, 2 ** 23, 40 * rows)
    means = odd * 2.0 ** -24                                               # 25 bits from 1 on
    apart = means[(means * cols * (1.0 / cols)).astype(np.float32) != means.astype(np.float32)]
    assert len(apart) >= 4
    means = np.resize(apart, rows)
    assert (means * cols / cols == means).all()
    x = rows_of_totals(means * cols, cols, dtype, rng)
    got = G.run_norm(x, dtype)["mean"].t.cpu().numpy()
    assert np.array_equal(got, means.astype(np.float32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(5, 3), (5, 40), (5, 1600), (5000, 96), (600, 1600), (5, 5001), (3, 20001)])
def test_deviations_that_pass_binary32(dtype, rows, cols):
    """Where x - mean overflows the row's rstd is 0: NaN at those elements, the bias at the others, no more than that."""
    big = {"bf16": 3.3895e38, "f32": 3.4028e38}[dtype]
    rng = np.random.default_rng([rows, cols])
    x, b, w = rng.standard_normal((rows, cols)), 1 + rng.random(cols), rng.standard_normal(cols)
    clean = G.run_norm(x, dtype, weight=w, bias=b)["y"].t.clone()
    x[1] = -big
    x[1, 1:3 if cols > 3 else 2] = big
    got = G.run_norm(x, dtype, weight=w, bias=b)
    assert np.isfinite(got["mean"].t[1].item()) and got["rstd"].t[1].item() == 0.0
    y, over = got["y"].t, torch.from_numpy(x[1] > 0).cuda()
    assert torch.isnan(y[1, over]).all()
    assert torch.equal(y[1, ~over], torch.from_numpy(b).float().cuda().to(y.dtype)[~over])
    assert torch.isnan(got["row_scales"].t[1]) and not got["row_codes"].t[1].any()
    others = torch.arange(rows, device="cuda") != 1
    assert torch.equal(y[others], clean[others])
