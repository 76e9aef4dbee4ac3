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


# ---- columns' sums of many rows ----------------------------------------------------------------

def added_in_a_row(rows, cols, dtype):
    """How many rows a lane adds one behind the other, and then teams, where 256 workgroups take the rows: pieces of 16 bytes to a lane, teams
    of 16 lanes or more, 1024 lanes to a workgroup."""
    team = 16
    while team * G.PIECES[dtype] < cols:
        team *= 2
    teams = 1024 // team
    return -(-rows // (256 * teams)) + teams


def sums_within(got, terms, longest, each):
    """Against the sum in 64 bits of terms that are `each` half steps off: `longest` additions and the last rounding."""
    want, size = terms.sum(dim=0), terms.abs().sum(dim=0)
    assert ((got.double() - want).abs() <= 1.01 * (longest + each + 1) * N.U * size).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(70000, 24), (20000, 300), (30000, 129), (9000, 1537), (5000, 4096)])
def test_sums_of_many_rows_are_as_near_as_their_order_allows(dtype, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x, dy = (torch.randn((rows, cols), device="cuda", generator=g).to(B.DTYPE_NAME[dtype]) for _ in range(2))
    d = B.make_layernorm_desc(rows=rows, cols=cols, dtype=dtype)
    mean, rstd, dw, db = (torch.empty(n, device="cuda") for n in (rows, rows, cols, cols))
    B.layernorm(d, x, mean=mean, rstd=rstd)
    B.layernorm_grad(d, dy, x, mean, rstd, torch.empty_like(x), dweight=dw, dbias=db)
    longest = added_in_a_row(rows, cols, dtype)
    sums_within(dw, dy.double() * ((x.double() - mean.double()[:, None]) * rstd.double()[:, None]), longest, 2)
    sums_within(db, dy.double(), longest, 0)


def test_the_gradient_of_more_rows_than_a_grid_has_teams():
    """70 million rows of 8, a period of 999983 again and again, by workgroups that keep the columns' sums: every period's dx is that of a call on
    one, whose rows go by teams as wide, and both sums are within their roundings."""
    period, rows, cols = 999983, 70_000_000, 8
    if torch.cuda.mem_get_info()[0] < (60 << 30):
        pytest.skip("needs 40 GB")
    g = torch.Generator(device="cuda").manual_seed(1)
    x1, dy1 = (torch.randn((period, cols), device="cuda", generator=g).half() for _ in range(2))
    few, d = (B.make_layernorm_desc(rows=n, cols=cols, dtype="f16") for n in (period, rows))
    mean1, rstd1 = torch.empty(period, device="cuda"), torch.empty(period, device="cuda")
    B.layernorm(few, x1, mean=mean1, rstd=rstd1)
    sums = [torch.empty(cols, device="cuda") for _ in range(4)]
    dx1 = torch.empty_like(x1)
    B.layernorm_grad(few, dy1, x1, mean1, rstd1, dx1, dweight=sums[0], dbias=sums[1])
    x, dy, mean, rstd = (t.repeat(rows // period + 1, *[1] * (t.dim() - 1))[:rows].contiguous() for t in (x1, dy1, mean1, rstd1))
    dx = torch.empty_like(x)
    B.layernorm_grad(d, dy, x, mean, rstd, dx, dweight=sums[2], dbias=sums[3])
    for at in range(0, rows, period):
        n = min(period, rows - at)
        assert torch.equal(dx[at:at + n], dx1[:n]), at
    xh1 = (x1.double() - mean1.double()[:, None]) * rstd1.double()[:, None]
    times = torch.full((period, 1), rows // period, dtype=torch.float64, device="cuda")
    times[:rows % period] += 1
    for terms, each, one, all_ in ((dy1.double() * xh1, 2, sums[0], sums[2]), (dy1.double(), 0, sums[1], sums[3])):
        sums_within(one, terms, added_in_a_row(period, cols, "f16"), each)
        sums_within(all_, terms * times, added_in_a_row(rows, cols, "f16"), each)
    del x, dy, dx
    torch.cuda.empty_cache()


# ---- several results in their inputs' places at once -------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(7, 3), (5000, 200), (33, 1537), (200, 1600), (9, 5001), (300, 8200), (3, 16385), (2, 70001)])
def test_sum_and_result_in_both_inputs_places(dtype, rows, cols):
    """The sum in x's place and the result in the residual's, and the other way round: as with buffers of their own, bit for bit."""
    x, res, w, b = (torch.from_numpy(v).cuda().to(B.DTYPE_NAME[dtype]) for v in G.inputs(rows, cols))
    d = B.make_layernorm_desc(rows=rows, cols=cols, dtype=dtype)

    def call(x, res, sum, y):
        rest = [torch.empty(rows, device="cuda") for _ in range(3)] + [torch.empty((rows, R.stride(cols)), dtype=torch.int8, device="cuda")]
        B.layernorm(d, x, residual=res, weight=w, bias=b, sum=sum, y=y, mean=rest[0], rstd=rest[1], row_scales=rest[2], row_codes=rest[3])
        return [sum, y, *rest]

    want = call(x, res, torch.empty_like(x), torch.empty_like(x))
    for swapped in (False, True):
        x1, res1 = x.clone(), res.clone()
        for got, good in zip(call(x1, res1, *((res1, x1) if swapped else (x1, res1))), want):
            assert torch.equal(got, good)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(7, 3), (7, 1600), (255, 1537), (700, 300), (1100, 9001), (1500, 40), (4097, 1600), (3, 16385), (2, 70001)])
def test_the_gradient_in_the_place_of_a_gradient_that_is_added_too(dtype, rows, cols):
    """dy, add and dx one buffer, with x a view of wider rows: as with buffers of their own, bit for bit."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    td = B.DTYPE_NAME[dtype]
    x = torch.randn((rows, cols + 5), device="cuda", generator=g).to(td)[:, :cols]
    dy, w = torch.randn((rows, cols), device="cuda", generator=g).to(td), torch.randn(cols, device="cuda", generator=g).to(td)
    d = B.make_layernorm_desc(rows=rows, cols=cols, ld=cols + 5, dtype=dtype)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.layernorm(d, x, mean=mean, rstd=rstd)
    want, got = ([torch.empty(cols, device="cuda") for _ in range(2)] for _ in range(2))
    dx, one = torch.empty_like(dy), dy.clone()
    B.layernorm_grad(d, dy, x, mean, rstd, dx, weight=w, add=dy, dweight=want[0], dbias=want[1])
    B.layernorm_grad(d, one, x, mean, rstd, one, weight=w, add=one, dweight=got[0], dbias=got[1])
    assert torch.equal(one, dx) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
