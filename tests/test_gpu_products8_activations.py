"""Activations and their slopes in binary32 far from zero, against 64 bits and relative to their values: what is small
there is right to its last bits, not only next to 1."""
import numpy as np
import pytest
import torch
from scipy.special import erfc

pytestmark = pytest.mark.gpu

import products8_reference as R
from paper_2206_01299_amd import binding as B

LEAST = 2.0 ** -149                     # a subnormal's step


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.fail("these tests need an MI355X")
    B.lib()


def block(x, act, dtype):
    """act(x): the block of a product that is zero, with x for its bias."""
    f, td = x.size, B.DTYPE_NAME[dtype]
    zero = [torch.zeros((1, 64), dtype=torch.int8).cuda(), torch.zeros(1).cuda(), torch.zeros((f, 64), dtype=torch.int8).cuda(),
            torch.zeros(f).cuda()]
    h = torch.empty((1, f), dtype=td, device="cuda")
    B.ffn8(B.make_ffn8_desc(m=1, f=f, k=64, dtype=dtype, act=act, gated=False), *zero, h, bias=torch.from_numpy(x).cuda().to(td))
    return h.double().cpu().numpy()[0]


def gradients(x, act, dtype):
    """The slope (the gate's gradient for dh = up = 1) and the value (the other half's) by ffn8_grad."""
    f, td = x.size, B.DTYPE_NAME[dtype]
    dh, pre = torch.ones((1, f), dtype=td, device="cuda"), torch.from_numpy(np.concatenate([x, np.ones_like(x)])[None]).cuda().to(td)
    out = torch.empty((1, 2 * f), dtype=td, device="cuda")
    B.ffn8_grad(B.make_ffn8_desc(m=1, f=f, dtype=dtype, act=act), dh, pre, out)
    both = out.double().cpu().numpy()[0]
    return both[:f], both[f:]


def held(x, dtype):
    """Numbers as the type holds them."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(B.DTYPE_NAME[dtype]).float().numpy()


def within(got, want, off, x, dtype, tag):
    """off: before the one rounding to the type."""
    off = off + R.HALF_STEP[dtype] * (np.abs(want) + off) + R.TINY[dtype]
    bad = np.argwhere(~(np.abs(got - want) <= off))
    assert bad.size == 0, (f"{tag}: {len(bad)} of {got.size} too far off, first at {x[bad[0, 0]]!r}: got {got[bad[0, 0]]!r}, "
                           f"want {want[bad[0, 0]]!r} +- {off[bad[0, 0]]:.3g}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_silu_is_right_relative_to_its_value(dtype):
    """float32: of e = exp(-|x|) (3 ulp allowed, 6 half steps), 1 + e (1), its reciprocal (an ulp, 2), their product (1) and
    that with x (1) come 11 half steps at most.  Below 2^-126, e and its product with the reciprocal are off by steps of 2^-149
    besides (4 in all), times |x|.  16 bits: the exponential's argument is rounded, which makes |x| half steps more, and
    two of those of its square."""
    rng = np.random.default_rng(4)
    x = held(np.concatenate([np.linspace(-104, 30, 40009), rng.uniform(-1.3, -1.2, 500), -(10.0 ** rng.uniform(-8, 0, 500)),
                             [0.0, -0.0, 88.0, -88.0, -87.5, -103.9]]), dtype)
    v = x.astype(np.float64)
    e = np.exp(-np.abs(v))
    p, q = np.where(v >= 0, 1 / (1 + e), e / (1 + e)), np.where(v >= 0, e / (1 + e), 1 / (1 + e))
    more = R.U * (0 if dtype == "f32" else 2 * np.abs(v) + 8)
    value_off = (12 * R.U + more) * np.abs(v) * p + 4 * np.abs(v) * LEAST
    if dtype == "f16":
        value_off = value_off + np.where(v < -87, np.abs(v) * 2.0 ** -125, 0.0)          # the exponential ends there
    within(block(x, "silu", dtype), v * p, value_off, x, dtype, "silu")
    slope, value = gradients(x, "silu", dtype)
    within(value, v * p, value_off, x, dtype, "silu's value")
    # p (10 half steps) and value q (11 and 10, and a product), added
    slope_off = (12 * R.U + more) * p + 2 * (12 * R.U + more) * np.abs(v) * p * q + (8 * np.abs(v) + 8) * LEAST
    if dtype == "f16":
        slope_off = slope_off + np.where(v < -87, np.abs(v) * 2.0 ** -124, 0.0)
    within(slope, p + v * p * q, slope_off, x, dtype, "silu's slope")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gradients_of_what_is_far_below_zero(dtype, act):
    """Where the exponential ends, in every type, up to the largest values: no infinity and no NaN."""
    x = np.concatenate([np.linspace(-130, -80, 2001), [-200.0, -1e3, -1e4, -6e4]])
    if dtype != "f16":
        x = np.concatenate([x, [-1e9, -1e18, -1e19, -1e20, -1e30, -3e38]])
    td, f = B.DTYPE_NAME[dtype], x.size
    pre = torch.from_numpy(np.concatenate([x, np.ones(f)])[None]).to(torch.float32).cuda().to(td)
    v = pre[0, :f].double().cpu().numpy()
    dh, out = torch.full((1, f), 0.5, dtype=td, device="cuda"), torch.empty((1, 2 * f), dtype=td, device="cuda")
    B.ffn8_grad(B.make_ffn8_desc(m=1, f=f, dtype=dtype, act=act), dh, pre, out)
    with np.errstate(over="ignore"):
        want = 0.5 * np.concatenate([R.act_slope(v, act), R.act(v, act)])
    got = out[0].double().cpu().numpy()
    # a tail below 2^-114, times x at most 80 of it in a slope: all of them are far below 2^-100 |x|
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= 2.0 ** -100 * np.abs(np.concatenate([v, v])) + R.TINY[dtype]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gelu_is_right_relative_to_its_value(dtype):
    """The erf form below 0 is x times a tail of the normal distribution.  float32: exp(-x^2 / 2) from an exact square (the
    exponential 6 half steps, the square's second part 1); t = 1 / (1 + c |x|) (a sum 1, a reciprocal 2), which the tail
    follows with a factor of 2.4 at most (7 in all); the polynomial (3.1 by its partial sums, 1 its own distance); two products
    and that with x (3): 21.1.  Subnormal densities are off by steps of 2^-149 (4 with the product), times |x|.  16 bits: the
    exponent's square, product and constant are rounded, half a step of x^2 / 2 each, once more where it is a square."""
    rng = np.random.default_rng(6)
    x = held(np.concatenate([np.linspace(-14.5, 14.5, 40001), rng.uniform(-0.8, -0.7, 500), -(10.0 ** rng.uniform(-8, 0, 500)),
                             10.0 ** rng.uniform(0, 4, 500), [0.0, -0.0, -5.0, -5.5, -6.0, -13.5, -14.2]]), dtype)
    v = x.astype(np.float64)
    below, phi = 0.5 * erfc(-v / np.sqrt(2)), np.exp(-0.5 * v * v) / np.sqrt(2 * np.pi)
    more = 0.0 if dtype == "f32" else R.U * (1.5 * np.minimum(v * v, 400) + 8)
    # above 0 it is 1 less a tail, rounded once
    cdf_off = (23 * R.U + more) * 0.5 * erfc(np.abs(v) / np.sqrt(2)) + np.where(v < 0, 0, R.U) + 4 * LEAST
    if dtype == "f16":
        cdf_off = cdf_off + np.where(np.abs(v) > 13, 2.0 ** -125, 0.0)               # the exponential ends there
    value_off = np.abs(v) * cdf_off + R.U * np.abs(v) * below
    within(block(x, "gelu", dtype), v * below, value_off, x, dtype, "gelu")
    slope, value = gradients(x, "gelu", dtype)
    within(value, v * below, value_off, x, dtype, "gelu's value")
    # x times a density (exponential 6, second part 1, its factor and two products 3), added
    bell_off = np.abs(v) * ((12 * R.U + more) * phi + 4 * LEAST + (2.0 ** -125 * (np.abs(v) > 13) if dtype == "f16" else 0))
    within(slope, below + v * phi, cdf_off + bell_off + R.U * np.abs(below + v * phi), x, dtype, "gelu's slope")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activations_of_no_numbers(dtype, act):
    """A NaN stays one, in the value and in the slope, an infinity is its own value, and what stands beside them is as without
    them.  Below, an infinity times 0 is a NaN, as in the formulas."""
    x = held(np.linspace(-8, 8, 67), dtype)
    x[[5, 20, 40, 66]] = np.nan, np.inf, -np.inf, np.nan
    ordinary = held(np.linspace(-8, 8, 67), dtype)
    plain = np.isfinite(x)
    for values, alone in ((block(x, act, dtype), block(ordinary, act, dtype)),
                          (gradients(x, act, dtype)[1], gradients(ordinary, act, dtype)[1])):
        assert np.isnan(values[[5, 40, 66]]).all() and values[20] == np.inf
        assert np.array_equal(values[plain], alone[plain])
    slope, alone = gradients(x, act, dtype)[0], gradients(ordinary, act, dtype)[0]
    assert np.isnan(slope[[5, 66]]).all() and np.array_equal(slope[plain], alone[plain])
