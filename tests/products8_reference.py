"""Plain forms of the 8-bit operators on the host: codes by the binary32 steps the header lists (numpy
rounds each once), everything else in 64 bits."""
import math

import numpy as np
from scipy.special import erf

FLOOR = np.float32(2.0 ** -120)
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}      # half a step, relative to the value
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}        # half a step among the subnormals
U = 2.0 ** -24


def stride(n):
    return -(-n // 64) * 64


def philox(c0, c1, seed):
    """The four words of Philox4x32-10 for arrays of counters (c0, c1, 0, 0)."""
    c0, c1 = (np.asarray(c, dtype=np.uint64) for c in np.broadcast_arrays(c0, c1))
    c2, c3 = np.zeros_like(c0), np.zeros_like(c0)
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c0, np.uint64(0xCD9E8D57) * c2
        c0, c1, c2, c3 = ((p1 >> np.uint64(32)) ^ c1 ^ np.uint64(k0), p1 & low,
                          (p0 >> np.uint64(32)) ^ c3 ^ np.uint64(k1), p0 & low)
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack([c0, c1, c2, c3], axis=-1)


def draws(rows, cols, seed, by_rows):
    """The uniform draw of every element of a [rows, cols] matrix, for its row or its column codes."""
    blocks = np.arange(-(-cols // 4), dtype=np.uint64) + np.uint64(2 ** 30 if by_rows else 2 ** 31)
    w = philox(blocks[None, :], np.arange(rows, dtype=np.uint64)[:, None], seed)
    return ((w >> np.uint64(8)).astype(np.float32) * np.float32(2.0 ** -24)).reshape(rows, -1)[:, :cols]


def quantise(x, r=np.float32(0.5)):
    """Codes (padded) and scales of the rows of a binary32 matrix."""
    x = np.asarray(x, dtype=np.float32)
    codes = np.zeros((x.shape[0], stride(x.shape[1])), dtype=np.int8)
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.abs(x).max(axis=1)
        live = np.isfinite(s) & (s >= FLOOR)
        inv = np.where(live, np.float32(127.0) / np.where(live, s, np.float32(1)), np.float32(0))
        y = np.floor((x * inv[:, None]).astype(np.float32) + r)
    y = np.where(live[:, None], y, np.float32(0))
    codes[:, :x.shape[1]] = np.clip(y, -127, 127).astype(np.int8)
    return codes, np.where(live, s, np.where(np.isfinite(s), np.float32(0), np.float32(np.nan)))


def projections(a, sa, b, sb, k, message=False):
    """The scaled product in 64 bits, and how far binary32 steps may put it off: the sum is exact, its
    conversion, the quotient of each scale and the two products round once each (5 half steps; a message's
    sum is formed of two parts, each converted, and added: 3 more, relative to the parts)."""
    ai = (a if message else a[:, :k]).astype(np.float64)          # whole numbers: their sums are exact
    bi = b[:, :k].astype(np.float64)
    steps = (sa.astype(np.float64) / (127.5 if message else 127.0))[:, None] * (sb.astype(np.float64) / 127.0)[None, :]
    if message:
        whole, ones = (ai - 128) @ bi.T, bi.sum(axis=1)[None, :]
        sums = whole + 0.5 * ones
        off = 5 * np.abs(sums) + 3 * (np.abs(whole) + 0.5 * np.abs(ones))
    else:
        sums = ai @ bi.T
        off = 5 * np.abs(sums)
    return sums * steps, off * U * np.abs(steps)


def plus(y, off, extra):
    """One more term, added in binary32 (one half step of the result)."""
    return y + extra, off + U * np.abs(y + extra)


def act(x, kind):
    if kind == "silu":
        return x / (1.0 + np.exp(-x))
    if kind == "gelu":
        return 0.5 * x * (1.0 + erf(x / math.sqrt(2.0)))
    return 0.5 * x * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))


def act_slope(x, kind):
    if kind == "silu":
        p = 1.0 / (1.0 + np.exp(-x))
        return p + x * p * (1.0 - p)
    if kind == "gelu":
        return 0.5 * (1.0 + erf(x / math.sqrt(2.0))) + x * np.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)
    t = np.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3))
    return 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 0.134145 * x * x)


# An activation's value is x times a number between 0 and 1.  That number is off by at most 8 half steps of 1:
# silu and tanh form: the exponential 2, one sum, one quotient, one product 4 in all, the argument's own
# roundings (at most 5, tanh form) weighted by y p (1 - p) <= 0.23; erf form: erf 4, argument 2 weighted by
# y phi(y) <= 0.25, one sum, halved.  The slope adds a term x p (1 - p) s (or x phi), below 1 and off by at
# most 8 half steps more.  Slopes are below 1.14 in magnitude.
VALUE_OFF, SLOPE_OFF, STEEPEST = 10 * U, 16 * U, 1.14


def after_act(y, off, kind):
    return act(y, kind), STEEPEST * off + VALUE_OFF * np.abs(y)


def times(a, off_a, b, off_b):
    return a * b, np.abs(a) * off_b + np.abs(b) * off_a + off_a * off_b + U * np.abs(a * b)


def close(got, want, off, dtype, tag):
    """got: the stored values; want, off in 64 bits, before the one rounding to the stored type."""
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape, f"{tag}: {got.shape} instead of {want.shape}"
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), f"{tag}: NaN in other places"
    allow = 1.0001 * (off + HALF_STEP[dtype] * (np.abs(want) + off) + TINY[dtype])
    miss = np.where(nan, 0.0, np.abs(got - np.where(nan, 0.0, want)) - np.where(nan, 0.0, allow))
    bad = np.argwhere(miss > 0)
    assert bad.size == 0, (f"{tag}: {len(bad)} of {got.size} values too far off, first at {bad[0].tolist()}: "
                           f"got {got[tuple(bad[0])]!r}, want {want[tuple(bad[0])]!r} +- {allow[tuple(bad[0])]:.3g}")
