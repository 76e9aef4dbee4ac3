"""Plain forms of the layer norm, of AdamW and of the gradients' norm on the host: what the header fixes by binary32 steps
in binary32 (numpy rounds each once), everything else in 64 bits with how far the kernels' roundings may put it off."""
import math

import numpy as np

import products8_reference as R

U = R.U
F = np.float32
STATE_FLOOR = F(2.0 ** -100)
GROUP, M_TOP, R_TOP = 256, 127, 255


# ---- layer norm --------------------------------------------------------------------------------

def stored_sum(x, residual, to_type):
    """x + residual in binary32, as the type holds it."""
    return to_type((np.asarray(x, F) + np.asarray(residual, F)).astype(F))


def mean_of(s):
    """The rows' means in 64 bits, and how far a mean may be off: its one rounding, and n - 1 additions in binary64."""
    n = s.shape[1]
    s = s.astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        mean, size = s.sum(axis=1) / n, np.abs(s).sum(axis=1) / n
        return mean, U * np.abs(mean) + 2 * n * 2.0 ** -53 * size + R.TINY["f32"]


def rstd_of(s, mean, eps):
    """From the binary32 mean of the call itself: d rounds in binary32, the rest does in binary64, the result once."""
    n = s.shape[1]
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        d = (np.asarray(s, F) - np.asarray(mean, F)[:, None]).astype(F).astype(np.float64)
        rstd = 1.0 / np.sqrt((d * d).sum(axis=1) / n + eps)
        rstd = np.where(rstd >= 2.0 ** 128, np.inf, rstd)                       # past what binary32 holds
        return d, rstd, (U + (n + 8) * 2.0 ** -53) * np.abs(rstd) + R.TINY["f32"]


def normalised(d, rstd, weight, bias):
    """y in 64 bits from the call's own mean (in d) and rstd, and how far three binary32 steps may put it off."""
    with np.errstate(invalid="ignore", over="ignore"):
        y = d * np.asarray(rstd, np.float64)[:, None]
        off = U * np.abs(y)
        if weight is not None:
            y, off = y * weight, off * np.abs(weight) + U * np.abs(y * weight)
        if bias is not None:
            y, off = R.plus(y, off, bias)
        return y, off


def sums_off(terms, longest):
    """How far a binary32 sum of rounded terms may be off where no partial sum is added to more than `longest` times."""
    return longest * U * np.abs(terms)


def norm_grad(dy, x, mean, rstd, weight, add):
    """dx, dweight, dbias in 64 bits from the binary32 statistics, and how far off each may be.  Roundings, in half steps:
    x - mean and its product with rstd 2 (xh); dy * weight 1 (g); a term g * xh 4.  No lane adds more than 128 + cols / 64
    terms of a row one behind the other (twelve more levels join the lanes), nor more than 128 + rows / 64 rows of a
    column (a workgroup that takes 128 bytes of every row reads 64 rows at a time; and its 64 sums at most); the joined sums are added in binary64."""
    rows, cols = x.shape
    dy, x = dy.astype(np.float64), x.astype(np.float64)
    mean, rstd = mean.astype(np.float64)[:, None], rstd.astype(np.float64)[:, None]
    xh = (x - mean) * rstd
    g = dy if weight is None else dy * weight.astype(np.float64)
    along, across = g.mean(axis=1, keepdims=True), (g * xh).mean(axis=1, keepdims=True)
    longest = 128 + cols // 64 + 12
    along_off = (longest + 2) * U * np.abs(g).mean(axis=1, keepdims=True) + U * np.abs(along)
    across_off = (longest + 5) * U * np.abs(g * xh).mean(axis=1, keepdims=True) + U * np.abs(across)
    inner = g - along - xh * across
    inner_off = (U * np.abs(g) + along_off + np.abs(xh) * across_off + 3 * U * np.abs(xh * across)
                 + 2 * U * (np.abs(g) + np.abs(along) + np.abs(xh * across)))
    dx, dx_off = rstd * inner, rstd * inner_off + U * np.abs(rstd * inner)
    if add is not None:
        dx, dx_off = R.plus(dx, dx_off, add.astype(np.float64))
    deepest = 128 + rows // 64 + 64
    dw, db = (dy * xh).sum(axis=0), dy.sum(axis=0)
    dw_off = (deepest + 5) * U * np.abs(dy * xh).sum(axis=0)
    db_off = (deepest + 1) * U * np.abs(dy).sum(axis=0)
    return (dx, 1.01 * dx_off), (dw, 1.01 * dw_off), (db, 1.01 * db_off)


# ---- AdamW -------------------------------------------------------------------------------------

def up(n, to):
    return -(-n // to) * to


def state_bytes(n, bits):
    return 2 * up(4 * n, 64) if bits == 32 else 2 * up(n, 64) + 2 * up(4 * up(n, GROUP) // GROUP, 64)


def grouped(x):
    return np.pad(x, (0, up(len(x), GROUP) - len(x))).reshape(-1, GROUP)


def hold(x, top, least, z):
    """Codes and scales of binary32 magnitudes; z: a number, or one for each element of the groups."""
    n, x = len(x), grouped(np.asarray(x, F))
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        s = np.max(x, axis=1) if x.size else np.zeros(0, F)
        live = np.isfinite(s) & (s >= STATE_FLOOR)
        inv = np.where(live, F(top * top) / np.where(live, s, F(1)), F(0)).astype(F)
        u = (x * inv[:, None]).astype(F)
        u = np.where(live[:, None], u, F(0))
        k = np.floor(np.sqrt(u.astype(np.float64)))
        k = np.minimum(k, top)
        more = (u.astype(np.float64) - k * k) >= (np.asarray(z, F) * (2 * k + 1).astype(F)).astype(F)
        k = np.minimum(k + more, top)
        k = np.where(live[:, None] & (x > 0), np.maximum(k, least), 0)
    return k.reshape(-1)[:n], np.where(live, s, np.where(np.isfinite(s), F(0), F(np.nan))).astype(F)


def held_values(k, scales, top):
    """What (signed) codes stand for."""
    with np.errstate(invalid="ignore"):
        step = (scales / F(top * top)).astype(F)
        k = k.astype(F)
        return (grouped(k * np.abs(k)) * step[:, None]).astype(F).reshape(-1)[:len(k)]


class State:
    """One tensor's moments."""

    def __init__(self, n, bits):
        self.n, self.bits = n, bits
        groups = up(n, GROUP) // GROUP
        self.m, self.v = np.zeros(n, F), np.zeros(n, F)
        self.mk, self.rk = np.zeros(n, np.int8), np.zeros(n, np.uint8)
        self.ms, self.rs = np.zeros(groups, F), np.zeros(groups, F)

    def parts(self):
        return (self.m, self.v) if self.bits == 32 else (self.mk, self.rk, self.ms, self.rs)


def factors(lr, beta1, beta2, step, decay):
    return (F(1.0 - lr * decay), F(lr / (1.0 - beta1 ** step)), F(1.0 / math.sqrt(1.0 - beta2 ** step)))


def adamw(w, g, state, *, lr, beta1, beta2, eps, step, decay, scale=None, seed=None, first=0):
    """One step of one tensor: the new binary32 weights; `state` is updated.  `seed`: of stochastic rounding; `first`: the
    number of the tensor's first element in the call."""
    with np.errstate(invalid="ignore", over="ignore", under="ignore", divide="ignore"):
        keep, length, correct = factors(lr, beta1, beta2, step, decay)
        w, g = np.asarray(w, F), np.asarray(g, F)
        if scale is not None:
            g = (g * F(scale)).astype(F)
        if state.bits == 32:
            m, v = state.m, state.v
        else:
            m, r = held_values(state.mk, state.ms, M_TOP), held_values(state.rk, state.rs, R_TOP)
            v = (r * r).astype(F)
        m = ((m * F(beta1)).astype(F) + (g * F(1.0 - beta1)).astype(F)).astype(F)
        v = ((v * F(beta2)).astype(F) + ((g * F(1.0 - beta2)).astype(F) * g).astype(F)).astype(F)
        r = np.sqrt(v).astype(F)
        denominator = ((r * correct).astype(F) + F(eps)).astype(F)
        new = ((w * keep).astype(F) - ((m / denominator).astype(F) * length).astype(F)).astype(F)
        if state.bits == 32:
            state.m, state.v = m, v
            return new
        zm = zr = F(0.5)
        if seed is not None:
            blocks = np.arange(first // 4, first // 4 + up(state.n, GROUP) // 4, dtype=np.uint64)
            words = R.philox(blocks & np.uint64(0xFFFFFFFF), blocks >> np.uint64(32), (seed + step) % 2 ** 64).reshape(-1, GROUP)
            zm = ((words & np.uint64(0xFFFF)) + np.uint64(1)).astype(F) * F(2.0 ** -16)
            zr = ((words >> np.uint64(16)) + np.uint64(1)).astype(F) * F(2.0 ** -16)
        k, state.ms = hold(np.abs(m), M_TOP, 0, zm)
        state.mk = np.where(m < 0, -k, k).astype(np.int8)
        k, state.rs = hold(r, R_TOP, 1, zr)
        state.rk = k.astype(np.uint8)
        return new
