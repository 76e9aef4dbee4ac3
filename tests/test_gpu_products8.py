"""The 8-bit operators on the GPU against their plain forms in 64 bits: codes and scales exactly, products
and activations within the roundings that their binary32 steps make."""
import threading

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import products8_reference as R
from paper_2206_01299_amd import binding as B
from paper_2206_01299_amd import workloads as W

DTYPES = ["f32", "f16", "bf16"]
ACTS = ["silu", "gelu", "gelu_tanh"]
MARK = 77                               # what memory holds that a call must leave alone


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.fail("these tests need an MI355X")
    B.lib()


def stored(x, dtype):
    """Values as the type holds them: (device tensor, binary32 array)."""
    t = torch.from_numpy(np.asarray(x, dtype=np.float32)).cuda().to(B.DTYPE_NAME[dtype])
    return t, t.float().cpu().numpy()


def numbers(t):
    return t.double().cpu().numpy()


class Framed:
    """A tensor inside a larger allocation whose other bytes are checked to be left alone."""

    def __init__(self, shape, dtype, lead=64):
        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        self.raw = torch.full((lead + n + 256,), MARK, dtype=torch.uint8, device="cuda")
        self.lead, self.n = lead, n
        self.t = self.raw[lead:lead + n].view(dtype).view(shape)

    def check(self, tag):
        r = self.raw.cpu()
        assert (r[:self.lead] == MARK).all() and (r[self.lead + self.n:] == MARK).all(), f"{tag}: written outside"


def activations(rng, rows, cols):
    x = rng.standard_normal((rows, cols))
    x[:, rng.random(cols) < 0.02] *= 20.0
    return x


# ---- quant8 ------------------------------------------------------------------------------------

def run_quant8(x, dtype, pad=0, rounding=0, seed=0, by_rows=True, by_cols=True, sums=True, offset=0, workspace=True):
    rows, cols = x.shape
    wide = torch.full((rows * (cols + pad) + offset,), 3.0, dtype=B.DTYPE_NAME[dtype], device="cuda")
    t = wide[offset:].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.from_numpy(np.asarray(x, dtype=np.float32)))
    xf = t.float().cpu().numpy()
    d = B.make_quant8_desc(rows=rows, cols=cols, ld=cols + pad, dtype=dtype, rounding=rounding, rng_seed=seed)
    rc, rs = Framed((rows, R.stride(cols)), torch.int8), Framed((rows,), torch.float32)
    cc, cs = Framed((cols, R.stride(rows)), torch.int8), Framed((cols,), torch.float32)
    cq = Framed((cols,), torch.float32)
    ws = Framed((B.quant8_workspace_bytes(d),), torch.uint8)
    B.quant8(d, t, row_codes=rc.t if by_rows else None, row_scales=rs.t if by_rows else None,
             col_codes=cc.t if by_cols else None, col_scales=cs.t if by_cols else None, col_sums=cq.t if sums else None,
             workspace=ws.t if workspace else None)
    torch.cuda.synchronize()
    tag = f"{dtype} {rows}x{cols} pad {pad} rounding {rounding}"
    for f in (rc, rs, cc, cs, cq, ws):
        f.check(tag)
    for on, codes, scales, v, r in ((by_rows, rc, rs, xf, True), (by_cols, cc, cs, xf.T, False)):
        if not on:
            assert (codes.raw == MARK).all() and (scales.raw == MARK).all()
            continue
        off = np.float32(0.5) if not rounding else R.draws(rows, cols, seed, r) if r else R.draws(rows, cols, seed, r).T
        want_codes, want_scales = R.quantise(v, off)
        assert np.array_equal(scales.t.cpu().numpy(), want_scales, equal_nan=True), f"{tag}: scales of {'rows' if r else 'columns'}"
        got = codes.t.cpu().numpy()
        bad = np.argwhere(got != want_codes)
        assert bad.size == 0, f"{tag}: {len(bad)} codes of {'rows' if r else 'columns'}, first at {bad[0].tolist()}"
    if sums:
        with np.errstate(invalid="ignore"):
            want = xf.astype(np.float64).sum(axis=0)
            # one half step of a partial sum per addition, in any order: at most rows of them, each at most sum |x|
            off = np.nan_to_num(rows * R.U * np.abs(xf.astype(np.float64)).sum(axis=0), nan=0, posinf=0)
        got = cq.t.cpu().numpy()
        fin = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want)), tag
        assert (np.abs(got - want)[fin] <= off[fin] + R.TINY["f32"]).all(), f"{tag}: sums"
    return rc.t, rs.t, cc.t, cs.t, cq.t


SIZES = [(1, 1), (1, 1600), (1, 7), (7, 1), (3, 64), (64, 64), (65, 63), (129, 130), (2, 5000), (5000, 3), (257, 1537),
         (1024, 256), (33, 12800), (640, 4096), (4097, 72), (1, 70001), (9000, 520)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quant8(dtype, rows, cols):
    rng = np.random.default_rng([rows, cols])
    x = activations(rng, rows, cols)
    run_quant8(x, dtype)
    run_quant8(x, dtype, pad=1 + rows % 9, by_cols=False, sums=False)
    run_quant8(x, dtype, pad=8, by_rows=False, offset=1, workspace=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 33), (70, 130), (300, 67), (65, 1600)])
def test_quant8_stochastic(dtype, rows, cols):
    x = activations(np.random.default_rng(5), rows, cols)
    run_quant8(x, dtype, rounding=1, seed=0x123456789ABCDEF + rows)
    run_quant8(x, dtype, rounding=1, seed=2 ** 64 - 1, pad=3, sums=False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_quant8_of_what_is_no_ordinary_number(dtype):
    """Rows and columns of zeros, below the floor, among the subnormals, of the largest values, and with an
    infinity or a NaN in them: scale 0 or NaN and codes 0, the others untouched by them."""
    big = {"f16": 65504.0, "bf16": 3.3895e38, "f32": 3.4028e38}[dtype]
    tiny = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}[dtype]
    x = np.random.default_rng(1).standard_normal((200, 150))
    x[3] = 0.0
    x[:, 5] = -0.0
    x[7] *= tiny * 4
    x[:, 9] = tiny
    x[11] = np.where(np.arange(150) % 2, big, -big)
    run_quant8(x, dtype, sums=False)
    x[13, 20] = np.inf
    x[15, 22] = np.nan
    x[17, 24] = -np.inf
    run_quant8(x, dtype, sums=False)
    x = np.random.default_rng(2).standard_normal((130, 70)) * 1e-3
    x[40, 3], x[41, 3] = np.inf, -np.inf
    run_quant8(x, dtype)
    x = np.full((70, 70), np.nan)
    run_quant8(x, dtype)
    half = np.zeros((64, 130))                      # every value on a tie
    half[:, 0], half[0] = 127, 127
    half[1:, 1:] = (np.arange(129) % 127 - 63)[None, :] + 0.5
    run_quant8(half, dtype)


# ---- matmul8 -----------------------------------------------------------------------------------

def operands(rng, m, n, k, message=False):
    a = activations(rng, m, k)
    if message:
        d = B.make_desc(batch=1, n_per=m * k, bits=8, group=k, dtype="f32") if k else None
        codes, scales = torch.empty((m, k), dtype=torch.uint8, device="cuda"), torch.zeros(m, device="cuda")
        if k:
            B.grad_quant(d, torch.from_numpy(a.astype(np.float32)).cuda(), codes, scales)
        ac, sa = codes.cpu().numpy(), scales.cpu().numpy()
    else:
        ac, sa = R.quantise(a) if k else (np.zeros((m, 0), np.int8), np.ones(m, np.float32))
    bc, sb = R.quantise(rng.standard_normal((n, k)) * 0.02) if k else (np.zeros((n, 0), np.int8), np.ones(n, np.float32))
    return ac, sa, bc, sb


def run_matmul8(m, n, k, dtype, message=False, bias=False, add=False, in_place=False, seed=0, workspace=True, data=None, lead=64):
    rng = np.random.default_rng([m, n, k, seed])
    ac, sa, bc, sb = data if data is not None else operands(rng, m, n, k, message)
    want, off = R.projections(ac, sa, bc, sb, k, message)
    tb = ta = None
    if bias:
        tb, v = stored(rng.standard_normal(n), dtype)
        want, off = R.plus(want, off, v[None, :].astype(np.float64))
    if add:
        ta, v = stored(rng.standard_normal((m, n)), dtype)
        want, off = R.plus(want, off, v.astype(np.float64))
    out = Framed((m, n), B.DTYPE_NAME[dtype], lead)
    if in_place:
        out.t.copy_(ta)
        ta = out.t
    d = B.make_matmul8_desc(m=m, n=n, k=k, dtype=dtype, message=message)
    ws = Framed((B.matmul8_workspace_bytes(d),), torch.uint8)
    dev = [torch.from_numpy(v).cuda() for v in (ac, sa, bc, sb)]
    B.matmul8(d, *dev, out.t, bias=tb, add=ta, workspace=ws.t if workspace else None)
    torch.cuda.synchronize()
    tag = f"{dtype} {m}x{n}x{k} message {message} bias {bias} add {add}"
    out.check(tag)
    ws.check(tag)
    R.close(numbers(out.t), want, off, dtype, tag)


PRODUCTS = [(1, 1, 1), (1, 16, 64), (1, 1600, 640), (2, 100, 65), (3, 33, 1601), (5, 6400, 128), (16, 48, 63), (17, 130, 200),
            (31, 64, 4096), (33, 257, 320), (63, 65, 127), (64, 64, 64), (65, 300, 1000), (128, 128, 1536), (200, 96, 96),
            (257, 513, 385), (1000, 40, 70), (300, 1025, 1472), (513, 770, 2112), (1, 5, 100000), (40, 24, 131072)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_matmul8(dtype, m, n, k):
    run_matmul8(m, n, k, dtype, bias=True)
    run_matmul8(m, n, k, dtype, add=True, in_place=(m + n) % 2 == 0, workspace=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(1, 16, 16), (1, 1601, 1600), (4, 64, 48), (19, 33, 80), (64, 64, 64), (130, 129, 208), (257, 300, 1600),
                                   (70, 520, 4112), (515, 257, 1040)])
def test_matmul8_of_a_message(dtype, m, n, k):
    run_matmul8(m, n, k, dtype, message=True)
    run_matmul8(m, n, k, dtype, message=True, bias=True, add=True)


@pytest.mark.parametrize("m,n,k", [(1, 7, 0), (70, 65, 0)])
def test_matmul8_without_anything_to_sum(m, n, k):
    run_matmul8(m, n, k, "f16", bias=True)
    run_matmul8(m, n, k, "f32", message=True, add=True)


@pytest.mark.parametrize("m", [1, 8, 70, 300])
def test_matmul8_sums_at_the_limit_of_32_bits(m):
    """All codes at their extremes, at the longest sum: 131072 * 127 * 127, and 131072 * 127.5 * 127 of a message."""
    k, n = 131072, 80
    sa, sb = np.linspace(1, 2, m, dtype=np.float32), np.linspace(1, 3, n, dtype=np.float32)
    sign = np.where(np.arange(n) % 2, -127, 127).astype(np.int8)
    data = (np.full((m, k), 127, np.int8), sa, np.repeat(sign[:, None], k, axis=1), sb)
    run_matmul8(m, n, k, "f32", data=data)
    for level in (0, 255):
        run_matmul8(m, n, k, "f32", message=True, data=(np.full((m, k), level, np.uint8),) + data[1:])


@pytest.mark.parametrize("m", [1, 12, 100, 300])
def test_matmul8_scales_that_are_zero_or_no_number(m):
    rng = np.random.default_rng(3)
    ac, sa, bc, sb = operands(rng, m, 70, 200)
    sa[0], sb[3] = 0.0, 0.0
    sb[5] = np.nan
    run_matmul8(m, 70, 200, "bf16", bias=True, data=(ac, sa, bc, sb))
    if m > 1:
        sa[m - 1] = np.nan
        run_matmul8(m, 70, 200, "f32", data=(ac, sa, bc, sb))


@pytest.mark.parametrize("dtype", DTYPES)
def test_matmul8_at_any_elements_address(dtype):
    """out, bias and add may start at any element."""
    size = torch.empty(0, dtype=B.DTYPE_NAME[dtype]).element_size()
    for m, n in ((3, 37), (70, 131), (300, 260)):
        run_matmul8(m, n, 192, dtype, lead=64 + size, add=True, in_place=True)
        run_matmul8(m, n, 192, dtype, lead=64 + 3 * size, bias=True)


# ---- ffn8 --------------------------------------------------------------------------------------

def run_ffn8(m, f, k, dtype, act, gated, bias=False, pre=True, seed=0):
    rng = np.random.default_rng([m, f, k, seed])
    w = f * (2 if gated else 1)
    ac, sa, bc, sb = operands(rng, m, w, k)
    sb = (sb * 3).astype(np.float32)
    p, off = R.projections(ac, sa, bc, sb, k)
    tb = None
    if bias:
        tb, v = stored(rng.standard_normal(w), dtype)
        p, off = R.plus(p, off, v[None, :].astype(np.float64))
    h, hoff = R.after_act(p[:, :f], off[:, :f], act)
    if gated:
        h, hoff = R.times(h, hoff, p[:, f:], off[:, f:])
    d = B.make_ffn8_desc(m=m, f=f, k=k, dtype=dtype, act=act, gated=gated)
    out, po = Framed((m, f), B.DTYPE_NAME[dtype]), Framed((m, w), B.DTYPE_NAME[dtype])
    dev = [torch.from_numpy(v).cuda() for v in (ac, sa, bc, sb)]
    B.ffn8(d, *dev, out.t, bias=tb, pre=po.t if pre else None)
    torch.cuda.synchronize()
    tag = f"{dtype} {m}x{f}x{k} {act} gated {gated} bias {bias}"
    out.check(tag)
    po.check(tag)
    R.close(numbers(out.t), h, hoff, dtype, tag)
    if pre:
        R.close(numbers(po.t), p, off, dtype, tag + " pre")
    else:
        assert (po.raw == MARK).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,f,k", [(1, 1, 1), (1, 6400, 100), (2, 17, 64), (8, 33, 1536), (16, 64, 65), (30, 200, 320), (65, 31, 200),
                                   (64, 32, 128), (128, 129, 1600), (257, 400, 385), (300, 513, 640)])
def test_ffn8(dtype, m, f, k):
    for i, act in enumerate(ACTS):
        run_ffn8(m, f, k, dtype, act, gated=True, bias=i == 0, pre=i != 1)
        run_ffn8(m, f, k, dtype, act, gated=False, bias=i != 0, pre=i == 1)


def run_ffn8_grad(dh, pre, f, dtype, act, gated, in_place=False):
    m, w = pre.shape
    tdh, dhf = stored(dh, dtype)
    tpre, pf = stored(pre, dtype)
    out = Framed((m, w), B.DTYPE_NAME[dtype])
    if in_place:
        out.t.copy_(tpre)
        tpre = out.t
    B.ffn8_grad(B.make_ffn8_desc(m=m, f=f, dtype=dtype, act=act, gated=gated), tdh, tpre, out.t)
    torch.cuda.synchronize()
    tag = f"{dtype} {m}x{f} {act} gated {gated} in place {in_place}"
    out.check(tag)
    d, g = dhf.astype(np.float64), pf[:, :f].astype(np.float64)
    with np.errstate(over="ignore"):
        slope, value = R.act_slope(g, act), R.act(g, act)
    up = pf[:, f:].astype(np.float64) if gated else np.ones_like(g)
    # dh * up rounds once (gated), times the slope once more, each half a step of the product
    want = d * up * slope
    off = np.abs(d * up) * R.SLOPE_OFF + 2.0 * R.U * np.abs(want) + R.TINY["f32"] * R.STEEPEST
    if gated:
        low = d * value
        want, off = np.hstack([want, low]), np.hstack([off, np.abs(d) * R.VALUE_OFF * np.abs(g) + 2.0 * R.U * np.abs(low)])
    R.close(numbers(out.t), want, off, dtype, tag)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,f", [(1, 1), (1, 6400), (3, 7), (17, 64), (5, 1601), (130, 520), (1000, 48)])
def test_ffn8_grad(dtype, m, f):
    rng = np.random.default_rng([m, f])
    for act in ACTS:
        for gated in (True, False):
            run_ffn8_grad(rng.standard_normal((m, f)), 2.0 * rng.standard_normal((m, 2 * f if gated else f)), f, dtype, act,
                          gated, in_place=f % 2 == 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
def test_ffn8_grad_far_from_zero(dtype, act):
    """Where the slope is 0 or 1 to the last bit, up to the largest values: no infinity or NaN comes of it."""
    g = np.concatenate([np.linspace(-120, 120, 961), [1e4, -1e4, 6e4, -6e4, 0.0, -0.0]])[None, :]
    if dtype != "f16":
        g = np.concatenate([g, np.array([[1e19, -1e19, 1e30, -1e30, 3e38, -3e38]])], axis=1)
    g = np.clip(g, -88.0, None) if act == "silu" else g           # beyond, the plain form overflows
    f = g.shape[1]
    d = np.full((1, f), 0.5)
    run_ffn8_grad(d, np.hstack([g, np.ones((1, f))]), f, dtype, act, True)
    run_ffn8_grad(d, g, f, dtype, act, False)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [True, False])
def test_ffn8_grad_is_the_difference_of_ffn8(act, gated):
    """The slope along a direction against the change of the block's output between two biases a step apart.
    The product is zero (no tokens' codes), so the bias is the projection."""
    m, f, step = 1, 256, 2.0 ** -6
    w = 2 * f if gated else f
    rng = np.random.default_rng(9)
    pre, way, dh = rng.standard_normal(w), rng.standard_normal(w), rng.standard_normal((m, f))
    zero = [torch.zeros((m, 64), dtype=torch.int8).cuda(), torch.zeros(m).cuda(), torch.zeros((w, 64), dtype=torch.int8).cuda(),
            torch.zeros(w).cuda()]
    d = B.make_ffn8_desc(m=m, f=f, k=64, dtype="f32", act=act, gated=gated)

    def block(p):
        h = torch.empty((m, f), device="cuda")
        B.ffn8(d, *zero, h, bias=torch.from_numpy(p.astype(np.float32)).cuda())
        return (numbers(h) * dh).sum()

    out = torch.empty((m, w), device="cuda")
    B.ffn8_grad(d, torch.from_numpy(dh.astype(np.float32)).cuda(), torch.from_numpy(pre.astype(np.float32)[None]).cuda(), out)
    got = (numbers(out)[0] * way).sum()
    diff = (block(pre + step * way) - block(pre - step * way)) / (2 * step)
    # a central difference is off by step^2 / 6 of third derivatives (below 5 each way^3, up to the other factor),
    # and by the rounding of the two sums over the step
    room = step ** 2 / 6 * 5 * (np.abs(dh[0]) * (1 + np.abs(way[:f]) ** 3) * (1 + 2 * np.abs(pre[-f:]) + 3 * np.abs(way[-f:]))).sum()
    room += 40 * R.U * np.abs(dh).sum() * (1 + np.abs(pre).max()) ** 2 / step
    assert abs(got - diff) <= room, (got, diff, room)
    assert room < 0.2 * np.sqrt((numbers(out) ** 2).sum())                      # and it says something


# ---- together ----------------------------------------------------------------------------------

def stage_step(x, w1, w2, message, mscale, dtype, buf=None, stream=None):
    """A stage's gated block in 8 bits: forward from its tokens, backward from the message that the next stage
    sent; returns every result.  ``buf`` keeps what an earlier call of the same sizes allocated."""
    td = B.DTYPE_NAME[dtype]
    (m, k), f = x.shape, w2.shape[1]
    b = {} if buf is None else buf

    def get(name, shape, dt=td):
        if name not in b:
            b[name] = torch.empty(shape, dtype=dt, device="cuda")
        return b[name]

    def codes(name, t, rows=True, cols=False, sums=False):
        n, c = t.shape
        d = B.make_quant8_desc(rows=n, cols=c, dtype=t.dtype)
        out = {}
        if rows:
            out.update(row_codes=get(name + ".r", (n, R.stride(c)), torch.int8), row_scales=get(name + ".rs", (n,), torch.float32))
        if cols:
            out.update(col_codes=get(name + ".c", (c, R.stride(n)), torch.int8), col_scales=get(name + ".cs", (c,), torch.float32))
        if sums:
            out.update(col_sums=get(name + ".q", (c,), torch.float32))
        B.quant8(d, t, **out, workspace=get(name + ".ws", (B.quant8_workspace_bytes(d),), torch.uint8), stream=stream)
        return out

    def product(name, m_, n_, k_, *ops, dt=dtype, message=False):
        out = get(name, (m_, n_), B.DTYPE_NAME[dt])
        B.matmul8(B.make_matmul8_desc(m=m_, n=n_, k=k_, dtype=dt, message=message), *ops, out, stream=stream)
        return out

    qx = codes("x", x, cols=True)
    q1 = codes("w1", w1, cols=True)                       # [2 f, k]
    q2 = codes("w2", w2, cols=True)                       # [k, f]
    d = B.make_ffn8_desc(m=m, f=f, k=k, dtype=dtype)
    h, pre = get("h", (m, f)), get("pre", (m, 2 * f))
    B.ffn8(d, qx["row_codes"], qx["row_scales"], q1["row_codes"], q1["row_scales"], h, pre=pre, stream=stream)
    qh = codes("h", h, cols=True)
    y = product("y", m, k, f, qh["row_codes"], qh["row_scales"], q2["row_codes"], q2["row_scales"])
    dh = product("dh", m, f, k, message, mscale, q2["col_codes"], q2["col_scales"], message=True)
    dy = get("dy", (m, k))
    B.grad_dequant(B.make_desc(batch=1, n_per=m * k, bits=8, group=k, dtype=dtype), message, mscale, dy, stream)
    qdy = codes("dy", dy, rows=False, cols=True, sums=True)
    dw2 = product("dw2", k, f, m, qdy["col_codes"], qdy["col_scales"], qh["col_codes"], qh["col_scales"], dt="f32")
    dpre = get("dpre", (m, 2 * f))
    B.ffn8_grad(d, dh, pre, dpre, stream=stream)
    qp = codes("dpre", dpre, cols=True)
    dx = product("dx", m, k, 2 * f, qp["row_codes"], qp["row_scales"], q1["col_codes"], q1["col_scales"])
    dw1 = product("dw1", 2 * f, k, m, qp["col_codes"], qp["col_scales"], qx["col_codes"], qx["col_scales"], dt="f32")
    return dict(h=h, pre=pre, y=y, dh=dh, dw2=dw2, dpre=dpre, dx=dx, dw1=dw1, db2=qdy["col_sums"])


def stage_inputs(m, k, f, dtype, seed=0):
    rng = np.random.default_rng(seed)
    x, w1, w2 = (stored(v, dtype)[0] for v in (rng.standard_normal((m, k)), rng.standard_normal((2 * f, k)) / np.sqrt(k),
                                               rng.standard_normal((k, f)) / np.sqrt(f)))
    message, scales = torch.empty(m * k, dtype=torch.uint8, device="cuda"), torch.empty(m, device="cuda")
    B.grad_quant(B.make_desc(batch=1, n_per=m * k, bits=8, group=k, dtype="f32"),
                 torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32)).cuda(), message, scales)
    return x, w1, w2, message, scales


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,k,f", [(96, 64, 80), (300, 160, 224)])
def test_a_stages_step_in_8_bits(dtype, m, k, f):
    """Every result against the 64-bit chain of the values that the codes stand for: each quantisation is off by
    at most half a code's step (scale / 254) of its vector's largest value, so a sum of products over l terms is
    off by about sqrt(l) times the two operands' share; the chain's relative errors (2-norm) stay below 4 %."""
    x, w1, w2, message, scales = stage_inputs(m, k, f, dtype)
    got = stage_step(x, w1, w2, message, scales, dtype)
    torch.cuda.synchronize()
    X, W1, W2 = (numbers(t) for t in (x, w1, w2))
    G = (message.view(m, k).cpu().numpy().astype(np.float64) - 127.5) * (numbers(scales) / 127.5)[:, None]
    p = X @ W1.T
    value, slope, up = R.act(p[:, :f], "silu"), R.act_slope(p[:, :f], "silu"), p[:, f:]
    h = value * up
    dh = G @ W2
    dpre = np.hstack([dh * up * slope, dh * value])
    want = dict(h=h, pre=p, y=h @ W2.T, dh=dh, dw2=G.T @ h, dpre=dpre, dx=dpre @ W1, dw1=dpre.T @ X, db2=G.sum(axis=0))
    for name, w in want.items():
        rel = np.linalg.norm(numbers(got[name]) - w) / np.linalg.norm(w)
        assert rel < 0.04, f"{dtype} {name}: {rel:.4f}"


def test_a_stages_step_on_another_stream_and_in_a_graph():
    """The same bits on a side stream and from a captured graph, replayed with other inputs and eager work between
    the replays."""
    m, k, f = 200, 128, 96
    x, w1, w2, message, scales = stage_inputs(m, k, f, "bf16")
    plain = {n: t.clone() for n, t in stage_step(x, w1, w2, message, scales, "bf16").items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = stage_step(x, w1, w2, message, scales, "bf16")
    named = stage_step(x, w1, w2, message, scales, "bf16", stream=side)
    torch.cuda.synchronize()
    for n in plain:
        assert torch.equal(plain[n], other[n]) and torch.equal(plain[n], named[n]), n
    buf, g = {}, torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        stage_step(x, w1, w2, message, scales, "bf16", buf)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        out = stage_step(x, w1, w2, message, scales, "bf16", buf)
    for seed in (0, 1, 2, 1):
        nx, _, _, nm, ns = stage_inputs(m, k, f, "bf16", seed)
        want = {n: t.clone() for n, t in stage_step(nx, w1, w2, nm, ns, "bf16").items()}
        x.copy_(nx); message.copy_(nm); scales.copy_(ns)
        g.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(out[n], want[n]), f"replay with inputs {seed}: {n}"


def test_two_graphs_that_share_a_workspace():
    """Replayed one after the other on one stream: a call uses its workspace only while it runs."""
    torch.manual_seed(0)
    shapes, graphs = [(300, 200), (70, 333)], []
    ws = torch.empty(max(B.quant8_workspace_bytes(B.make_quant8_desc(rows=r, cols=c, dtype="f32")) for r, c in shapes),
                     dtype=torch.uint8, device="cuda")
    for r, c in shapes:
        x = torch.randn(r, c, device="cuda")
        d = B.make_quant8_desc(rows=r, cols=c, dtype="f32")
        cc, cs = torch.empty((c, R.stride(r)), dtype=torch.int8, device="cuda"), torch.empty(c, device="cuda")
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            B.quant8(d, x, col_codes=cc, col_scales=cs, workspace=ws)
        graphs.append((g, x, cc, cs))
    for _ in range(3):
        for g, x, cc, cs in graphs:
            x.copy_(torch.randn_like(x))
            g.replay()
        torch.cuda.synchronize()
        for _, x, cc, cs in graphs:
            codes, scales = R.quantise(x.cpu().numpy().T)
            assert np.array_equal(cc.cpu().numpy(), codes) and np.array_equal(cs.cpu().numpy(), scales)


def test_two_graphs_that_share_the_workspace_of_sliced_sums():
    """Long sums of few tiles go in slices through a workspace; replayed in turn, with eager calls between."""
    ws, graphs = None, []
    rng = np.random.default_rng(8)
    for m, n, k, message in ((16, 256, 16384, False), (5, 70, 20000, True)):
        d = B.make_matmul8_desc(m=m, n=n, k=k, dtype="f32", message=message)
        need = B.matmul8_workspace_bytes(d)
        assert need > 0
        if ws is None or ws.numel() < need:
            ws = torch.empty(4 * need, dtype=torch.uint8, device="cuda")
        ops = [torch.from_numpy(v).cuda() for v in operands(rng, m, n, k, message)]
        out = torch.empty((m, n), device="cuda")
        B.matmul8(d, *ops, out, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.matmul8(d, *ops, out, workspace=ws)
        graphs.append((d, g, ops, out))
    for turn in range(4):
        for _, g, ops, out in graphs:
            ops[0].copy_(ops[0].flip(0) if turn % 2 else ops[0].roll(1, 0))
            out.fill_(float("nan"))
            g.replay()
        torch.cuda.synchronize()
        for d, _, ops, out in graphs:
            again = torch.empty_like(out)
            B.matmul8(d, *ops, again)
            off = 127.5 if d.message else 0.0
            k = d.k
            want = ((ops[0][:, :k].double() - off) @ ops[2][:, :k].double().t())
            want = want * (ops[1].double() / (127.5 if d.message else 127.0))[:, None] * (ops[3].double() / 127.0)[None, :]
            assert torch.equal(out, again)
            # the sum's rounding, two steps' and two products'
            assert ((out.double() - want).abs() <= 6 * R.U * want.abs()).all()


def test_workspaces_come_in_the_order_of_the_calls_stream():
    """What the binding allocates for a call on another stream is no memory that the current stream may still use."""
    side, need = torch.cuda.Stream(), 5 << 20
    torch.cuda.synchronize()
    mine = torch.empty(need, dtype=torch.uint8, device="cuda")
    at = mine.data_ptr()
    like = torch.empty(1, device="cuda")
    del mine
    given, _ = B._workspace(need, None, like, side)
    assert given.value != at
    again, _ = B._workspace(need, None, like, None)
    assert again.value == at
    x = torch.randn(300, 200, device="cuda")
    d = B.make_quant8_desc(rows=300, cols=200, dtype="f32")
    cc, cs = torch.empty((200, R.stride(300)), dtype=torch.int8, device="cuda"), torch.empty(200, device="cuda")
    torch.cuda.synchronize()
    B.quant8(d, x, col_codes=cc, col_scales=cs, stream=side)
    torch.cuda.synchronize()
    codes, scales = R.quantise(x.cpu().numpy().T)
    assert np.array_equal(cc.cpu().numpy(), codes) and np.array_equal(cs.cpu().numpy(), scales)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_tokens(dtype):
    """A micro-batch without a token: its columns' scales and sums are 0, and it adds nothing to a weight's gradient."""
    td = B.DTYPE_NAME[dtype]
    codes, scales, sums = {}, {}, {}
    for name, cols in (("x", 70), ("dy", 1300)):
        d = B.make_quant8_desc(rows=0, cols=cols, dtype=dtype)
        sc, su = (Framed((cols,), torch.float32) for _ in range(2))
        sc.t.fill_(float("nan")); su.t.fill_(float("nan"))
        codes[name] = torch.empty((cols, 0), dtype=torch.int8, device="cuda")
        B.quant8(d, torch.empty((0, cols), dtype=td, device="cuda"), row_codes=torch.empty((0, R.stride(cols)), dtype=torch.int8, device="cuda"),
                 row_scales=torch.empty(0, device="cuda"), col_codes=codes[name], col_scales=sc.t, col_sums=su.t)
        torch.cuda.synchronize()
        sc.check(name); su.check(name)
        assert (sc.t == 0).all() and (su.t == 0).all()
        scales[name] = sc.t
    grad = torch.randn(1300, 70, device="cuda")
    before = grad.clone()
    B.matmul8(B.make_matmul8_desc(m=1300, n=70, k=0, dtype="f32"), codes["dy"], scales["dy"], codes["x"], scales["x"], grad, add=grad)
    assert torch.equal(grad, before)
    rs = torch.full((5,), float("nan"), device="cuda")
    B.quant8(B.make_quant8_desc(rows=5, cols=0, dtype=dtype), torch.empty((5, 0), dtype=td, device="cuda"),
             row_codes=torch.empty((5, 0), dtype=torch.int8, device="cuda"), row_scales=rs)
    assert (rs == 0).all()


def test_the_native_path_gives_what_the_ctypes_one_does(monkeypatch):
    """The same bits by both ways of the binding, with and without a workspace, on the current and on a named stream."""
    m, k, f = 70, 128, 96
    inputs = stage_inputs(m, k, f, "f16")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    first = [stage_step(*inputs, "f16"), stage_step(*inputs, "f16", stream=side)]
    torch.cuda.synchronize()
    monkeypatch.setattr(B, "_native", B._Ctypes())
    second = [stage_step(*inputs, "f16"), stage_step(*inputs, "f16", stream=side)]
    torch.cuda.synchronize()
    for n, want in first[0].items():
        for got in (first[1], *second):
            assert torch.equal(got[n], want), n


def test_calls_of_two_threads_at_once():
    """Each thread its own stream and results; the library keeps nothing between them."""
    want = {}
    jobs = [(96, 64, 80), (130, 160, 112)]
    inputs = [stage_inputs(*j, "bf16", seed=i) for i, j in enumerate(jobs)]
    want = [{n: t.clone() for n, t in stage_step(*x, "bf16").items()} for x in inputs]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(8):
                    got[i].append(stage_step(*inputs[i], "bf16"))
            stream.synchronize()
        except Exception as e:                                              # told to the test's own thread
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for i in range(2):
        for r in got[i]:
            for n, t in want[i].items():
                assert torch.equal(r[n], t), n


def test_the_time_of_a_call_of_two_launches():
    """aqsgd_profile_next_launch around calls that take one launch and two."""
    x = torch.randn(4096, 1600, device="cuda")
    d = B.make_quant8_desc(rows=4096, cols=1600, dtype="f32")
    cc, cs = torch.empty((1600, 4096), dtype=torch.int8, device="cuda"), torch.empty(1600, device="cuda")
    dm = B.make_matmul8_desc(m=16, n=256, k=16384, dtype="f32")
    ops = [torch.from_numpy(v).cuda() for v in operands(np.random.default_rng(0), 16, 256, 16384)]
    out = torch.empty((16, 256), device="cuda")
    for call in (lambda: B.quant8(d, x, col_codes=cc, col_scales=cs), lambda: B.matmul8(dm, *ops, out)):
        call()
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record(); stop.record()                                       # makes the events
        torch.cuda.synchronize()
        B.profile_next_launch(start, stop)
        call()
        torch.cuda.synchronize()
        assert 0.001 < start.elapsed_time(stop) < 5.0


# ---- every kernel ------------------------------------------------------------------------------
# Sizes at which the choice takes each of the kernels of larger products, small ones as far as that goes: rows of results
# that are whole sectors of 32 bytes and others, columns and rows that end inside a tile, k that ends in either half of
# a step.  The 64-bit products are the device's own here; sums of codes are whole numbers, exact in them.

TILES = [(97, 4129, 1808), (161, 2816, 1264), (33, 4160, 224), (4125, 33, 160), (65, 5195, 176), (65, 5312, 176), (1803, 4369, 160),
         (1539, 5088, 144), (2327, 5615, 160), (2309, 5664, 224), (3093, 4901, 1008), (5447, 2848, 896), (3597, 5637, 240),
         (1283, 1632, 9456), (5401, 3979, 240), (5935, 3648, 240), (1281, 5989, 224), (1667, 4704, 208), (1539, 5913, 160), (1569, 5792, 176),
         (2821, 4095, 144), (2339, 4832, 160)]
GATED = [(4131, 49, 1856), (161, 1408, 1264), (33, 2077, 160), (33, 2080, 224), (65, 2533, 160), (67, 2560, 160), (1557, 2499, 160),
         (1797, 2240, 144), (2069, 2693, 176), (2311, 2464, 176), (5385, 1417, 976), (5941, 1312, 992), (4613, 2197, 256), (4651, 2208, 240),
         (1667, 2337, 192), (1671, 2368, 208)]


def device_codes(rows, k, gen):
    t = torch.zeros((rows, R.stride(k)), dtype=torch.int8, device="cuda")
    t[:, :k] = torch.randint(-127, 128, (rows, k), generator=gen, device="cuda", dtype=torch.int8)
    return t, torch.rand(rows, generator=gen, device="cuda") * 0.02 + 0.01


def device_projections(a, sa, b, sb, k, message=False):
    """R.projections on the device."""
    ai, bi = a[:, :k].double(), b[:, :k].double()
    steps = (sa.double() / (127.5 if message else 127.0))[:, None] * (sb.double() / 127.0)[None, :]
    if message:
        whole, ones = (ai - 128) @ bi.t().contiguous(), bi.sum(dim=1)[None, :]
        sums = whole + 0.5 * ones
        off = 5 * sums.abs() + 3 * (whole.abs() + 0.5 * ones.abs())
    else:
        sums = ai @ bi.t().contiguous()
        off = 5 * sums.abs()
    return sums * steps, off * R.U * steps


def device_act(x, kind):
    if kind == "silu":
        return x / (1.0 + torch.exp(-x))
    if kind == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x / 2 ** 0.5))
    return 0.5 * x * (1.0 + torch.tanh((2.0 / np.pi) ** 0.5 * (x + 0.044715 * x ** 3)))


def device_close(got, want, off, dtype, tag):
    """R.close on the device."""
    miss = (got.double() - want).abs() - 1.0001 * (off + R.HALF_STEP[dtype] * (want.abs() + off) + R.TINY[dtype])
    bad = ~(miss <= 0)
    assert not bad.any(), f"{tag}: {int(bad.sum())} of {bad.numel()} values too far off, first at {bad.nonzero()[0].tolist()}"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", TILES)
def test_products_by_every_kernel(dtype, m, n, k):
    """Plain, added to in place, of a message, and through an activation."""
    gen = torch.Generator(device="cuda").manual_seed(m * n + k)
    td, tag = B.DTYPE_NAME[dtype], f"{dtype} {m}x{n}x{k}"
    a, sa = device_codes(m, k, gen)
    b, sb = device_codes(n, k, gen)
    bias = torch.randn(n, generator=gen, device="cuda").to(td)
    out = Framed((m, n), td, 128)
    p, off = device_projections(a, sa, b, sb, k)
    d = B.make_matmul8_desc(m=m, n=n, k=k, dtype=dtype)
    B.matmul8(d, a, sa, b, sb, out.t, bias=bias)
    device_close(out.t, p + bias.double(), off + R.U * (p + bias.double()).abs(), dtype, tag)
    before = torch.randn((m, n), generator=gen, device="cuda").to(td)
    out.t.copy_(before)
    B.matmul8(d, a, sa, b, sb, out.t, add=out.t)
    want = p + before.double()
    device_close(out.t, want, off + R.U * want.abs(), dtype, tag + " added")
    act = ACTS[(m + n) % 3]
    h, pre = Framed((m, n), td, 128), Framed((m, n), td, 160)
    B.ffn8(B.make_ffn8_desc(m=m, f=n, k=k, dtype=dtype, act=act, gated=False), a, sa, b, sb, h.t, bias=bias, pre=pre.t)
    y = p + bias.double()
    yoff = off + R.U * y.abs()
    device_close(pre.t, y, yoff, dtype, tag + " pre")
    device_close(h.t, device_act(y, act), R.STEEPEST * yoff + R.VALUE_OFF * y.abs(), dtype, tag + " " + act)
    levels = torch.randint(0, 256, (m, k), generator=gen, device="cuda", dtype=torch.uint8)
    p, off = device_projections(levels, sa, b, sb, k, message=True)
    B.matmul8(B.make_matmul8_desc(m=m, n=n, k=k, dtype=dtype, message=True), levels, sa, b, sb, out.t)
    device_close(out.t, p, off, dtype, tag + " message")
    torch.cuda.synchronize()
    for f in (out, h, pre):
        f.check(tag)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,f,k", GATED)
def test_gated_blocks_by_every_kernel(dtype, m, f, k):
    gen = torch.Generator(device="cuda").manual_seed(m * f + k)
    td, act, tag = B.DTYPE_NAME[dtype], ACTS[(m + f) % 3], f"{dtype} {m}x{f}x{k}"
    a, sa = device_codes(m, k, gen)
    b, sb = device_codes(2 * f, k, gen)
    bias = torch.randn(2 * f, generator=gen, device="cuda").to(td)
    h, pre = Framed((m, f), td, 128), Framed((m, 2 * f), td, 128)
    B.ffn8(B.make_ffn8_desc(m=m, f=f, k=k, dtype=dtype, act=act), a, sa, b, sb, h.t, bias=bias, pre=pre.t)
    p, off = device_projections(a, sa, b, sb, k)
    p = p + bias.double()
    off = off + R.U * p.abs()
    device_close(pre.t, p, off, dtype, tag + " pre")
    g, goff = device_act(p[:, :f], act), R.STEEPEST * off[:, :f] + R.VALUE_OFF * p[:, :f].abs()
    u, uoff = p[:, f:], off[:, f:]
    device_close(h.t, g * u, g.abs() * uoff + u.abs() * goff + goff * uoff + R.U * (g * u).abs(), dtype, f"{tag} {act}")
    alone = torch.empty((m, f), dtype=td, device="cuda")
    B.ffn8(B.make_ffn8_desc(m=m, f=f, k=k, dtype=dtype, act=act), a, sa, b, sb, alone, bias=bias)
    assert torch.equal(alone, h.t)
    torch.cuda.synchronize()
    h.check(tag)
    pre.check(tag)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(863, 33, 19264), (1033, 1, 16704), (515, 1, 16560), (1, 1, 10496), (1, 1035, 16384), (33, 896, 19376),
                                   (35, 384, 16720)])
def test_long_sums_in_slices(dtype, m, n, k):
    assert B.matmul8_workspace_bytes(B.make_matmul8_desc(m=m, n=n, k=k, dtype=dtype)) > 0
    run_matmul8(m, n, k, dtype, bias=True, add=True, in_place=True)
    run_matmul8(m, n, k, dtype, message=True, workspace=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(65601, 3), (33001, 131), (262200, 3), (1048700, 1)])
def test_quant8_of_many_rows(dtype, rows, cols):
    """Tiles of 128 rows, one, two and eight to a workgroup."""
    x = activations(np.random.default_rng([rows, cols]), rows, cols)
    run_quant8(x, dtype)
    run_quant8(x, dtype, by_rows=False, sums=False, pad=cols % 2)
    if cols == 3:
        run_quant8(x, dtype, rounding=1, seed=rows)
        run_quant8(x, dtype, rounding=1, seed=rows, by_rows=False, sums=False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_quant8_draws_of_rows_or_columns_alone(dtype):
    for cols in (40, 200, 900, 1500, 5001, 12000, 20000):
        run_quant8(activations(np.random.default_rng(cols), 5, cols), dtype, rounding=1, seed=cols, by_cols=False, sums=False)
    run_quant8(activations(np.random.default_rng(1), 300, 150), dtype, rounding=1, seed=9, by_rows=False, sums=False)
    run_quant8(activations(np.random.default_rng(1), 300, 150), dtype, by_rows=False, sums=False)
    run_quant8(activations(np.random.default_rng(2), 700, 150), dtype, by_rows=True, by_cols=False)


# ---- the largest -------------------------------------------------------------------------------

def test_matmul8_of_more_rows_than_a_grid_of_small_tiles_counts():
    """2^29 tokens: codes and results whose offsets pass 32 bits, and more tiles of the small kernels than a grid takes."""
    m, n, k = (1 << 29) + 65, 16, 16
    if torch.cuda.mem_get_info()[0] < (120 << 30):
        pytest.skip("needs 80 GB")
    torch.manual_seed(0)
    b = torch.randint(-127, 128, (n, 64), dtype=torch.int8, device="cuda")
    b[:, k:] = 0
    sb = torch.rand(n, device="cuda") + 0.5
    a = torch.zeros((m, 64), dtype=torch.int8, device="cuda")
    period = torch.randint(-127, 128, (999983, k), dtype=torch.int8, device="cuda")
    for at in range(0, m, 999983):
        a[at:at + 999983, :k] = period[:min(999983, m - at)]
    sa = torch.rand(999983, device="cuda").repeat(m // 999983 + 1)[:m].contiguous()
    out = torch.empty((m, n), device="cuda")
    B.matmul8(B.make_matmul8_desc(m=m, n=n, k=k, dtype="f32"), a, sa, b, sb, out)
    torch.cuda.synchronize()
    # sums below 2^24 are exact in binary32, and the steps follow one by one (on the host: divided, not multiplied
    # with a reciprocal)
    want = (period.float().cpu() @ b[:, :k].float().cpu().t()) * (sa[:999983].cpu() / torch.tensor([127.0]))[:, None]
    want = (want * (sb.cpu() / torch.tensor([127.0]))[None, :]).cuda()
    for at in range(0, m, 999983):
        assert torch.equal(out[at:at + 999983], want[:min(999983, m - at)]), at
    del a, sa, out
    torch.cuda.empty_cache()


def test_quant8_sums_of_the_most_columns():
    """2^30 columns of 33 rows: more workgroups of a block of rows each than a grid takes."""
    rows, cols = 33, 1 << 30
    if torch.cuda.mem_get_info()[0] < (130 << 30):
        pytest.skip("needs 90 GB")
    line = ((torch.arange(1 << 24, device="cuda") % 61).half() - 30) / 8
    x = torch.empty((rows, cols), dtype=torch.float16, device="cuda")
    for r in range(rows):
        x[r].view(64, 1 << 24)[:] = line * (1 + r % 2)
    sums = torch.full((cols,), float("nan"), device="cuda")
    B.quant8(B.make_quant8_desc(rows=rows, cols=cols, dtype="f16"), x, col_sums=sums)
    torch.cuda.synchronize()
    want = line.float() * 49                                                # 17 rows once, 16 twice: exact
    for part in sums.view(64, 1 << 24):
        assert torch.equal(part, want)
    del x, sums
    torch.cuda.empty_cache()
