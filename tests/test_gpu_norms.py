"""Layer norm and its gradient on the GPU against their plain forms: statistics and results within the roundings that the
header lists, codes exactly those of the quantiser."""
import threading

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import norms_reference as N
import products8_reference as R
from paper_2206_01299_amd import binding as B
from test_gpu_products8 import DTYPES, MARK, Framed, activations, numbers, stored


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.fail("these tests need an MI355X")
    B.lib()


def typed(dtype):
    """binary32 values as the type holds them."""
    return lambda v: torch.from_numpy(v).to(B.DTYPE_NAME[dtype]).float().numpy()


def rows_inside(x, dtype, pad, offset):
    """A matrix as a view of wider rows, from any element on; and its values."""
    rows, cols = x.shape
    wide = torch.full((rows * (cols + pad) + offset,), 3.0, dtype=B.DTYPE_NAME[dtype], device="cuda")
    t = wide[offset:].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.from_numpy(np.asarray(x, dtype=np.float32)))
    return t, t.float().cpu().numpy()


def framed_vector(v, dtype):
    t, values = stored(v, dtype)
    f = Framed(tuple(t.shape), t.dtype)
    f.t.copy_(t)
    return f, values


def run_norm(x, dtype, residual=None, weight=None, bias=None, pad=0, offset=0, eps=1e-5, y=True, codes=True, stats=True, sum=True, place=None, lead=64):
    """One call against the plain form.  place: which output lies where an input does, as "sum=x" or "y=residual"."""
    rows, cols = x.shape
    td, tag = B.DTYPE_NAME[dtype], f"{dtype} {rows}x{cols} pad {pad} place {place} residual {residual is not None} weight {weight is not None}"
    size = torch.empty(0, dtype=td).element_size()
    lead = lead * size if lead != 64 else 64
    if place:
        fx = Framed((rows, cols), td, lead)
        fx.t.copy_(torch.from_numpy(np.asarray(x, np.float32)))
        tx, xf = fx.t, fx.t.float().cpu().numpy()
    else:
        tx, xf = rows_inside(x, dtype, pad, offset)
    res = wf = bf = None
    s = xf
    if residual is not None:
        res, rf = framed_vector(residual, dtype)
        s = N.stored_sum(xf, rf, typed(dtype))
    if weight is not None:
        w, wf = framed_vector(weight, dtype)
    if bias is not None:
        b, bf = framed_vector(bias, dtype)
    frames = {"sum": Framed((rows, cols), td, lead), "y": Framed((rows, cols), td, lead), "mean": Framed((rows,), torch.float32),
              "rstd": Framed((rows,), torch.float32), "row_codes": Framed((rows, R.stride(cols)), torch.int8), "row_scales": Framed((rows,), torch.float32)}
    on = {"sum": sum and residual is not None, "y": y, "mean": stats, "rstd": stats, "row_codes": codes, "row_scales": codes}
    if place:
        out, into = place.split("=")
        frames[out] = fx if into == "x" else res
    d = B.make_layernorm_desc(rows=rows, cols=cols, ld=cols + pad, dtype=dtype, eps=eps)
    B.layernorm(d, tx, residual=None if res is None else res.t, weight=None if wf is None else w.t, bias=None if bf is None else b.t,
                **{n: f.t if on[n] else None for n, f in frames.items()})
    torch.cuda.synchronize()
    for n, f in frames.items():
        f.check(f"{tag} {n}")
        if not on[n] and not (place and place.startswith(n)):
            assert (f.raw == MARK).all(), f"{tag}: {n} was not asked for"
    if on["sum"]:
        assert np.array_equal(frames["sum"].t.float().cpu().numpy(), s, equal_nan=True), f"{tag}: sum"
    want, off = N.mean_of(s)
    mean = frames["mean"].t.cpu().numpy() if stats else want.astype(np.float32)
    if stats:
        R.close(mean, want, off, "f32", tag + " mean")
    deviation, want, off = N.rstd_of(s, mean, eps)
    rstd = frames["rstd"].t.cpu().numpy() if stats else want.astype(np.float32)
    if stats:
        R.close(rstd, want, off, "f32", tag + " rstd")
    if y and stats:
        want, off = N.normalised(deviation, rstd, wf, bf)
        R.close(numbers(frames["y"].t), want, off, dtype, tag + " y")
    if codes and y:
        check_codes(frames, frames["y"].t, cols, tag)
    return frames


def check_codes(frames, y, cols, tag):
    want, scales = R.quantise(y.float().cpu().numpy())
    assert np.array_equal(frames["row_scales"].t.cpu().numpy(), scales, equal_nan=True), f"{tag}: scales"
    assert np.array_equal(frames["row_codes"].t.cpu().numpy(), want), f"{tag}: codes"


def inputs(rows, cols, seed=0):
    rng = np.random.default_rng([rows, cols, seed])
    return (activations(rng, rows, cols), rng.standard_normal((rows, cols)), 1 + 0.1 * rng.standard_normal(cols), 0.1 * rng.standard_normal(cols))


SIZES = [(1, 1), (7, 3), (5, 4), (4, 7), (3, 8), (9, 9), (70, 24), (33, 63), (33, 64), (33, 65), (17, 127), (70, 128), (65, 129), (40, 256),
         (300, 257), (17, 511), (130, 512), (9, 513), (41, 1000), (9, 1024), (8, 1025), (1, 1600), (257, 1600), (40, 1537), (9, 2048), (12, 2049),
         (6, 4096), (9, 4097), (6, 8191), (5, 8200), (3, 16384), (3, 16385), (2, 32768), (2, 33000), (2, 65600), (3, 70001), (5000, 40)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_layernorm(dtype, rows, cols):
    x, res, w, b = inputs(rows, cols)
    run_norm(x, dtype, residual=res, weight=w, bias=b)
    run_norm(x, dtype, weight=w, bias=b, pad=1 + rows % 9, offset=1)
    full = run_norm(x, dtype, bias=b, pad=8, codes=False)
    alone = run_norm(x, dtype, bias=b, y=False, stats=False)                   # codes of a result that is not stored
    check_codes(alone, full["y"].t, cols, f"{dtype} {rows}x{cols} codes alone")
    run_norm(x, dtype, residual=res, weight=w, sum=False, lead=1)
    plain = run_norm(x, dtype)
    for place in ("sum=x", "sum=residual", "y=x", "y=residual"):
        got = run_norm(x, dtype, residual=res, weight=w, bias=b, place=place, sum=not place.startswith("y") or rows % 2 == 0)
        del got
    again = run_norm(x, dtype, stats=False, codes=False)
    assert torch.equal(again["y"].t.view(torch.uint8), plain["y"].t.view(torch.uint8))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [5, 24, 300, 1600, 5000, 20000, 70001])
def test_layernorm_of_what_is_no_ordinary_row(dtype, cols):
    """Constant rows, the largest values, subnormals, a mean far above the deviation, infinities and NaN: a row of the
    latter is NaN with codes of zero, its neighbours are as without it."""
    big = {"f16": 65504.0, "bf16": 3.3895e38, "f32": 3.4028e38}[dtype]
    tiny = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}[dtype]
    rng = np.random.default_rng(cols)
    x, w, b = rng.standard_normal((12, cols)), 1 + 0.1 * rng.standard_normal(cols), 0.1 * rng.standard_normal(cols)
    x[0] = 0.0
    x[1] = 3.0
    x[2] = np.where(np.arange(cols) % 2, big, -big)
    x[3] *= 4 * tiny
    x[4] += 1000.0
    run_norm(x, dtype, weight=w, bias=b)
    run_norm(x, dtype, eps=0.0, weight=w) if cols > 1 else None
    clean = run_norm(x, dtype, weight=w, bias=b)["y"].t.clone()
    x[6, cols // 2], x[7, 0], x[8, cols - 1] = np.inf, np.nan, -np.inf
    x[9, 0], x[9, 1] = np.inf, -np.inf
    y = run_norm(x, dtype, weight=w, bias=b)["y"].t
    assert torch.isnan(y[6:10]).all()
    for rows in (slice(0, 6), slice(10, 12)):                                  # bytes: in binary32 the largest values' deviations overflow
        assert torch.equal(y[rows].view(torch.uint8), clean[rows].view(torch.uint8))


def test_layernorm_of_no_rows():
    t = torch.empty((0, 40), device="cuda")
    B.layernorm(B.make_layernorm_desc(rows=0, cols=40, dtype="f32"), t, y=t, mean=torch.empty(0, device="cuda"), rstd=torch.empty(0, device="cuda"))


# ---- backward ----------------------------------------------------------------------------------

def run_grad(rows, cols, dtype, weight=True, add=False, accumulate=False, pad=0, offset=0, dw=True, db=True, place=None, workspace=True, seed=0, lead=64):
    td, tag = B.DTYPE_NAME[dtype], f"{dtype} {rows}x{cols} pad {pad} add {add} accumulate {accumulate} place {place}"
    rng = np.random.default_rng([rows, cols, seed, 1])
    size = torch.empty(0, dtype=td).element_size()
    lead = lead * size if lead != 64 else 64
    tx, x = rows_inside(activations(rng, rows, cols), dtype, pad, offset)
    mean, _ = N.mean_of(x)
    mean = mean.astype(np.float32)
    rstd = N.rstd_of(x, mean, 1e-5)[1].astype(np.float32)
    fdy = Framed((rows, cols), td, lead)
    fdy.t.copy_(torch.from_numpy(1e-2 * rng.standard_normal((rows, cols))))
    dy = fdy.t.float().cpu().numpy()
    fadd, af = framed_vector(1e-2 * rng.standard_normal((rows, cols)), dtype) if add else (None, None)
    fw, wf = framed_vector(1 + 0.1 * rng.standard_normal(cols), dtype) if weight else (None, None)
    before = rng.standard_normal((2, cols)).astype(np.float32)
    sums = [Framed((cols,), torch.float32) for _ in range(2)]
    for f, v in zip(sums, before):
        f.t.copy_(torch.from_numpy(v))
    dx = {"dy": fdy, "add": fadd, None: Framed((rows, cols), td, lead)}[place]
    d = B.make_layernorm_desc(rows=rows, cols=cols, ld=cols + pad, dtype=dtype, accumulate=accumulate)
    ws = Framed((B.layernorm_grad_workspace_bytes(d),), torch.uint8)
    B.layernorm_grad(d, fdy.t, tx, torch.from_numpy(mean).cuda(), torch.from_numpy(rstd).cuda(), dx.t, weight=fw.t if weight else None,
                     add=fadd.t if add else None, dweight=sums[0].t if dw else None, dbias=sums[1].t if db else None,
                     workspace=ws.t if workspace else None)
    torch.cuda.synchronize()
    for f in (dx, ws, *sums):
        f.check(tag)
    want = N.norm_grad(dy, x, mean, rstd, wf, af)
    R.close(numbers(dx.t), *want[0], dtype, tag + " dx")
    for f, on, (w, off), v, name in zip(sums, (dw, db), want[1:], before, ("dweight", "dbias")):
        got = f.t.cpu().numpy()
        if not on:
            assert np.array_equal(got, v), f"{tag}: {name} was not asked for"
            continue
        if accumulate:
            w, off = R.plus(w, off + N.U * np.abs(w), v.astype(np.float64))
        R.close(got, w, off, "f32", f"{tag} {name}")
    return dx.t, sums[0].t, sums[1].t


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_layernorm_grad(dtype, rows, cols):
    run_grad(rows, cols, dtype, add=True)
    run_grad(rows, cols, dtype, accumulate=True, pad=1 + rows % 9, offset=1, lead=1)
    run_grad(rows, cols, dtype, weight=False, pad=8, db=False)
    run_grad(rows, cols, dtype, add=True, dw=False, db=False, place="add")
    run_grad(rows, cols, dtype, add=True, dw=False, place="dy", workspace=False)
    for place in (None, "dy"):
        first = [t.clone() for t in run_grad(rows, cols, dtype, add=True, place=place)]
        for a, b in zip(first, run_grad(rows, cols, dtype, add=True, place="add" if place is None else place)):
            assert torch.equal(a, b)                                           # the same bits on every call


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 40), (2, 1600), (15, 1600), (16, 130), (511, 64), (513, 1600), (1025, 40), (1024, 700), (1025, 1001), (2049, 200), (4100, 1600), (1030, 4096),
                                       (1027, 8191), (1500, 130), (2000, 3001), (1025, 8200), (1100, 3), (70000, 24), (20000, 300)])
def test_layernorm_grad_by_rows(dtype, rows, cols):
    run_grad(rows, cols, dtype, add=rows % 2 == 0, accumulate=rows % 3 == 0)
    run_grad(rows, cols, dtype, add=rows % 2 == 1, place="dy", weight=rows % 3 == 0)


def test_layernorm_grad_of_no_rows():
    """Nothing adds to the sums: they are 0, or stay."""
    z = torch.empty((0, 70), device="cuda")
    none = torch.empty(0, device="cuda")
    for accumulate, want in ((False, 0.0), (True, 5.0)):
        dw, db = torch.full((70,), 5.0, device="cuda"), torch.full((70,), 5.0, device="cuda")
        B.layernorm_grad(B.make_layernorm_desc(rows=0, cols=70, dtype="f32", accumulate=accumulate), z, z, none, none, z, dweight=dw, dbias=db)
        assert (dw == want).all() and (db == want).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [40, 1600, 9000])
def test_layernorm_grad_keeps_a_bad_row_to_itself(dtype, cols):
    """A NaN in one row's gradient is in that row of dx and in its column's sums, nowhere else."""
    rows, bad = 33, 5
    rng = np.random.default_rng(cols)
    x, dy = (torch.from_numpy(rng.standard_normal((rows, cols))).cuda().to(B.DTYPE_NAME[dtype]) for _ in range(2))
    d = B.make_layernorm_desc(rows=rows, cols=cols, dtype=dtype)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.layernorm(d, x, mean=mean, rstd=rstd)
    got = []
    for spoil in (False, True):
        if spoil:
            dy[bad, 7] = float("nan")
        dx, dw, db = torch.empty_like(dy), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        B.layernorm_grad(d, dy, x, mean, rstd, dx, dweight=dw, dbias=db)
        got.append((dx, dw, db))
    assert torch.isnan(got[1][0][bad]).all()
    rest, others = torch.arange(rows, device="cuda") != bad, torch.arange(cols, device="cuda") != 7
    assert torch.equal(got[0][0][rest], got[1][0][rest])
    for a, b in zip(got[0][1:], got[1][1:]):
        assert torch.isnan(b[7]) and torch.equal(a[others], b[others])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(20, 9), (20, 33), (20, 1537), (1100, 9), (1100, 33), (1100, 1537), (1100, 40), (9, 5000), (5, 40000), (5, 70001)])
def test_layernorm_grad_of_constant_rows_of_large_values(dtype, rows, cols):
    """Every deviation is 0, and so is xh; what is formed where a row has no column must not overflow into its sums."""
    x = torch.full((rows, cols), 2.0 ** 127, device="cuda").to(B.DTYPE_NAME[dtype])
    dy = torch.ones((rows, cols), device="cuda").to(B.DTYPE_NAME[dtype])
    dy[:, 0] = 2.0
    d = B.make_layernorm_desc(rows=rows, cols=cols, dtype=dtype)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    y = torch.empty_like(x)
    B.layernorm(d, x, y=y, mean=mean, rstd=rstd)
    assert (mean == 2.0 ** 127).all() and not y.any()
    dx, dw, db = torch.empty_like(dy), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    for sums in (True, False):
        B.layernorm_grad(d, dy, x, mean, rstd, dx, dweight=dw if sums else None, dbias=db if sums else None)
        want = rstd.double()[:, None] * (dy.double() - dy.double().mean(dim=1, keepdim=True))
        # a mean of ones and a two: exact but for its product with 1 / cols, two half steps of about 1, times rstd
        allow = 4 * N.U * rstd.double()[:, None] + 1.01 * R.HALF_STEP[dtype] * want.abs()
        assert ((dx.double() - want).abs() <= allow).all()
    assert not dw.any() and (db[1:] == rows).all() and db[0] == 2 * rows


def test_layernorm_grad_is_the_differences_of_the_norm():
    """In float32: each loss is a sum of 10 x 24 results, differences over 2^-6 steps."""
    rows, cols, h = 10, 24, 2.0 ** -6
    rng = np.random.default_rng(3)
    x, dy, w, b = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in ((rows, cols), (rows, cols), cols, cols))
    d = B.make_layernorm_desc(rows=rows, cols=cols, dtype="f32")

    def loss(x, w, b):
        y = torch.empty((rows, cols), device="cuda")
        B.layernorm(d, x, weight=w, bias=b, y=y)
        return (y.double() * dy.double()).sum(dim=1) if x.dim() == 2 else None

    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.layernorm(d, x, mean=mean, rstd=rstd)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    B.layernorm_grad(d, dy, x, mean, rstd, dx, weight=w, dweight=dw, dbias=db)
    # roundings: results below 8, half a step each, 24 of them, over h; the third derivative's share is h^2 times some tens
    allow = 24 * 8 * N.U * 8 / h + 40 * h * h
    for c in range(cols):                                                      # a column at a time: rows do not mix
        e = torch.zeros_like(x)
        e[:, c] = h
        assert ((loss(x + e, w, b) - loss(x - e, w, b)) / (2 * h) - dx[:, c].double()).abs().max() < allow
        for i, (at, got) in enumerate(((w, dw), (b, db))):
            e = torch.zeros_like(at)
            e[c] = h
            more, less = (loss(x, *((at + s * e, b) if i == 0 else (w, at + s * e))).sum() for s in (1, -1))
            assert abs((more - less) / (2 * h) - got[c].double()) < rows * allow


# ---- every kernel ------------------------------------------------------------------------------
# Sizes at which the choice takes each of the kernels: pieces of 16 bytes a row, and rows; with whole pieces and with a
# last one that is not.

PIECES = {"f32": 4, "f16": 8, "bf16": 8}
NORMS = [(7, 5), (16, 40), (30, 9), (64, 7), (100, 9), (190, 600), (250, 600), (200, 5), (500, 3), (700, 3), (1000, 3), (2000, 2), (2900, 2), (4000, 2),
         (1500, 300), (2000, 300), (7, 4100), (15, 4100), (22, 4100), (30, 4100), (45, 4100), (60, 4100), (90, 4100), (120, 4100)]
GRADS = [(10, 1100), (30, 1100), (64, 1100), (100, 1100), (200, 1100), (400, 1100), (1000, 1100), (60, 20), (200, 20), (128, 300), (150, 300), (250, 300), (500, 5),
         (900, 5), (1500, 5), (2048, 4), (4000, 3), (3, 300), (25, 700), (64, 1024), (1024, 6), (1024, 140), (1100, 130),
         (10, 1409), (30, 1409), (64, 1500), (200, 1500), (400, 1409), (600, 2049), (600, 1409)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pieces,rows", NORMS)
def test_norms_by_every_kernel(dtype, pieces, rows):
    for less in (0, 1, PIECES[dtype] // 2):
        cols = pieces * PIECES[dtype] - less
        x, res, w, b = inputs(rows, cols)
        run_norm(x, dtype, residual=res, weight=w, bias=b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pieces,rows", GRADS)
def test_gradients_by_every_kernel(dtype, pieces, rows):
    for less in (0, 1, PIECES[dtype] // 2):
        cols = pieces * PIECES[dtype] - less
        run_grad(rows, cols, dtype, add=less > 0, accumulate=less != 1)
        run_grad(rows, cols, dtype, dw=False, db=False, add=True)


# ---- streams, graphs, threads, both ways of the binding ----------------------------------------

def block(x, res, dy, w, b, dtype, buf=None, stream=None):
    """Forward and backward pass, into buffers that are kept."""
    buf = {} if buf is None else buf
    rows, cols = x.shape
    td = B.DTYPE_NAME[dtype]
    d = B.make_layernorm_desc(rows=rows, cols=cols, dtype=dtype)

    def get(name, shape, t):
        if name not in buf:
            buf[name] = torch.zeros(shape, dtype=t, device="cuda")
        return buf[name]

    f = torch.float32
    out = {n: get(n, s, t) for n, s, t in (("sum", (rows, cols), td), ("y", (rows, cols), td), ("mean", (rows,), f), ("rstd", (rows,), f),
                                           ("row_codes", (rows, R.stride(cols)), torch.int8), ("row_scales", (rows,), f))}
    B.layernorm(d, x, residual=res, weight=w, bias=b, **out, stream=stream)
    back = {n: get(n, s, t) for n, s, t in (("dx", (rows, cols), td), ("dw", (cols,), f), ("db", (cols,), f))}
    B.layernorm_grad(d, dy, out["sum"], out["mean"], out["rstd"], back["dx"], weight=w, add=dy, dweight=back["dw"], dbias=back["db"],
                     stream=stream)
    return {**out, **back}


def block_inputs(rows, cols, dtype, seed=0):
    rng = np.random.default_rng([rows, cols, seed])
    return [stored(v, dtype)[0] for v in (activations(rng, rows, cols), rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols)),
                                          1 + 0.1 * rng.standard_normal(cols), 0.1 * rng.standard_normal(cols))]


@pytest.mark.parametrize("rows,cols", [(300, 200), (65, 1600), (40, 9000), (5, 70001)])
def test_streams_and_graphs(rows, cols):
    first = block_inputs(rows, cols, "bf16")
    plain = {n: t.clone() for n, t in block(*first, "bf16").items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = block(*first, "bf16")
    named = block(*first, "bf16", stream=side)
    torch.cuda.synchronize()
    for n in plain:
        assert torch.equal(plain[n], other[n]) and torch.equal(plain[n], named[n]), n
    buf, g = {}, torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        block(*first, "bf16", buf)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        out = block(*first, "bf16", buf)
    for seed in (0, 1, 2, 1):
        new = block_inputs(rows, cols, "bf16", seed)
        want = {n: t.clone() for n, t in block(*new, "bf16").items()}
        for a, b in zip(first, new):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(out[n], want[n]), f"replay with inputs {seed}: {n}"


def test_two_graphs_that_share_a_workspace():
    graphs = []
    shapes = [(300, 200), (1000, 1600)]
    ws = torch.empty(max(B.layernorm_grad_workspace_bytes(B.make_layernorm_desc(rows=r, cols=c, dtype="f32")) for r, c in shapes),
                     dtype=torch.uint8, device="cuda")
    for r, c in shapes:
        x, _, dy, w, _ = block_inputs(r, c, "f32")
        d = B.make_layernorm_desc(rows=r, cols=c, dtype="f32")
        mean, rstd = torch.empty(r, device="cuda"), torch.empty(r, device="cuda")
        B.layernorm(d, x, mean=mean, rstd=rstd)
        out = [torch.empty_like(dy), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")]
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            B.layernorm_grad(d, dy, x, mean, rstd, out[0], weight=w, dweight=out[1], dbias=out[2], workspace=ws)
        graphs.append((g, d, dy, x, mean, rstd, w, out))
    for _ in range(3):
        for g, d, dy, *_ in graphs:
            dy.copy_(torch.randn_like(dy))
            g.replay()
        torch.cuda.synchronize()
        for g, d, dy, x, mean, rstd, w, out in graphs:
            again = [torch.empty_like(t) for t in out]
            B.layernorm_grad(d, dy, x, mean, rstd, again[0], weight=w, dweight=again[1], dbias=again[2])
            for a, b in zip(out, again):
                assert torch.equal(a, b)


def test_the_native_path_gives_what_the_ctypes_one_does(monkeypatch):
    first = block_inputs(70, 130, "f16")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [block(*first, "f16"), block(*first, "f16", stream=side)]
    torch.cuda.synchronize()
    monkeypatch.setattr(B, "_native", B._Ctypes())
    got += [block(*first, "f16"), block(*first, "f16", stream=side)]
    torch.cuda.synchronize()
    for n, want in got[0].items():
        for other in got[1:]:
            assert torch.equal(other[n], want), n


def test_calls_of_two_threads_at_once():
    shapes = [(96, 1600), (130, 160)]
    first = [block_inputs(*s, "bf16", seed=i) for i, s in enumerate(shapes)]
    want = [{n: t.clone() for n, t in block(*x, "bf16").items()} for x in first]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(8):
                    got[i].append(block(*first[i], "bf16"))
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


def test_rows_whose_offsets_pass_32_bits():
    """2^20 rows of 2304 columns: the last ones are as a call on them alone gives."""
    rows, cols = 1 << 20, 2304
    if torch.cuda.mem_get_info()[0] < (60 << 30):
        pytest.skip("needs 40 GB")
    d = B.make_layernorm_desc(rows=rows, cols=cols, dtype="f16")
    x = torch.randn((1024, cols), device="cuda").half().repeat(1024, 1)
    x[-3:] *= 2
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.layernorm(d, x, y=y, mean=mean, rstd=rstd)
    few = B.make_layernorm_desc(rows=3, cols=cols, dtype="f16")
    y3, m3, r3 = torch.empty_like(y[-3:]), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    B.layernorm(few, x[-3:], y=y3, mean=m3, rstd=r3)
    assert torch.equal(y[-3:], y3) and torch.equal(mean[-3:], m3) and torch.equal(rstd[-3:], r3)
    dx3 = torch.empty_like(y3)
    B.layernorm_grad(few, y3, x[-3:], m3, r3, dx3)
    B.layernorm_grad(d, y, x, mean, rstd, y)
    assert torch.equal(y[-3:], dx3)
    del x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("cols", [3, 8])
def test_more_rows_than_a_grid_has_teams(cols):
    """70 million short rows, a period of 999983 again and again: every period's results are the first one's."""
    period, rows = 999983, 70_000_000
    d = B.make_layernorm_desc(rows=rows, cols=cols, dtype="f16")
    x = torch.randn((period, cols), device="cuda").half().repeat(rows // period + 1, 1)[:rows].contiguous()
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.layernorm(d, x, y=y, mean=mean, rstd=rstd)
    few = B.make_layernorm_desc(rows=period, cols=cols, dtype="f16")
    y1, m1, r1, dx1 = torch.empty_like(x[:period]), torch.empty(period, device="cuda"), torch.empty(period, device="cuda"), torch.empty_like(x[:period])
    B.layernorm(few, x[:period], y=y1, mean=m1, rstd=r1)
    dx, dw = torch.empty_like(x), torch.empty(cols, device="cuda")
    B.layernorm_grad(few, x[:period], x[:period], m1, r1, dx1)
    B.layernorm_grad(d, x, x, mean, rstd, dx)
    for at in range(0, rows, period):
        n = min(period, rows - at)
        assert torch.equal(y[at:at + n], y1[:n]) and torch.equal(dx[at:at + n], dx1[:n]) and torch.equal(mean[at:at + n], m1[:n]), at
    again = torch.empty_like(x)
    B.layernorm_grad(d, x, x, mean, rstd, again, dbias=dw)
    assert torch.equal(again, dx) or cols == 8                                # by blocks the sums are formed in another order
    want, size = x.double().sum(dim=0), x.double().abs().sum(dim=0)
    assert ((dw.double() - want).abs() <= (128 + rows // 128 + 64) * N.U * size).all()
    del x, y, dx
    torch.cuda.empty_cache()


def test_the_time_of_a_call_of_two_launches():
    """aqsgd_profile_next_launch around calls that take one launch and two."""
    x, _, dy, w, _ = block_inputs(4096, 1600, "f16")
    d = B.make_layernorm_desc(rows=4096, cols=1600, dtype="f16")
    mean, rstd = torch.empty(4096, device="cuda"), torch.empty(4096, device="cuda")
    dx, dw = torch.empty_like(dy), torch.empty(1600, device="cuda")
    for call in (lambda: B.layernorm(d, x, y=dx, mean=mean, rstd=rstd), lambda: B.layernorm_grad(d, dy, x, mean, rstd, dx, dweight=dw),
                 lambda: B.layernorm_grad(d, dy, x, mean, rstd, dx)):
        call()
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record(); stop.record()                                       # makes the events
        torch.cuda.synchronize()
        B.profile_next_launch(start, stop)
        call()
        torch.cuda.synchronize()
        assert 0.001 < start.elapsed_time(stop) < 5.0
