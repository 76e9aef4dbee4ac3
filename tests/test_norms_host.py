"""Layer norm, AdamW and the gradients' norm as far as the host sees them: sizes, refusals before any launch, and the plain
forms that the GPU tests compare with."""
import ctypes
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import norms_reference as N
import products8_reference as R
from paper_2206_01299_amd import binding as B

OK = ctypes.c_void_p(4096)            # never followed
NULL = None


def ln(d, x=OK, res=OK, w=OK, b=OK, sum=ctypes.c_void_p(8192), y=ctypes.c_void_p(16384), mean=OK, rstd=OK, codes=OK, scales=OK):
    return B.lib().aqsgd_layernorm(ctypes.byref(d) if d else None, x, res, w, b, sum, y, mean, rstd, codes, scales, None)


def lg(d, dy=OK, x=OK, mean=OK, rstd=OK, w=OK, add=OK, dx=OK, dw=OK, db=OK, ws=OK, n=1 << 40):
    return B.lib().aqsgd_layernorm_grad(ctypes.byref(d) if d else None, dy, x, mean, rstd, w, add, dx, dw, db, ws, n, None)


def tensors(*entries, **change):
    array = (B.AdamwTensor * max(1, len(entries)))()
    for e, n in zip(array, entries):
        e.param, e.grad, e.state, e.master, e.n, e.weight_decay = 4096, 4096, 4096, None, n, 0.0
        for k, v in change.items():
            setattr(e, k, v)
    return array, len(entries)


def aw(d, listed, lr=NULL, step=NULL, scale=NULL):
    return B.lib().aqsgd_adamw(ctypes.byref(d) if d else None, listed[0], listed[1], lr, step, scale, None)


def gn(listed, dtype=0, most=1.0, loss=NULL, result=OK, ws=OK, n=1 << 40):
    return B.lib().aqsgd_grad_norm(dtype, listed[0], listed[1], most, loss, result, ws, n, None)


def test_descriptors_match_the_header():
    assert ctypes.sizeof(B.LayernormDesc) == 40 and B.LayernormDesc.eps.offset == 32
    assert ctypes.sizeof(B.AdamwTensor) == 48 and B.AdamwTensor.weight_decay.offset == 40
    assert ctypes.sizeof(B.AdamwDesc) == 64 and B.AdamwDesc.rng_seed.offset == 56 and B.AdamwDesc.state_bits.offset == 48


BAD_ROWS = [(dict(rows=-1), -5), (dict(rows=2 ** 31), -5), (dict(cols=0), -5), (dict(cols=2 ** 25, ld=2 ** 25), -5), (dict(ld=39), -5),
            (dict(ld=2 ** 62), -5), (dict(rows=2 ** 30, ld=2 ** 39), -5), (dict(dtype=3), -4), (dict(eps=-1e-9), -5),
            (dict(eps=float("nan")), -5), (dict(eps=float("inf")), -5), (dict(accumulate=2), -5)]


def row_desc(**change):
    d = B.make_layernorm_desc(rows=16, cols=40, dtype="f16")
    for name, v in change.items():
        setattr(d, name, v)
    return d


def test_layernorm_refusals():
    d = row_desc()
    assert ln(None) == -1
    for change, status in BAD_ROWS:
        assert ln(row_desc(**change)) == status, change
    assert ln(row_desc(rows=0), *[None] * 10) == 0
    for lack in (dict(x=NULL), dict(res=NULL), dict(mean=NULL), dict(rstd=NULL), dict(codes=NULL), dict(scales=NULL)):
        assert ln(d, **lack) == -1, lack
    for name in ("x", "res", "w", "b", "sum", "y"):
        assert ln(d, **{name: ctypes.c_void_p(4097)}) == -6, name
    for name in ("mean", "rstd", "scales"):
        assert ln(d, **{name: ctypes.c_void_p(4098)}) == -6, name
    assert ln(d, codes=ctypes.c_void_p(4104)) == -6
    assert ln(d, sum=OK, y=OK) == -5                                            # one for the other
    wide = row_desc(ld=48)
    assert ln(wide, res=ctypes.c_void_p(256), sum=OK) == -5 and ln(wide, res=ctypes.c_void_p(256), y=OK) == -5
    assert ln(d, sum=NULL, y=NULL, mean=NULL, rstd=NULL, codes=NULL, scales=NULL) == 0      # nothing asked for


def test_layernorm_grad_refusals():
    d = row_desc(rows=4096)
    need = B.layernorm_grad_workspace_bytes(d)
    assert need > 0 and lg(None) == -1
    for change, status in BAD_ROWS:
        assert lg(row_desc(**change)) == status, change
        assert B.layernorm_grad_workspace_bytes(row_desc(**change)) == 0
    assert lg(row_desc(rows=0), dw=NULL, db=NULL, dy=NULL, x=NULL, dx=NULL) == 0
    for name in ("dy", "x", "mean", "rstd", "dx"):
        assert lg(d, **{name: NULL}) == -1, name
    for name, at in (("dy", 4097), ("x", 4097), ("w", 4097), ("add", 4097), ("dx", 4097), ("mean", 4098), ("rstd", 4098),
                     ("dw", 4098), ("db", 4098), ("ws", 4104)):
        assert lg(d, **{name: ctypes.c_void_p(at)}) == -6, name
    assert lg(d, ws=NULL) == -9 and lg(d, n=need - 1) == -9
    assert lg(d, dx=OK, x=OK) == -5 and lg(row_desc(), dx=OK, x=OK, dw=NULL, db=NULL) == -5      # in x's place
    for few in (row_desc(), row_desc(rows=4096, cols=2 ** 20, ld=2 ** 20)):             # no block's sums to join
        assert B.layernorm_grad_workspace_bytes(few) == 0


def test_adamw_refusals():
    make = lambda **kw: B.make_adamw_desc(dtype="f16", grad_dtype="f32", **kw)  # noqa: E731
    one = tensors(40)
    assert aw(None, one) == -1
    for change, status in ((dict(state_bits=16), -2), (dict(rounding=2), -4), (dict(step=0), -5), (dict(lr=-1e-3), -5),
                           (dict(lr=math.nan), -5), (dict(lr=math.inf), -5), (dict(eps=-1.0), -5), (dict(beta1=1.0), -5), (dict(beta1=-0.1), -5),
                           (dict(beta2=1.5), -5), (dict(beta2=math.nan), -5)):
        assert aw(make(**change), one) == status, change
        assert B.adamw_state_bytes(make(**change), 40) == 0
    bad = make()
    for name, v, status in (("dtype", 3, -4), ("grad_dtype", 3, -4), ("grad_dtype", 2, -4)):
        bad = make()
        setattr(bad, name, v)
        assert aw(bad, one) == status
    d = make()
    assert aw(d, (one[0], -1)) == -5 and aw(d, (None, 1)) == -1
    assert aw(d, (None, 0)) == 0 and aw(d, tensors()) == 0 and aw(d, tensors(0, 0, param=None, grad=None, state=None)) == 0
    assert aw(d, tensors(-1)) == -5 and aw(d, tensors((1 << 34) + 1)) == -5
    for name in ("param", "grad", "state"):
        assert aw(d, tensors(40, **{name: None})) == -1, name
    for name, at in (("param", 4097), ("grad", 4098), ("state", 4104), ("master", 4098)):
        assert aw(d, tensors(40, **{name: at})) == -6, name
    for decay in (-0.1, math.nan, math.inf):
        assert aw(d, tensors(40, weight_decay=decay)) == -5
    mixed = tensors(40, 40)
    mixed[0][1].master = 4096
    assert aw(d, mixed) == -1
    mixed[0][0].master, mixed[0][1].master = 4096, None
    assert aw(d, mixed) == -1
    assert aw(B.make_adamw_desc(dtype="f32"), tensors(40, master=4096)) == -1
    assert aw(d, one, lr=ctypes.c_void_p(4098)) == -6 and aw(d, one, step=ctypes.c_void_p(4100)) == -6 and aw(d, one, scale=ctypes.c_void_p(4098)) == -6


def test_grad_norm_refusals():
    one = tensors(40)
    assert gn(one, dtype=3) == -4 and gn((one[0], -1)) == -5 and gn((None, 1)) == -1 and gn(tensors(-1)) == -5
    assert gn(one, most=-1.0) == -5 and gn(one, most=math.nan) == -5
    assert gn(one, result=NULL) == -1 and gn(tensors(40, grad=None)) == -1
    assert gn(tensors(40, grad=4098)) == -6 and gn(one, loss=ctypes.c_void_p(4098)) == -6 and gn(one, result=ctypes.c_void_p(4098)) == -6
    need = B.lib().aqsgd_grad_norm_workspace_bytes(*one)
    assert need >= 8 and gn(one, ws=NULL) == -9 and gn(one, n=need - 1) == -9 and gn(one, ws=ctypes.c_void_p(4104)) == -6
    assert B.lib().aqsgd_grad_norm_workspace_bytes(None, 0) == 0 and B.lib().aqsgd_grad_norm_workspace_bytes(*tensors(0)) == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_states(bits):
    d = B.make_adamw_desc(dtype="f32", state_bits=bits)
    for n in (0, 1, 15, 16, 17, 63, 64, 65, 255, 256, 257, 4097):
        assert B.adamw_state_bytes(d, n) == N.state_bytes(n, bits)
        state = torch.zeros(N.state_bytes(n, bits), dtype=torch.uint8)
        views = B.adamw_state_views(d, state, n)
        for k, (view, like) in enumerate(zip(views, N.State(n, bits).parts())):
            assert view.numel() == len(like) and str(view.dtype).split(".")[1] == str(like.dtype)
            assert n == 0 or view.data_ptr() % 64 == state.data_ptr() % 64
            view.fill_(k + 1)
        for k, view in enumerate(views):                                        # none lies in another
            assert (view == k + 1).all()
    assert B.adamw_state_bytes(d, -1) == 0 and B.adamw_state_bytes(d, 1 << 40) == 0
    with pytest.raises(ValueError):
        B.adamw_state_views(d, torch.zeros(64, dtype=torch.uint8), 100)


@pytest.fixture
def host_tensors(monkeypatch):
    """Host tensors stand in for device ones: addresses are taken, nothing is called with them."""
    monkeypatch.setattr(B, "_dev", lambda t, what: ctypes.c_void_p(t.data_ptr()))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    monkeypatch.setattr(B, "_stream", lambda s: ctypes.c_void_p(0))


def test_a_list_of_tensors_is_checked_when_it_is_made(host_tensors):
    z = torch.zeros
    d = B.make_adamw_desc(dtype="f16", grad_dtype="f32", state_bits=8)
    state = lambda n: z(B.adamw_state_bytes(d, n), dtype=torch.uint8)  # noqa: E731
    good = dict(params=[z(3, 4).half(), z(5).half()], grads=[z(3, 4), z(5)], states=[state(12), state(5)])
    made = B.adamw_tensors(d, **good, masters=[z(3, 4), z(5)], weight_decays=[0.1, 0.0])
    assert len(made) == 2 and made.array[0].n == 12 and made.array[0].weight_decay == 0.1 and made.array[1].master is not None
    bad = [dict(good, params=good["params"][:1]), dict(good, states=[state(12), state(600)]), dict(good, params=[z(3, 4), z(5)]),
           dict(good, grads=[z(3, 4).half(), z(5)]), dict(good, params=[z(4, 3).half(), z(5).half()]), dict(good, states=None),
           dict(good, masters=[z(3, 4).half(), z(5)]), dict(grads=good["grads"], masters=[z(3, 4), z(5)]), dict(good, weight_decays=[0.1]),
           dict(good, params=[good["params"][0], good["params"][0].view(-1)[7:]]),           # overlap
           dict(good, states=[good["states"][0]] * 2, params=[z(12).half(), z(12).half()], grads=[z(12), z(12)])]
    for kw in bad:
        with pytest.raises(ValueError):
            B.adamw_tensors(d, **kw)
    only = B.adamw_tensors(d, grads=good["grads"])
    with pytest.raises(ValueError, match="alone"):
        B.adamw(d, only)
    other = B.make_adamw_desc(dtype="f16", grad_dtype="f32", state_bits=32)
    with pytest.raises(ValueError, match="other types"):
        B.adamw(other, made)
    for kw in (dict(lr=z(1, dtype=torch.float64)), dict(step=z(1)), dict(scale=z(2))):
        with pytest.raises(ValueError):
            B.adamw(d, made, **kw)
    for args in ((only, z(3)), (only, z(2).double())):
        with pytest.raises(ValueError):
            B.grad_norm(*args)
    made.device = 1
    with pytest.raises(ValueError, match="the tensors are on cuda:1"):
        B.adamw(d, made)
    with pytest.raises(ValueError, match="the tensors are on cuda:1"):
        B.grad_norm(made, z(2))
    bad = B.make_adamw_desc(dtype="f16")
    bad.dtype = 9
    with pytest.raises(B.AqsgdError):
        B.adamw_tensors(bad, grads=[])


def moved(t, how):
    """Leaves the same tensor object with other memory, or with other elements in the same memory."""
    if how == "data":
        t.data = t.data.clone()
    elif how == "set":
        t.set_(torch.zeros_like(t))
    elif how == "freed":
        t.untyped_storage().resize_(0)
    elif how == "grown":
        t.resize_(100000)
    elif how == "shrunk":
        t.resize_(2)
    elif how == "turned":
        t.t_()


@pytest.mark.parametrize("how", ["data", "set", "freed", "grown", "shrunk", "turned"])
@pytest.mark.parametrize("which", ["params", "grads", "states", "masters"])
def test_a_list_whose_tensors_have_moved_is_refused(host_tensors, which, how):
    """The list holds addresses: what is written there after a tensor has got other memory is no weight any more."""
    if how == "turned" and which == "states":
        return                                                                # one dimension
    d = B.make_adamw_desc(dtype="f16", grad_dtype="f32", state_bits=8)
    shapes = [(3, 4), (0,), (30, 50)]
    lists = {"params": [torch.zeros(s).half() for s in shapes], "grads": [torch.zeros(s) for s in shapes], "masters": [torch.zeros(s) for s in shapes],
             "states": [torch.zeros(B.adamw_state_bytes(d, math.prod(s)), dtype=torch.uint8) for s in shapes]}
    made, only = B.adamw_tensors(d, **lists), B.adamw_tensors(d, grads=lists["grads"])
    moved(lists[which][2], how)
    message = which + r"\[2\] is no longer"
    with pytest.raises(ValueError, match=message):
        B.adamw(d, made)
    if which == "grads":
        for listed in (made, only):
            with pytest.raises(ValueError, match=message):
                B.grad_norm(listed, torch.zeros(2))


def test_the_binding_checks_rows_against_the_descriptor(host_tensors):
    z = torch.zeros
    d = B.make_layernorm_desc(rows=4, cols=6, dtype="f32")
    x = z(4, 6)
    bad = [dict(residual=z(4, 7)), dict(weight=z(4)), dict(bias=z(6).half()), dict(sum=z(4, 6).half()), dict(y=z(6, 4)), dict(mean=z(5)),
           dict(rstd=z(4).double()), dict(row_codes=z(4, 6, dtype=torch.int8)), dict(row_scales=z(3))]
    for kw in bad:
        with pytest.raises(ValueError, match="must be"):
            B.layernorm(d, x, **kw)
    g = dict(dy=x, x=x, mean=z(4), rstd=z(4), dx=z(4, 6))
    for kw in (dict(dy=z(4, 5)), dict(mean=z(3)), dict(rstd=z(4, 1)), dict(dx=z(4, 6).half()), dict(add=z(4)), dict(dweight=z(6).half()), dict(dbias=z(4)),
               dict(x=z(6, 4).t()), dict(x=z(4, 7)[:, :6])):
        with pytest.raises(ValueError):
            B.layernorm_grad(d, **{**g, **kw})


def test_a_stream_of_another_device_is_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    away = SimpleNamespace(cuda_stream=0, device_index=1)
    z, x = torch.zeros, torch.zeros(4, 6)
    d = B.make_layernorm_desc(rows=4, cols=6, dtype="f32")
    listed = B.AdamwTensors((B.AdamwTensor * 1)(), (0, 0, 32), True, 0, None)
    for call in (lambda: B.layernorm(d, x, y=x, stream=away), lambda: B.layernorm_grad(d, x, x, z(4), z(4), x, stream=away),
                 lambda: B.adamw(B.make_adamw_desc(dtype="f32"), listed, stream=away), lambda: B.grad_norm(listed, z(2), stream=away)):
        with pytest.raises(ValueError, match="the stream is of cuda:1"):
            call()


# ---- the plain forms ---------------------------------------------------------------------------

def test_the_plain_gradient_is_the_differences_of_the_plain_norm():
    rng = np.random.default_rng(0)
    rows, cols, eps, h = 3, 7, 1e-5, 1e-6
    x, dy, w, b = (rng.standard_normal(s) for s in ((rows, cols), (rows, cols), cols, cols))

    def loss(x, w, b):
        d = x - x.mean(axis=1, keepdims=True)
        return (dy * (d / np.sqrt((d * d).mean(axis=1, keepdims=True) + eps) * w + b)).sum()

    mean = x.mean(axis=1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    (dx, _), (dw, _), (db, _) = N.norm_grad(dy, x, mean, rstd, w, None)
    for got, at in ((dx, 0), (dw, 1), (db, 2)):
        for i in np.ndindex(got.shape):
            args = [x.copy(), w.copy(), b.copy()]
            args[at][i] += h
            more = loss(*args)
            args[at][i] -= 2 * h
            assert abs((more - loss(*args)) / (2 * h) - got[i]) < 1e-6


def test_codes_of_states_by_hand():
    """Squares of codes: 127^2 = 16129 steps to the largest; ties go up; what is not 0 stays so where asked."""
    x = np.zeros(300, np.float32)
    x[:8] = [16129, 0.5, 0.49, 2.5, 2.49, 6.5, 15876, 16002.5]
    x[256:260] = [2.0 ** -101, 0, 2.0 ** -110, 0]
    k, s = N.hold(x, 127, 0, 0.5)
    assert k[:8].tolist() == [127, 1, 0, 2, 1, 3, 126, 127] and s.tolist() == [16129, 0] and not k[256:].any()
    assert np.array_equal(N.held_values(k.astype(np.int8), s, 127)[:3], np.float32([16129, 1, 0]))
    k, s = N.hold(np.float32([65025, 1e-20, 0, 4]), 255, 1, 0.5)
    assert k.tolist() == [255, 1, 0, 2]
    for bad in (np.inf, np.nan):
        k, s = N.hold(np.float32([1, bad, 2]), 255, 1, 0.5)
        assert not k.any() and np.isnan(s).all()


def test_stochastic_codes_stand_for_their_value_on_average():
    """Over the 65536 draws the code's square has the expectation u, but for one draw's share."""
    z = (np.arange(65536, dtype=np.float64) + 1).astype(np.float32) * np.float32(2.0 ** -16)
    z = np.concatenate([z, np.full(256 - 65536 % 256 if 65536 % 256 else 0, 0.5, np.float32)]).reshape(-1, 256)
    for u in (0.0, 0.3, 1.0, 2.0, 7.77, 100.0, 15000.3, 16128.5):
        x = np.full(z.size, u, np.float32)
        x[::256] = 16129                                                        # each group's largest
        k, _ = N.hold(x, 127, 0, z)
        k = np.delete(k, np.arange(0, z.size, 256))
        low = math.floor(math.sqrt(u))
        assert set(np.unique(k)) <= {low, low + 1}
        # draws left out: one in 256, so the mean moves by a fraction of the neighbours' distance
        assert abs((k ** 2).mean() - np.float32(u)) <= (2 * low + 1) * (1 / 256 + 2 / 65536)


@pytest.mark.parametrize("bits", [32, 8])
def test_the_plain_step_is_adamw(bits):
    """Against the step in 64 bits; with states in 8 bits on the states it starts from, none."""
    rng = np.random.default_rng(1)
    n, lr, b1, b2, eps, decay = 1000, 1e-2, 0.9, 0.99, 1e-8, 0.1
    w, state = rng.standard_normal(n).astype(np.float32), N.State(n, bits)
    m = v = np.zeros(n)
    want = w.astype(np.float64)
    for step in range(1, 4 if bits == 32 else 2):
        g = rng.standard_normal(n).astype(np.float32)
        w = N.adamw(w, g, state, lr=lr, beta1=b1, beta2=b2, eps=eps, step=step, decay=decay, scale=0.5)
        h = 0.5 * g.astype(np.float64)
        m, v = b1 * m + (1 - b1) * h, b2 * v + (1 - b2) * h * h
        want = want * (1 - lr * decay) - lr * (m / (1 - b1 ** step)) / (np.sqrt(v / (1 - b2 ** step)) + eps)
        # per step: two roundings of w, one of the difference; m / r is at most 1 / sqrt(1 - b2) and off by ten half steps
        assert np.abs(w - want).max() <= step * N.U * (4 * np.abs(want).max() + 20 * lr * 10)
    if bits == 8:
        back = N.held_values(state.mk, state.ms, 127), N.held_values(state.rk, state.rs, 255)
        for got, x, top in ((back[0], m, 127), (back[1], np.sqrt(v), 255)):
            s = np.abs(N.grouped(x)).max(axis=1).repeat(256)[:n]
            # half the distance of the neighbouring squares, (2 k + 1) / 2 of s / top^2
            assert (np.abs(got - x) <= (np.sqrt(np.abs(x) / s) * top + 1.5) * s / top ** 2).all()


def test_draws_differ_from_tensor_to_tensor_and_from_step_to_step():
    n = 512
    rng = np.random.default_rng(2)
    w, g = rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    got = []
    for step, first in ((1, 0), (1, 512), (2, 0)):
        s = N.State(n, 8)
        N.adamw(w, g, s, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=step, decay=0.0, seed=7, first=first)
        got.append(s.mk)
    assert not np.array_equal(got[0], got[1]) and not np.array_equal(got[0], got[2])
    assert [hex(int(x)) for x in R.philox(0, 0, 0)] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
