"""AdamW and the gradients' norm on the GPU: weights and states bit for bit as the header's binary32 steps give them."""
import math
import threading

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import norms_reference as N
import products8_reference as R
from paper_2206_01299_amd import binding as B
from test_gpu_norms import typed
from test_gpu_products8 import DTYPES, Framed, stage_inputs, stage_step, stored

TYPES = [("f32", "f32"), ("f16", "f32"), ("f16", "f16"), ("bf16", "f32"), ("bf16", "bf16")]
KINDS = [(32, 0), (8, 0), (8, 1)]                                               # state bits, rounding


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.fail("these tests need an MI355X")
    B.lib()


class Program:
    """Some tensors with their plain counterparts, stepped side by side."""

    def __init__(self, sizes, dtype, grad_dtype, bits, rounding=0, master=False, seed=0, lead=64, decays=True, **settings):
        self.rng = np.random.default_rng([seed, len(sizes)])
        self.dtype, self.grad_dtype, self.bits, self.master = dtype, grad_dtype, bits, master
        self.settings = {"lr": 1e-2, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8, **settings}
        self.desc = B.make_adamw_desc(dtype=dtype, grad_dtype=grad_dtype, state_bits=bits, rounding=rounding, rng_seed=seed + 77, **self.settings)
        self.seed = seed + 77 if rounding else None
        pt, gt = B.DTYPE_NAME[dtype], B.DTYPE_NAME[grad_dtype]
        size = torch.empty(0, dtype=pt).element_size()
        w = [self.rng.standard_normal(n).astype(np.float32) for n in sizes]
        self.params = [Framed((n,), pt, lead if lead == 64 else lead * size) for n in sizes]
        self.masters = [Framed((n,), torch.float32) for n in sizes] if master else None
        self.grads = [Framed((n,), gt, lead if lead == 64 else lead * torch.empty(0, dtype=gt).element_size()) for n in sizes]
        self.states = [Framed((N.state_bytes(n, bits),), torch.uint8) for n in sizes]
        for i, x in enumerate(w):
            self.params[i].t.copy_(torch.from_numpy(x))
            if master:
                self.masters[i].t.copy_(torch.from_numpy(x))
            self.states[i].t.zero_()
        self.weights = [x if master else typed(dtype)(x) for x in w]
        self.plain = [N.State(n, bits) for n in sizes]
        self.decays = [0.01 * (i % 3) if decays else 0.0 for i in range(len(sizes))]
        self.list = B.adamw_tensors(self.desc, params=[f.t for f in self.params], grads=[f.t for f in self.grads],
                                    states=[f.t for f in self.states], masters=[f.t for f in self.masters] if master else None,
                                    weight_decays=self.decays)

    def draw(self, scale=1.0):
        for f in self.grads:
            f.t.copy_(torch.from_numpy(scale * self.rng.standard_normal(f.t.numel()) * np.exp(self.rng.standard_normal(f.t.numel()))))

    def step(self, step, scale=None, **kw):
        self.desc.step = step
        given = None if scale is None else torch.tensor(scale, device="cuda")
        B.adamw(self.desc, self.list, scale=given, **kw)
        self.follow(step, scale)

    def follow(self, step, scale=None, lr=None):
        first = 0
        for i, (f, s) in enumerate(zip(self.grads, self.plain)):
            new = N.adamw(self.weights[i], f.t.float().cpu().numpy(), s, **{**self.settings, **({} if lr is None else {"lr": lr})}, step=step,
                          decay=self.decays[i], scale=scale, seed=self.seed, first=first)
            self.weights[i] = new if self.master else typed(self.dtype)(new)
            first += N.up(s.n, 256)

    def check(self, tag=""):
        torch.cuda.synchronize()
        for i, s in enumerate(self.plain):
            where = f"{self.dtype}/{self.grad_dtype} {self.bits} bits {tag}: tensor {i} of {s.n}"
            for f in (self.params[i], self.grads[i], self.states[i], *([self.masters[i]] if self.master else [])):
                f.check(where)
            got = B.adamw_state_views(self.desc, self.states[i].t, s.n)
            for name, a, b in zip("mv" if self.bits == 32 else ("m codes", "r codes", "m scales", "r scales"), got, s.parts()):
                a = a.cpu().numpy()
                bad = np.flatnonzero(~((a == b) | (np.isnan(a.astype(np.float32)) & np.isnan(b.astype(np.float32)))))
                assert bad.size == 0, f"{where}: {name} differs at {bad[:3]}: {a[bad[:3]]} instead of {b[bad[:3]]} ({bad.size} do)"
            if self.master:
                assert np.array_equal(self.masters[i].t.cpu().numpy(), self.weights[i], equal_nan=True), f"{where}: master"
            want = typed(self.dtype)(self.weights[i])
            assert np.array_equal(self.params[i].t.float().cpu().numpy(), want, equal_nan=True), f"{where}: weights"


SIZES = [1, 3, 0, 255, 256, 257, 2047, 2048, 2049, 5000, 4, 70001]


@pytest.mark.parametrize("bits,rounding", KINDS)
@pytest.mark.parametrize("dtype,grad_dtype", TYPES)
def test_adamw(dtype, grad_dtype, bits, rounding):
    p = Program(SIZES, dtype, grad_dtype, bits, rounding)
    for step in range(1, 5):
        p.draw()
        p.step(step, scale=None if step % 2 else 0.25)
        p.check(f"step {step}")


@pytest.mark.parametrize("bits,rounding", KINDS)
@pytest.mark.parametrize("dtype,grad_dtype", TYPES[1:])
def test_adamw_with_a_binary32_copy(dtype, grad_dtype, bits, rounding):
    p = Program(SIZES, dtype, grad_dtype, bits, rounding, master=True, lead=1, seed=3)
    for step in (1, 2, 1000):
        p.draw()
        p.step(step, scale=3.0)
        p.check(f"step {step}")


@pytest.mark.parametrize("bits,rounding", KINDS)
def test_adamw_of_more_tensors_than_a_launch_holds(bits, rounding):
    sizes = [(37 * i) % 700 for i in range(150)]
    p = Program(sizes, "f16", "f32", bits, rounding, seed=1)
    for step in (1, 2):
        p.draw()
        p.step(step)
        p.check(f"step {step}")


@pytest.mark.parametrize("bits,rounding", KINDS)
def test_adamw_of_many_groups(bits, rounding):
    p = Program([1_000_003, 300_000], "bf16", "bf16", bits, rounding, seed=2)
    p.draw()
    p.step(1)
    p.draw(1e-3)
    p.step(2)
    p.check()


@pytest.mark.parametrize("bits,rounding", KINDS)
def test_adamw_settings(bits, rounding):
    for i, settings in enumerate((dict(beta1=0.0), dict(beta2=0.0, eps=0.0), dict(lr=0.0), dict(eps=1.0, beta2=0.9), dict(beta1=0.0, beta2=0.0, lr=3.0))):
        p = Program([513, 40], "f32", "f32", bits, rounding, seed=10 + i, decays=False, **settings)
        for step in (1, 2):
            p.draw()
            p.step(step)
            p.check(str(settings))


@pytest.mark.parametrize("bits,rounding", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_adamw_of_gradients_that_are_no_ordinary_numbers(dtype, bits, rounding):
    """Zeros from the first step on, subnormals, the largest, infinities and NaN: in 32 bits they stay with their element, in
    8 with their group."""
    big = {"f16": 65504.0, "bf16": 3e38, "f32": 3e38}[dtype]
    tiny = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}[dtype]
    p = Program([2000, 300], dtype, dtype, bits, rounding, seed=5)
    for step in range(1, 4):
        p.draw()
        g = p.grads[0].t
        g[:256] = 0.0
        g[300:400] = tiny * step
        g[512:768] = 1e-30
        g[1024:1100] = big
        if step == 2:
            g[1300], g[1600], g[1999] = math.inf, math.nan, -math.inf
        p.step(step)
        p.check(f"step {step}")
    codes = B.adamw_state_views(p.desc, p.states[0].t, 2000)
    if bits == 8:
        assert torch.isnan(codes[2][[1300 // 256, 1600 // 256, 1999 // 256]]).all() and torch.isfinite(codes[2][[0, 1, 2]]).all()
    assert torch.isfinite(p.params[1].t).all()


@pytest.mark.parametrize("bits,rounding", KINDS)
@pytest.mark.parametrize("settings", [{}, dict(eps=0.0), dict(eps=1e-30), dict(eps=2.0 ** -48), dict(eps=1e-15), dict(eps=2.0 ** 48), dict(eps=1e16),
                                      dict(beta2=1 - 2.0 ** -53), dict(beta1=1 - 2.0 ** -53, beta2=1 - 2.0 ** -53, eps=2.0 ** 48)])
def test_adamw_at_the_ends_of_the_quick_ranges(settings, bits, rounding):
    """Gradients of every size, and such whose moments lie right at or beside 2^-70, 2^60 (m), 2^-48 and 2^20 (r)."""
    p = Program([256 * 40, 777], "f32", "f32", bits, rounding, seed=9, **settings)
    d = p.desc
    for step in (1, 2, 3):
        p.draw()
        g = p.grads[0].t
        signs = torch.where(torch.arange(256 * 8, device="cuda") % 3 == 0, -1.0, 1.0)
        g[:256 * 8] = signs * torch.exp2(torch.linspace(-149, 126, 256 * 8, device="cuda", dtype=torch.float64)).float()
        for group, (at, part) in enumerate(((2.0 ** -70, 1 - d.beta1), (2.0 ** 60, 1 - d.beta1), (2.0 ** -48, (1 - d.beta2) ** 0.5), (2.0 ** 20, (1 - d.beta2) ** 0.5)), 8):
            exact = np.float32(at / part)
            beside = [exact]
            for _ in range(4):
                beside = [np.nextafter(beside[0], np.float32(0)), *beside, np.nextafter(beside[-1], np.float32(np.inf))]
            for k, v in enumerate(beside):                                      # one such element to a group
                g[256 * (group + 6 * (k % 4)) + 17 * k] = float(v)
        p.step(step)
        p.check(f"step {step}")


@pytest.mark.parametrize("bits,rounding", KINDS)
def test_a_factor_that_is_not_finite_skips_the_step(bits, rounding):
    p = Program([700, 70], "f16", "f32", bits, rounding, master=True)
    p.draw()
    p.step(1, scale=0.5)
    frames = [f.raw.clone() for f in (*p.params, *p.masters, *p.states)]
    for bad in (math.nan, math.inf, -math.inf):
        p.draw()
        p.desc.step = 2
        B.adamw(p.desc, p.list, scale=torch.tensor(bad, device="cuda"))
        torch.cuda.synchronize()
        for f, before in zip((*p.params, *p.masters, *p.states), frames):
            assert torch.equal(f.raw, before)
    p.draw()
    p.step(2, scale=0.5)
    p.check()


@pytest.mark.parametrize("bits,rounding", KINDS)
def test_steps_of_a_captured_call_go_on(bits, rounding):
    """lr, step and scale on the device: replays with new values, eager work between them, against the plain steps."""
    p = Program([513, 5000, 40], "bf16", "f32", bits, rounding, master=True, seed=4)
    lr, step, scale = torch.tensor([0.0], device="cuda"), torch.tensor(0, device="cuda"), torch.tensor(1.0, device="cuda")
    result, ws = torch.empty(2, device="cuda"), torch.empty(B.grad_norm_workspace_bytes(p.list), dtype=torch.uint8, device="cuda")
    p.draw()
    lr.fill_(1e-3); step.fill_(1)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.grad_norm(p.list, result, max_norm=1.0, loss_scale=scale, workspace=ws)
        B.adamw(p.desc, p.list, lr=lr, step=step, scale=result[1:])
    for t in (1, 2, 3, 50, 100_000):
        p.draw(float(t))
        lr.fill_(0.01 / t); step.fill_(t); scale.fill_(2.0 ** (t % 7))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        norm = math.sqrt(sum((f.t.double() ** 2).sum().item() for f in p.grads)) / 2.0 ** (t % 7)
        got = result.cpu().numpy()
        assert abs(got[0] - norm) <= 2 * N.U * norm and abs(got[1] - min(1.0, 1.0 / norm) / 2.0 ** (t % 7)) <= 2 * N.U * got[1]
        p.follow(t, scale=got[1], lr=float(lr.item()))
        p.check(f"replay at step {t}")
        again = torch.empty(2, device="cuda")
        B.grad_norm(p.list, again, max_norm=1.0, loss_scale=scale)
        assert torch.equal(again, result)


def test_a_step_below_one_on_the_device_counts_as_one():
    p = Program([300], "f32", "f32", 32)
    p.draw()
    B.adamw(p.desc, p.list, step=torch.tensor([-5], device="cuda"))
    p.follow(1)
    p.check()


def test_streams_and_both_ways_of_the_binding(monkeypatch):
    side = torch.cuda.Stream()
    programs = [Program([513, 5000, 40], "f16", "f16", 8, 1, seed=6) for _ in range(4)]
    for i, p in enumerate(programs):
        if i == 2:
            monkeypatch.setattr(B, "_native", B._Ctypes())
        p.draw()
        torch.cuda.synchronize()
        if i == 0:
            p.step(1)
        elif i == 1:
            p.step(1, stream=side)
        else:
            with torch.cuda.stream(side if i == 3 else torch.cuda.current_stream()):
                p.step(1, scale=None)
        result = torch.empty(2, device="cuda")
        torch.cuda.synchronize()
        B.grad_norm(p.list, result, max_norm=3, stream=side)
        torch.cuda.synchronize()
        p.check(f"way {i}")
        p.result = result
    for p in programs[1:]:
        assert torch.equal(p.result, programs[0].result)


def test_calls_of_two_threads_at_once():
    programs = [Program([513, 70001, 40], "bf16", "f32", 8, 1, seed=8 + i) for i in range(2)]
    errors = []

    def work(p):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for step in range(1, 5):
                    p.draw()
                    p.step(step)
                torch.cuda.current_stream().synchronize()
        except Exception as e:                                              # told to the test's own thread
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(p,)) for p in programs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for p in programs:
        p.check()


def test_lists_without_elements():
    d = B.make_adamw_desc(dtype="f32")
    empty = torch.empty(0, device="cuda")
    for n in (0, 3):
        made = B.adamw_tensors(d, params=[empty] * n, grads=[empty] * n, states=[torch.empty(0, dtype=torch.uint8, device="cuda")] * n)
        B.adamw(d, made)
        result = torch.full((2,), 7.0, device="cuda")
        B.grad_norm(made, result, max_norm=1.0, loss_scale=torch.tensor(4.0, device="cuda"))
        assert result.tolist() == [0.0, 0.25]


# ---- the norm ----------------------------------------------------------------------------------

def grads_of(sizes, dtype, seed=0, scale=1.0):
    rng = np.random.default_rng([seed, len(sizes)])
    return [stored(scale * rng.standard_normal(n), dtype)[0] for n in sizes]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sizes", [[1], [3], [4095, 4096, 4097], [0, 5, 0, 70001], [(31 * i) % 900 for i in range(150)], [9_000_001], [5_000_000, 7, 3_000_001]])
def test_grad_norm(dtype, sizes):
    grads = grads_of(sizes, dtype)
    made = B.adamw_tensors(B.make_adamw_desc(dtype=dtype), grads=grads)
    want = math.sqrt(sum((g.double() ** 2).sum().item() for g in grads))
    ws = Framed((B.grad_norm_workspace_bytes(made),), torch.uint8)
    for most, loss in ((1.0, None), (math.inf, 8.0), (want / 3, 0.5), (want * 2, None), (0.0, 2.0)):
        result = Framed((2,), torch.float32)
        B.grad_norm(made, result.t, max_norm=most, loss_scale=None if loss is None else torch.tensor(loss, device="cuda"), workspace=ws.t)
        torch.cuda.synchronize()
        ws.check("workspace")
        result.check("result")
        inverse = 1.0 if loss is None else 1.0 / loss
        got, norm = result.t.tolist(), want * inverse
        # one rounding to binary32; sums in binary64 are off by far less than the other half step
        assert abs(got[0] - norm) <= 2 * N.U * norm
        assert abs(got[1] - min(1.0, most / norm) * inverse) <= 2 * N.U * abs(got[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sizes", [[2, 7, 8, 9, 0, 255, 256, 257, 1, 511, 512, 513], [512] * 32, [1] * 64, [256] * 65, [16384], [16385], [32768], [32769], [9, 16000]])
def test_grad_norm_of_few_elements(dtype, sizes):
    """Around what one launch takes; from addresses of any alignment, among infinities that belong to nothing."""
    grads, want = [], 0.0
    for i, g in enumerate(grads_of(sizes, dtype, 1)):
        at = 1 + i % 7
        held = torch.full((g.numel() + 16,), math.inf, dtype=g.dtype, device="cuda")
        held[at:at + g.numel()] = g
        grads.append(held[at:at + g.numel()])
        want += (g.double() ** 2).sum().item()
    made, result = B.adamw_tensors(B.make_adamw_desc(dtype=dtype), grads=grads), Framed((2,), torch.float32)
    ws = Framed((B.grad_norm_workspace_bytes(made),), torch.uint8)
    got = []
    for _ in range(2):
        B.grad_norm(made, result.t, max_norm=0.5, workspace=ws.t)
        torch.cuda.synchronize()
        got.append(result.t.tolist())
    ws.check("workspace")
    result.check("result")
    want = math.sqrt(want)
    assert got[0] == got[1] and abs(got[0][0] - want) <= 2 * N.U * want
    assert abs(got[0][1] - min(1.0, 0.5 / want)) <= 2 * N.U * got[0][1]


def test_grad_norm_of_what_is_no_ordinary_number():
    for dtype, value in (("f32", 3e38), ("bf16", 3e38), ("f16", 65504.0), ("f32", 2.0 ** -149), ("f16", 2.0 ** -24)):
        g = torch.full((5000,), value, dtype=B.DTYPE_NAME[dtype], device="cuda")
        result = torch.empty(2, device="cuda")
        B.grad_norm(B.adamw_tensors(B.make_adamw_desc(dtype=dtype), grads=[g]), result, max_norm=1.0,
                    loss_scale=torch.tensor(256.0, device="cuda"))
        want = g[0].double().item() * math.sqrt(5000) / 256
        assert abs(result[0].item() - want) <= 2 * N.U * want + 2.0 ** -149
        assert abs(result[1].item() - min(1.0, 1.0 / want) / 256) <= 2 * N.U / 256
    for bad, n in ((math.inf, 5000), (math.nan, 5000), (-math.inf, 5000), (math.nan, 50000), (math.inf, 50000)):
        g = torch.ones(n, device="cuda")
        g[n - 1] = bad
        result = torch.empty(2, device="cuda")
        B.grad_norm(B.adamw_tensors(B.make_adamw_desc(dtype="f32"), grads=[g]), result, max_norm=1.0)
        assert not math.isfinite(result[0].item()) and math.isnan(result[1].item())


def test_two_graphs_that_share_a_workspace():
    lists = [B.adamw_tensors(B.make_adamw_desc(dtype="f16"), grads=grads_of(s, "f16", i)) for i, s in enumerate(([5000, 70001], [300_000]))]
    ws = torch.empty(max(B.grad_norm_workspace_bytes(x) for x in lists), dtype=torch.uint8, device="cuda")
    graphs = []
    for made in lists:
        result, g = torch.empty(2, device="cuda"), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            B.grad_norm(made, result, workspace=ws)
        graphs.append((g, made, result))
    for _ in range(3):
        for g, made, _ in graphs:
            for t in made.held[0]:
                t.copy_(torch.randn(t.shape, device="cuda"))
            g.replay()
        torch.cuda.synchronize()
        for _, made, result in graphs:
            want = math.sqrt(sum((t.double() ** 2).sum().item() for t in made.held[0]))
            assert abs(result[0].item() - want) <= 2 * N.U * want and result[1].item() == 1.0


# ---- the largest -------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [8, 32])
def test_a_tensor_whose_offsets_pass_32_bits(bits):
    """2^31 + 300 weights: the first and the last groups are as a call on them alone gives."""
    n, part = (1 << 31) + 300, 256 * 40
    if torch.cuda.mem_get_info()[0] < (60 << 30):
        pytest.skip("needs 50 GB")
    d = B.make_adamw_desc(dtype="f16", state_bits=bits, step=3)
    last = n // 256 * 256 - part
    cuts = [(0, part), (last, n - last)]
    w, g = torch.zeros(n, dtype=torch.float16, device="cuda"), torch.zeros(n, dtype=torch.float16, device="cuda")
    state = torch.zeros(B.adamw_state_bytes(d, n), dtype=torch.uint8, device="cuda")
    few = []
    for at, k in cuts:
        w[at:at + k] = torch.randn(k, device="cuda").half()
        g[at:at + k] = torch.randn(k, device="cuda").half()
        few.append((w[at:at + k].clone(), g[at:at + k].clone(), torch.zeros(B.adamw_state_bytes(d, k), dtype=torch.uint8, device="cuda")))
    made = B.adamw_tensors(d, params=[w], grads=[g], states=[state])
    for _ in range(2):
        B.adamw(d, made)
    result, want = torch.empty(2, device="cuda"), math.sqrt(sum((x[1].double() ** 2).sum().item() for x in few))
    B.grad_norm(made, result)
    assert abs(result[0].item() - want) <= 2 * N.U * want
    for (at, k), (fw, fg, fs) in zip(cuts, few):
        alone = B.adamw_tensors(d, params=[fw], grads=[fg], states=[fs])
        for _ in range(2):
            B.adamw(d, alone)
        assert torch.equal(w[at:at + k], fw)
        for view, whole in zip(B.adamw_state_views(d, fs, k), B.adamw_state_views(d, state, n)):
            first = at if view.numel() == k else at // 256
            assert torch.equal(whole[first:first + view.numel()], view)
    del w, g, state, made
    torch.cuda.empty_cache()


def test_the_time_of_a_call_of_several_launches():
    p = Program([700] * 150, "f32", "f32", 32)
    p.draw()
    result = torch.empty(2, device="cuda")
    few = B.adamw_tensors(p.desc, params=[p.params[0].t], grads=[p.grads[0].t], states=[p.states[0].t])
    for call in (lambda: B.adamw(p.desc, p.list), lambda: B.adamw(p.desc, few), lambda: B.grad_norm(p.list, result), lambda: B.grad_norm(few, result)):
        call()
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record(); stop.record()                                       # makes the events
        torch.cuda.synchronize()
        B.profile_next_launch(start, stop)
        call()
        torch.cuda.synchronize()
        assert 0.0005 < start.elapsed_time(stop) < 5.0


# ---- together: a stage's step from its norm to its weights -----------------------------------------

class Stage:
    """A block behind a norm over the residual stream: float16 weights with binary32 copies, states in 8 bits, trained on
    messages of the next stage."""

    def __init__(self, m, k, f, seed=0):
        self.m, self.k, self.f = m, k, f
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.masters = [1 + 0.1 * n(k), 0.1 * n(k), n(2 * f, k) / k ** 0.5, n(k, f) / f ** 0.5]
        self.weights = [w.half() for w in self.masters]
        self.grads = [torch.zeros_like(w) for w in self.masters]
        self.desc = B.make_adamw_desc(dtype="f16", grad_dtype="f32", state_bits=8, rounding=B.STOCHASTIC, rng_seed=5, lr=1e-2)
        self.states = [torch.zeros(B.adamw_state_bytes(self.desc, w.numel()), dtype=torch.uint8, device="cuda") for w in self.weights]
        self.list = B.adamw_tensors(self.desc, params=self.weights, grads=self.grads, states=self.states, masters=self.masters, weight_decays=[0, 0, 0.1, 0.1])
        self.at, self.result = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty(2, device="cuda")
        self.ws = torch.empty(B.grad_norm_workspace_bytes(self.list), dtype=torch.uint8, device="cuda")
        self.inner, self.buf = {}, {}

    def step(self, x, res, message, scales):
        d = B.make_layernorm_desc(rows=self.m, cols=self.k, dtype="f16")
        b, (lw, lb, w1, w2) = self.buf, self.weights
        for name, shape, t in (("sum", (self.m, self.k), torch.float16), ("y", (self.m, self.k), torch.float16), ("mean", (self.m,), torch.float32),
                               ("rstd", (self.m,), torch.float32), ("row_codes", (self.m, R.stride(self.k)), torch.int8),
                               ("row_scales", (self.m,), torch.float32), ("dx", (self.m, self.k), torch.float16)):
            if name not in b:
                b[name] = torch.zeros(shape, dtype=t, device="cuda")
        B.layernorm(d, x, residual=res, weight=lw, bias=lb, **{n: b[n] for n in ("sum", "y", "mean", "rstd", "row_codes", "row_scales")})
        out = stage_step(b["y"], w1, w2, message, scales, "f16", self.inner)
        B.layernorm_grad(d, out["dx"], b["sum"], b["mean"], b["rstd"], b["dx"], weight=lw, add=out["dx"], dweight=self.grads[0], dbias=self.grads[1])
        self.grads[2].copy_(out["dw1"])
        self.grads[3].copy_(out["dw2"])
        self.at.add_(1)
        B.grad_norm(self.list, self.result, max_norm=1.0, workspace=self.ws)
        B.adamw(self.desc, self.list, step=self.at, scale=self.result[1:])
        return {**out, **b, "block_dx": out["dx"]}


def test_a_stages_step_with_its_norm_and_its_update():
    """Eager steps against the plain ones: the norm's codes are those that the block quantises its input to, its gradient is that
    of the binary32 values, weights and states follow the plain update bit for bit; and a captured step, replayed with new inputs, goes
    the same way."""
    m, k, f = 300, 160, 224
    eager, captured = Stage(m, k, f), Stage(m, k, f)
    rng = np.random.default_rng(0)

    def draw(seed):
        x, _, _, message, scales = stage_inputs(m, k, f, "f16", seed)
        return x, stored(rng.standard_normal((m, k)), "f16")[0], message, scales

    data = [draw(i) for i in range(4)]
    held = [t.clone() for t in data[0]]
    captured.step(*held)                                                       # makes the buffers
    torch.cuda.synchronize()
    for a, b in zip(captured.masters + captured.weights + captured.states, eager.masters + eager.weights + eager.states):
        a.copy_(b)
    captured.at.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step(*held)
    for a, b in zip(captured.masters + captured.weights + captured.states, eager.masters + eager.weights + eager.states):
        a.copy_(b)
    captured.at.zero_()
    plain = [N.State(w.numel(), 8) for w in eager.masters]
    masters = [w.cpu().numpy().reshape(-1) for w in eager.masters]
    for step, inputs in enumerate(data, 1):
        out = eager.step(*inputs)
        torch.cuda.synchronize()
        codes, scales = R.quantise(out["y"].float().cpu().numpy())
        assert np.array_equal(out["row_codes"].cpu().numpy(), codes) and np.array_equal(out["row_scales"].cpu().numpy(), scales)
        dy = out["block_dx"].float().cpu().numpy()
        want = N.norm_grad(dy, out["sum"].float().cpu().numpy(), out["mean"].cpu().numpy(), out["rstd"].cpu().numpy(), typed("f16")(masters[0]), dy)
        for got, (w, off), dt in zip((out["dx"], eager.grads[0], eager.grads[1]), want, ("f16", "f32", "f32")):
            R.close(got.double().cpu().numpy(), w, off, dt, f"step {step}")
        norm = math.sqrt(sum((g.double() ** 2).sum().item() for g in eager.grads))
        factor = eager.result[1].item()
        assert abs(eager.result[0].item() - norm) <= 2 * N.U * norm and abs(factor - min(1.0, 1.0 / norm)) <= 2 * N.U * factor
        first = 0
        for i, s in enumerate(plain):
            masters[i] = N.adamw(masters[i], eager.grads[i].cpu().numpy().reshape(-1), s, lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, step=step,
                                 decay=[0, 0, 0.1, 0.1][i], scale=np.float32(factor), seed=5, first=first)
            first += N.up(s.n, 256)
            assert np.array_equal(eager.masters[i].cpu().numpy().reshape(-1), masters[i]), f"step {step}: weight {i}"
            for a, b in zip(B.adamw_state_views(eager.desc, eager.states[i], s.n), s.parts()):
                assert np.array_equal(a.cpu().numpy(), b), f"step {step}: state {i}"
        for a, b in zip(held, inputs):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured.masters + captured.weights + captured.states, eager.masters + eager.weights + eager.states):
            assert torch.equal(a, b), f"replay {step}"


@pytest.mark.parametrize("which", ["params", "grads", "states", "masters"])
@pytest.mark.parametrize("how", ["data", "grown"])
def test_a_list_whose_tensors_have_moved_is_refused(which, how):
    """Both ways of the binding refuse it before anything is launched; a list made anew goes on."""
    d = B.make_adamw_desc(dtype="f16", grad_dtype="f32", state_bits=8)
    sizes = [700, 0, 3, 5000]
    lists = {"params": [torch.nn.Parameter(torch.ones(n, device="cuda").half(), requires_grad=False) for n in sizes],
             "grads": [torch.ones(n, device="cuda") for n in sizes], "masters": [torch.ones(n, device="cuda") for n in sizes],
             "states": [torch.zeros(B.adamw_state_bytes(d, n), dtype=torch.uint8, device="cuda") for n in sizes]}
    made, result = B.adamw_tensors(d, **lists), torch.empty(2, device="cuda")
    ws = torch.empty(B.grad_norm_workspace_bytes(made), dtype=torch.uint8, device="cuda")

    def calls():
        return (B._native.adamw(d, made, None, None, None, None), B._native.grad_norm(made, result, 1.0, None, ws, None))

    assert calls() == (0, 0)
    t = lists[which][3]
    size = t.numel()
    if how == "data":
        t.data = t.data.clone()
    else:
        t.resize_(1 << 20)
    torch.cuda.synchronize()
    before = [p.clone() for p in lists["params"]]
    assert calls() == (None, None if which == "grads" else 0)
    with pytest.raises(ValueError, match=which + r"\[3\] is no longer"):
        B.adamw(d, made)
    torch.cuda.synchronize()
    for a, b in zip(before, lists["params"]):
        assert torch.equal(a, b)
    t.resize_(size)
    made = B.adamw_tensors(d, **lists)
    assert calls() == (0, 0)
    torch.cuda.synchronize()
    assert result[0] > 0 and (lists["params"][0] != before[0]).all()
