"""Parity of the gradients' norm and the AdamW step with the 64-bit oracle (needs a B200).

Tolerances (u = 2^-24).  Moments: m = (beta1 s) code + (1 - beta1) (f g), every product rounded (at most three roundings a term, beta and scale included)
and the sum once: at most 4u of |beta1 m| + |(1 - beta1) f g|, which can be far above |m| where the two cancel.  The update is m times
lr / (1 - beta1^step) / (sqrt + eps): it carries that error along and adds at most 24u of its own size (two products, square root, division, reciprocal
approximations of 2^-22), its weight decay 4u of the weight; the weight is then rounded once to its type (half a step).  8-bit states are compared by what they stand for: within one step of the unrounded moment, and equal to the
oracle's codes but for a share of 2^-10 (a code can go the other way where the dither lies within the fp32 error of the value's share)."""
import numpy as np
import pytest
import torch

import paper_2306_08162_b200 as ql
from oracle import qlora_oracle as orc
from gpu_util import CANARY, canaries_intact, guarded, to_f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
HYPER = dict(beta1=0.9, beta2=0.995, eps=1e-7, weight_decay=0.02)


class Model:
    """Parameters of the given sizes with gradients and states, each between canaries."""

    def __init__(self, sizes, param="bf16", grad="fp32", bits=32, master=False, seed=0, fresh=False, **hyper):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.sizes, self.bits, self.hyper = sizes, bits, {**HYPER, **hyper}
        self.raw = []

        def tensor(n, dtype, values):
            t, raw = guarded((n,), dtype)
            t.copy_(values)
            self.raw.append((raw, (n,), dtype))
            return t
        randn = lambda n: torch.randn(n, device="cuda", generator=gen)  # noqa: E731
        e4 = torch.float8_e4m3fn
        self.master = [tensor(n, torch.float32, 0.05 * randn(n)) for n in sizes] if master else None
        self.param = [tensor(n, DTYPES[param], self.master[i] if master else 0.05 * randn(n)) for i, n in enumerate(sizes)]
        self.grad = [tensor(n, DTYPES[grad], randn(n) * 10.0 ** (-(i % 4))) for i, n in enumerate(sizes)]
        state = (lambda x: 0.0 * x) if fresh else (lambda x: x)
        self.m_scale = self.v_scale = None
        if bits == 32:
            self.m = [tensor(n, torch.float32, state(0.3 * randn(n))) for n in sizes]
            self.v = [tensor(n, torch.float32, state(randn(n).square())) for n in sizes]
        else:
            blocks = [-(-n // 256) for n in sizes]
            self.m = [tensor(n, e4, state((randn(n) * 100).clamp(-448, 448)).to(e4)) for n in sizes]
            self.v = [tensor(n, e4, state((randn(n).abs() * 100).clamp(2.0 ** -9, 448)).to(e4)) for n in sizes]
            self.m_scale = [tensor(b, torch.float32, state(0.001 * torch.rand(b, device="cuda", generator=gen) + 1e-4)) for b in blocks]
            self.v_scale = [tensor(b, torch.float32, state(0.003 * torch.rand(b, device="cuda", generator=gen) + 3e-4)) for b in blocks]
        self.desc = ql.adamw_desc(self.param, self.grad, self.m, self.v, master=self.master, m_scale=self.m_scale, v_scale=self.v_scale, **self.hyper)

    def tensors(self):
        return [t for ts in (self.param, self.master, self.m, self.v, self.m_scale, self.v_scale) for t in ts or ()]

    def snapshot(self):
        return [t.clone() for t in self.tensors()]

    def held(self, j):
        """(m, v) that the states of tensor j stand for, float64."""
        m, v = to_f64(self.m[j].float()), to_f64(self.v[j].float())
        if self.bits == 32:
            return m, v
        n = self.sizes[j]
        return m * np.repeat(to_f64(self.m_scale[j]), 256)[:n], (v * np.repeat(to_f64(self.v_scale[j]), 256)[:n]) ** 2

    def expected(self, step, lr, factor=1.0):
        """(w, m, v) after the step, and what the terms of m alone would move w by (the size that rounding errors of m are relative to)."""
        h, out = self.hyper, []
        for j in range(len(self.sizes)):
            g, (m, v) = to_f64(self.grad[j]), self.held(j)
            stepped = orc.adamw_step(to_f64((self.master or self.param)[j]), g, m, v, step, lr, h["beta1"], h["beta2"], h["eps"], h["weight_decay"], factor)
            terms = h["beta1"] * np.abs(m) + (1 - h["beta1"]) * np.abs(factor * g)
            out.append((*stepped, lr * terms / (1 - h["beta1"] ** step) / (np.sqrt(stepped[2] / (1 - h["beta2"] ** step)) + h["eps"])))
        return out

    def check(self, want, before, step, lr):
        torch.cuda.synchronize()
        for raw, shape, dtype in self.raw:
            assert canaries_intact(raw, shape, dtype), "write outside a tensor"
        for j, (w, m, v, terms) in enumerate(want):
            n = self.sizes[j]
            if n == 0:
                continue
            old = before[j]
            update = np.abs(w - old * (1 - lr * self.hyper["weight_decay"]))
            tol = 24 * U * update + 4 * U * terms + 4 * U * np.abs(old) + 1e-30
            if self.master is not None:
                got = to_f64(self.master[j])
                assert (np.abs(got - w) <= tol).all()
                assert torch.equal(self.param[j], self.master[j].to(self.param[j].dtype))
            else:
                info = torch.finfo(self.param[j].dtype)
                assert (np.abs(to_f64(self.param[j]) - w) <= tol + info.eps / 2 * (np.abs(w) + tol) + info.tiny * info.eps).all()
            gm, gv = self.held(j)
            if self.bits == 32:
                g = np.abs(to_f64(self.grad[j]))                     # (|beta1 m| + |(1 - beta1) g| is below |m| + 2 |g|)
                assert (np.abs(gm - m) <= 4 * U * (np.abs(m) + 2 * g)).all() and (np.abs(gv - v) <= 8 * U * v + 1e-44).all()
                continue
            place = np.arange(n)
            for got, scale, x, r, root in ((self.m[j], self.m_scale[j], m, 0, False), (self.v[j], self.v_scale[j], np.sqrt(v), 1, True)):
                codes, scales = orc.held_in_8_bits(x, orc.dither(place, step)[r], root)
                assert (np.abs(to_f64(scale) - scales) <= 8 * U * scales).all()
                got = to_f64(got.float())
                assert (np.abs(got) <= 448).all() and np.mean(got != codes) <= 2.0 ** -10 + 1.5 / n
                assert (np.abs(got - codes) <= np.maximum(orc.e4m3_step(got), orc.e4m3_step(codes))).all()

    def step_and_check(self, step=7, lr=1e-2, norm=None, factor=1.0, lr_arg=None, step_arg=None):
        want = self.expected(step, lr, factor)
        before = [to_f64(t) for t in (self.master or self.param)]
        ql.qlora_adamw(self.desc, lr if lr_arg is None else lr_arg, step if step_arg is None else step_arg, norm)
        self.check(want, before, step, lr)


SIZES = [[1], [8], [255, 256, 257], [2048, 2049, 4095], [32768, 88064, 5], [0, 3, 0, 1000], [100003]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_step_of_every_size(sizes, bits):
    Model(sizes, bits=bits, seed=len(sizes)).step_and_check()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("grad", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("master", [False, True])
def test_step_of_every_type(param, grad, bits, master):
    if master and param == "fp32":
        return
    Model([1000, 777, 4096], param=param, grad=grad, bits=bits, master=master, seed=3).step_and_check()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("beta1,beta2,decay,step", [(0.0, 0.0, 0.0, 1), (0.9, 0.999, 0.1, 1), (0.9, 0.999, 0.0, 100000), (0.5, 0.9, 0.3, 3)])
def test_hyperparameters_and_first_steps(bits, beta1, beta2, decay, step):
    Model([3000], bits=bits, beta1=beta1, beta2=beta2, weight_decay=decay, fresh=step == 1, seed=5).step_and_check(step=step)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_one_launch_takes(bits):
    sizes = [3 + (i * 37) % 700 for i in range(1000)]
    m = Model(sizes, bits=bits, seed=9)
    out, ws = torch.full((2,), float("nan"), device="cuda"), torch.full((ql.GRAD_NORM_WORKSPACE_BYTES,), 0xFF, dtype=torch.uint8, device="cuda")
    ql.qlora_grad_norm(m.desc, 1.0, 2.0, out, ws)
    norm, factor = orc.grad_norm([to_f64(g) for g in m.grad], 1.0, 2.0)
    assert abs(out[0].item() - norm) <= 2 * U * norm and abs(out[1].item() - factor) <= 4 * U * factor
    m.step_and_check(norm=out, factor=out[1].item())


@pytest.mark.parametrize("grad", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("sizes", [[1], [7, 0, 300], [32768, 32768], [1000003, 5]], ids=str)
def test_norm(sizes, grad):
    m = Model(sizes, grad=grad, seed=13)
    out, ws = torch.empty(2, device="cuda"), torch.empty(ql.GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    grads = [to_f64(g) for g in m.grad]
    full = orc.grad_norm(grads, 1.0, 0.0)[0]
    for prescale, max_norm in ((1.0, 0.0), (0.125, full), (0.5, full / 8), (-2.0, full), (1.0, -1.0), (1.0, float("inf"))):
        ql.qlora_grad_norm(m.desc, prescale, max_norm, out, ws)
        norm, factor = orc.grad_norm(grads, prescale, max_norm)
        assert abs(out[0].item() - norm) <= 2 * U * norm and abs(out[1].item() - factor) <= 4 * U * abs(factor), (prescale, max_norm)
    first = out.clone()
    ql.qlora_grad_norm(m.desc, 1.0, float("inf"), out, ws)
    assert torch.equal(first, out)                                    # the same bits again


def test_norm_of_very_large_and_small_gradients_and_of_none():
    """Squares that leave fp32's range do not leave that of the sum."""
    ws, out = torch.empty(ql.GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda"), torch.empty(2, device="cuda")
    for size in (1e30, 1e-30):
        m = Model([5000], seed=1)
        m.grad[0].mul_(size)
        norm, factor = orc.grad_norm([to_f64(m.grad[0])], 1.0, size)
        ql.qlora_grad_norm(m.desc, 1.0, size, out, ws)
        assert abs(out[0].item() - norm) <= 2 * U * norm and abs(out[1].item() - factor) <= 4 * U * factor
    ql.qlora_grad_norm(Model([0]).desc, 0.5, 1.0, out, ws)
    assert out.tolist() == [0.0, 0.5]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_broken_gradients_skip_the_step(bits, bad):
    m = Model([3000, 17], bits=bits, master=True, seed=17)
    m.grad[1][5] = bad
    out, ws = torch.empty(2, device="cuda"), torch.empty(ql.GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    before = m.snapshot()
    ql.qlora_grad_norm(m.desc, 1.0, 1.0, out, ws)
    assert not torch.isfinite(out[0]) and torch.isnan(out[1])
    ql.qlora_adamw(m.desc, 1e-3, 4, out)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, m.snapshot()))


@pytest.mark.parametrize("bits", [32, 8])
def test_rate_and_number_of_the_step_in_device_memory_and_replayed(bits):
    """One captured clip + step, replayed with other rates, step numbers and gradients, against the same steps issued one by one."""
    a, b = (Model([5000, 321], bits=bits, master=True, seed=19) for _ in range(2))
    lr, step = torch.tensor([0.0], device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda")
    out, ws = torch.empty(2, device="cuda"), torch.empty(ql.GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            ql.qlora_grad_norm(a.desc, 1.0, 3.0, out, ws)
            ql.qlora_adamw(a.desc, lr, step, out)
    out2, ws2 = torch.empty_like(out), torch.empty_like(ws)
    for i in range(1, 5):
        for x, y in zip(a.grad, b.grad):
            g = torch.randn(x.shape, device="cuda") * i
            x.copy_(g)
            y.copy_(g)
        lr.fill_(1e-3 * i)
        step.fill_(10 * i)
        want = a.expected(10 * i, float(np.float32(1e-3 * i)), orc.grad_norm([to_f64(g) for g in a.grad], 1.0, 3.0)[1])
        before = [to_f64(t) for t in a.master]
        graph.replay()
        a.check(want, before, 10 * i, 1e-3 * i)
        ql.qlora_grad_norm(b.desc, 1.0, 3.0, out2, ws2)
        ql.qlora_adamw(b.desc, 1e-3 * i, 10 * i, out2)
        torch.cuda.synchronize()
        assert torch.equal(out, out2)
        for x, y in zip(a.master, b.master):                             # (the corrections of the step number come from the device's own expm1)
            assert torch.allclose(x, y, rtol=1e-5, atol=1e-7)
            y.copy_(x)
        for x, y in zip(a.tensors(), b.tensors()):
            y.copy_(x)


def test_8_bit_states_follow_the_moments():
    """200 steps with gradients of slowly growing size: what the dithered 8-bit states stand for follows the exact moments in the mean,
    where nearest rounding would hold the second one still.  The root's mean over 4096 elements: each step leaves an error of at most one code step
    (an eighth), kept for some 1 / (1 - beta2) steps, independent between elements -> well below 5 % in the mean."""
    n = 4096
    m = Model([n], bits=8, fresh=True, beta2=0.99, weight_decay=0.0, seed=23)
    gen = torch.Generator(device="cuda").manual_seed(2)
    em, ev = np.zeros(n), np.zeros(n)
    for step in range(1, 201):
        m.grad[0].copy_(torch.randn(n, device="cuda", generator=gen) * (1.0 + step / 50))
        ql.qlora_adamw(m.desc, 1e-4, step)
        g = to_f64(m.grad[0])
        em, ev = 0.9 * em + 0.1 * g, 0.99 * ev + 0.01 * g * g
    gm, gv = m.held(0)
    assert abs(np.sqrt(gv).mean() / np.sqrt(ev).mean() - 1) < 0.05
    assert np.corrcoef(gm, em)[0, 1] > 0.98


def test_tensors_and_scales_cut_from_flat_buffers():
    """The tensors of a model in one buffer each, at multiples of 256 elements: the scales then begin at any float.  Each tensor like one alone."""
    sizes = [300, 257, 1000]
    alone = Model(sizes, bits=8, seed=37)
    starts = [0, 512, 1024]
    flat = dict(param=torch.zeros(2048, dtype=torch.bfloat16, device="cuda"), grad=torch.zeros(2048, device="cuda"), m=torch.zeros(2048, device="cuda").to(torch.float8_e4m3fn),
                v=torch.zeros(2048, device="cuda").to(torch.float8_e4m3fn), m_scale=torch.full((9,), 7.0, device="cuda"), v_scale=torch.full((9,), 7.0, device="cuda"))
    views = {}
    for name, buf in flat.items():
        scale = name.endswith("_scale")
        views[name] = [buf[1 + a // 256:1 + a // 256 + -(-n // 256)] if scale else buf[a:a + n] for a, n in zip(starts, sizes)]
        for view, t in zip(views[name], getattr(alone, name)):
            view.copy_(t)
    kept = {name: buf.clone() for name, buf in flat.items()}
    desc = ql.adamw_desc(views["param"], views["grad"], views["m"], views["v"], m_scale=views["m_scale"], v_scale=views["v_scale"], **HYPER)
    ql.qlora_adamw(desc, 1e-2, 5)
    ql.qlora_adamw(alone.desc, 1e-2, 5)
    for name, buf in flat.items():
        for view, t in zip(views[name], getattr(alone, name)):
            assert torch.equal(view.view(torch.uint8), t.view(torch.uint8)), name
            view.view(torch.uint8).zero_()
        for view in (kept[name][1 + a // 256:1 + a // 256 + -(-n // 256)] if name.endswith("_scale") else kept[name][a:a + n] for a, n in zip(starts, sizes)):
            view.view(torch.uint8).zero_()
        assert torch.equal(buf.view(torch.uint8), kept[name].view(torch.uint8)), name      # nothing between the tensors is touched


def test_descriptor_refuses_what_would_race():
    m = Model([300, 300])
    with pytest.raises(ValueError, match="overlap"):
        ql.adamw_desc([m.param[0], m.param[0]], m.grad, m.m, m.v)
    with pytest.raises(ValueError, match="one CUDA device"):
        ql.adamw_desc([m.param[0].cpu()], [m.grad[0]], [m.m[0]], [m.v[0]])
    with pytest.raises(ql.QloraError) as e:
        ql.qlora_adamw(m.desc, 1e-3, 0)
    assert e.value.status == -1
    with pytest.raises(ValueError, match="int32"):
        ql.qlora_adamw(m.desc, 1e-3, torch.tensor([1], device="cuda"))


def test_two_streams_at_once():
    a, b = Model([40000, 300], seed=29), Model([50000], bits=8, seed=31)
    wa, wb = a.expected(3, 1e-3), b.expected(3, 1e-3)
    ba, bb = [to_f64(t) for t in a.param], [to_f64(t) for t in b.param]
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    ql.qlora_adamw(a.desc, 1e-3, 3, stream=sa)
    ql.qlora_adamw(b.desc, 1e-3, 3, stream=sb.cuda_stream)
    a.check(wa, ba, 3, 1e-3)
    b.check(wb, bb, 3, 1e-3)
    assert CANARY == 0x7B
