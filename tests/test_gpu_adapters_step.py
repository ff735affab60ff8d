"""The pieces of a step of several adapters on one frozen base, as a program uses them: the quantized projection without a branch, the adapters beside it, the
head's cross entropy, and the way back to every adapter's gradients and the optimizer."""
import numpy as np
import pytest
import torch

import paper_2306_08162_b200 as ql
from gpu_util import to_f64

pytestmark = pytest.mark.gpu

HALF_BF16 = 2.0 ** -8


class Model:
    def __init__(self, M, K, D, V, r, L, seed=3):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
        self.M, self.K, self.D, self.V, self.r, self.L = M, K, D, V, r, L
        self.layer = ql.desc(4, 64, K, D, 0, 0.0)
        self.Q = torch.empty((K * 4 // 32, D), dtype=torch.int32, device="cuda")
        self.sc, self.zp = (torch.empty((K // 64, D), dtype=torch.float16, device="cuda") for _ in range(2))
        ql.qlora_quantize_rtn(self.layer, 0.05 * randn(D, K), self.Q, self.sc, self.zp)
        self.W = torch.empty((D, K), dtype=torch.bfloat16, device="cuda")
        ql.qlora_dequant(self.layer, self.Q, self.sc, self.zp, self.W)
        self.A, self.B = (randn(L, r, K) / K ** 0.5).bfloat16(), (0.1 * randn(L, D, r)).bfloat16()
        self.scales = torch.full((L,), 2.0, device="cuda")
        self.head = (randn(V, D) / D ** 0.5).bfloat16()
        self.X = randn(M, K).bfloat16()
        self.labels = torch.randint(0, V, (M,), device="cuda", generator=gen).int()
        self.labels[::7] = -1                                          # the prompts' tokens
        requests = torch.randint(-1, L, (9,), device="cuda", generator=gen)
        self.adapter_of = requests[torch.arange(M, device="cuda") * 9 // M].int()
        self.adapters = ql.adapters_desc(K, D, r, L)
        self.n = int((self.labels >= 0).sum())
        self.d_loss = torch.full((M,), 1.0 / self.n, device="cuda")
        byte = dict(dtype=torch.uint8, device="cuda")
        self.ws = torch.empty(ql.qlora_workspace_bytes(self.layer, M), **byte)
        self.ws_a = torch.empty(ql.qlora_adapters_workspace_bytes(self.adapters, M), **byte)
        self.ws_h = torch.empty(ql.qlora_head_loss_workspace_bytes(M, V, D, True), **byte)
        self.hidden, self.dh = (torch.empty((M, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.dX = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
        self.H, self.G = (torch.empty((M, r), device="cuda") for _ in range(2))
        self.loss = torch.empty(M, device="cuda")
        self.dA, self.dB = torch.empty((L, r, K), device="cuda"), torch.empty((L, D, r), device="cuda")

    def step(self):
        m = self
        ql.qlora_fwd(m.layer, m.M, m.X, m.Q, m.sc, m.zp, None, None, m.hidden, None, m.ws)
        ql.qlora_adapters_fwd(m.adapters, m.M, m.X, m.adapter_of, m.A, m.B, m.scales, m.hidden, m.hidden, m.H, m.ws_a)
        ql.qlora_head_loss(m.hidden, m.head, m.labels, m.loss, m.ws_h, d_loss=m.d_loss, d_hidden=m.dh)
        ql.qlora_bwd_input(m.layer, m.M, m.dh, m.Q, m.sc, m.zp, None, None, m.dX, None, m.ws)
        ql.qlora_adapters_bwd_input(m.adapters, m.M, m.dh, m.adapter_of, m.A, m.B, m.scales, m.dX, m.dX, m.G, m.ws_a)
        ql.qlora_adapters_bwd_lora(m.adapters, m.M, m.X, m.dh, m.adapter_of, m.A, m.B, m.scales, m.H, m.G, m.dA, m.dB, 0, m.ws_a)


def near(got, want, factor):
    """Within `factor` roundings to bf16 of the tensor's size: every step of the chain rounds what it hands on once or twice, and what it hands on is multiplied by
    matrices that neither grow nor shrink it on average."""
    want = want if isinstance(want, np.ndarray) else to_f64(want)
    off = np.linalg.norm(to_f64(got) - want) / np.linalg.norm(want)
    assert off <= factor * HALF_BF16, off


@pytest.mark.parametrize("M,r", [(40, 8), (700, 16), (1500, 40)])
def test_a_step_against_float64(M, r):
    m = Model(M, 512, 384, 3000, r, 4)
    m.step()
    torch.cuda.synchronize()
    assert ql.qlora_device_status() == 0
    A, B = m.A.double().requires_grad_(True), m.B.double().requires_grad_(True)
    X = m.X.double().requires_grad_(True)
    a = m.adapter_of.long()
    on = (a >= 0).double()[:, None]
    chosen = a.clamp_min(0)
    low = torch.einsum("tk,tjk->tj", X, A[chosen])
    hidden = X @ m.W.double().t() + 2.0 * on * torch.einsum("tj,tdj->td", low, B[chosen])
    loss = torch.nn.functional.cross_entropy(hidden @ m.head.double().t(), m.labels.long(), ignore_index=-1, reduction="none")
    dX, dA, dB = torch.autograd.grad(loss.sum() / m.n, (X, A, B))
    # hidden: the projection's and the adapters' output, each rounded; the weights' own rounding is in W
    near(m.hidden, hidden.detach(), 2.0)
    near(m.loss, loss.detach(), 4.0)
    near(m.dX, dX, 6.0)
    near(m.dA, dA, 6.0)
    near(m.dB, dB, 6.0)


def test_gradients_against_differences():
    """The loss of the whole step moves along the gradient as its length says."""
    m = Model(600, 512, 384, 2000, 16, 3)
    m.step()
    keep, grads = [m.A.clone(), m.B.clone()], [m.dA.clone(), m.dB.clone()]
    length = float(sum(g.double().square().sum() for g in grads)) ** 0.5
    moved, losses = [], []
    for sign in (0.5, -0.5):
        for param, k, g in zip((m.A, m.B), keep, grads):
            param.copy_((k.float() + sign * g / length).bfloat16())
        moved.append([t.double() for t in (m.A, m.B)])
        m.step()
        losses.append(float(m.loss.double().sum()) / m.n)
    change = losses[0] - losses[1]
    want = sum(float((g.double() * (x - y)).sum()) for g, x, y in zip(grads, *moved))
    assert 0.9 * length < want < 1.1 * length                          # (the moves are rounded to bf16; what was moved counts)
    # Half a unit either way, against adapters of length 12: third-order terms are below (0.5 / 12)^2 of the change, second-order ones cancel but for the moves'
    # rounding.  Hidden states are rounded by half a step of their spread (below 2), independently in every token.
    assert abs(change - want) <= 0.02 * abs(want) + 4 * HALF_BF16 / m.n ** 0.5


def test_captured_step_with_the_optimizer():
    m = Model(500, 512, 384, 2000, 16, 3)
    zeros = lambda ts: [torch.zeros_like(t, dtype=torch.float32) for t in ts]  # noqa: E731
    params = [m.A, m.B]
    mom, var = zeros(params), zeros(params)
    opt = ql.adamw_desc(params, [m.dA, m.dB], mom, var, master=[p.float() for p in params])
    norm, ws = torch.empty(2, device="cuda"), torch.empty(ql.GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    number = torch.ones(1, dtype=torch.int32, device="cuda")

    def train():
        m.step()
        ql.qlora_grad_norm(opt, 1.0, 1.0, norm, ws)
        ql.qlora_adamw(opt, 1e-3, number, norm)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        train()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        train()
    for i in range(2, 5):
        number.fill_(i)
        m.adapter_of.copy_(m.adapter_of.roll(40))
        graph.replay()
    torch.cuda.synchronize()
    assert ql.qlora_device_status() == 0
    assert all(torch.isfinite(t.float()).all() for t in (*params, *mom, *var, norm, m.loss))
    used = torch.unique(m.adapter_of[m.adapter_of >= 0]).long()
    assert all((mom[0][a] != 0).any() and (var[1][a] > 0).any() for a in used)
