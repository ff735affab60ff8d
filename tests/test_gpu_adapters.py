"""Adapters of many requests on the GPU against float64: every rank, ragged sizes, tokens in any order, tokens without an adapter, and what must not
reach a neighbour."""
import numpy as np
import pytest
import torch

import paper_2306_08162_b200 as ql
from gpu_util import agree, canaries_intact, guarded, to_f64

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -23          # a step of the fp32 sums, which may be cut off rather than rounded
HALF_BF16 = 2.0 ** -8     # rounding to bf16, relative to the value
SPLIT = 2.0 ** -16        # a value held as two bf16


def orders(kind, M, L, gen):
    if kind == "scattered":
        ids = torch.randint(-1, L + 1, (M,), generator=gen)
    elif kind == "rows":                                               # requests in a row, adapters in several places
        cuts = torch.randint(0, M + 1, (5,), generator=gen).sort().values
        ids = torch.randint(-1, L, (6,), generator=gen)[torch.searchsorted(cuts, torch.arange(M), right=True)]
    elif kind == "each":
        ids = torch.arange(M) % L
    elif kind == "none":
        ids = torch.tensor([-1, L, -(2 ** 31), 2 ** 31 - 1])[torch.arange(M) % 4]
    else:
        ids = torch.full((M,), L - 1)
    return ids.to(torch.int32)


class Problem:
    def __init__(self, M, K, N, r, L, kind, seed=0):
        gen = torch.Generator().manual_seed(seed + 1000 * M + r)
        rand = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
        self.M, self.K, self.N, self.r, self.L = M, K, N, r, L
        self.adapter_of = orders(kind, M, L, gen).cuda()
        self.X, self.dY = rand(M, K).bfloat16().cuda(), rand(M, N).bfloat16().cuda()
        self.A, self.B = (rand(L, r, K) / K ** 0.5).bfloat16().cuda(), (0.2 * rand(L, N, r)).bfloat16().cuda()
        self.scales = (1.0 + torch.rand(L, generator=gen)).cuda()
        self.Yb, self.dXb = rand(M, N).bfloat16().cuda(), rand(M, K).bfloat16().cuda()
        self.desc = ql.adapters_desc(K, N, r, L)
        self.ws = torch.full((ql.qlora_adapters_workspace_bytes(self.desc, M),), 0xFF, dtype=torch.uint8, device="cuda")   # (NaN wherever it is read unwritten)

    def empty(self, *shape):
        return torch.full(shape, float("nan"), device="cuda")

    def forward(self, Y=None, H=None, base=None, stream=None):
        Y = torch.empty_like(self.Yb) if Y is None else Y
        ql.qlora_adapters_fwd(self.desc, self.M, self.X, self.adapter_of, self.A, self.B, self.scales, self.Yb if base is None else base, Y, H, self.ws, stream=stream)
        return Y

    def back(self, dX=None, G=None, base=None):
        dX = torch.empty_like(self.dXb) if dX is None else dX
        ql.qlora_adapters_bwd_input(self.desc, self.M, self.dY, self.adapter_of, self.A, self.B, self.scales, self.dXb if base is None else base, dX, G, self.ws)
        return dX

    def grads(self, H, G, dA=None, dB=None, accumulate=0):
        dA = self.empty(self.L, self.r, self.K) if dA is None else dA
        dB = self.empty(self.L, self.N, self.r) if dB is None else dB
        ql.qlora_adapters_bwd_lora(self.desc, self.M, self.X, self.dY, self.adapter_of, self.A, self.B, self.scales, H, G, dA, dB, accumulate, self.ws)
        return dA, dB

    def low(self, x, first):
        """What the first product gives and the sum of its terms' sizes, float64; first [L, r, T]."""
        x, first = to_f64(x), to_f64(first)
        out, size = np.zeros((self.M, self.r)), np.zeros((self.M, self.r))
        for a in range(self.L):
            mine = np.flatnonzero(self.adapter_of.cpu().numpy() == a)
            out[mine], size[mine] = x[mine] @ first[a].T, np.abs(x[mine]) @ np.abs(first[a]).T
        return out, size

    def high(self, low, size, second, base, terms):
        """The second product on top of base; second [L, r, C].  Also how far off the sum may be before it is rounded to bf16."""
        second, out = to_f64(second), to_f64(base).copy()
        off = np.zeros_like(out)
        for a in range(self.L):
            mine = np.flatnonzero(self.adapter_of.cpu().numpy() == a)
            s = float(self.scales[a])
            out[mine] += s * (low[mine] @ second[a])
            off[mine] = s * ((terms * U32) * size[mine] + (SPLIT + (self.r + 8) * U32) * np.abs(low[mine])) @ np.abs(second[a]) + 2 * U32 * np.abs(out[mine])
        return out, off


SIZES = [
    (1, 32, 8, 8, 1, "one"), (1, 4096, 4096, 16, 8, "each"), (3, 96, 40, 24, 2, "scattered"), (4, 512, 1000, 64, 4, "each"), (5, 160, 72, 8, 9, "none"),
    (17, 1024, 520, 40, 3, "scattered"), (64, 2080, 1376, 16, 64, "each"), (256, 512, 264, 32, 7, "rows"),
    (257, 32, 8, 8, 2, "scattered"), (260, 96, 1000, 64, 5, "rows"), (300, 1056, 552, 16, 300, "each"), (301, 800, 104, 24, 4, "none"),
    (149, 544, 520, 64, 40, "scattered"), (200, 1024, 264, 24, 4, "none"), (256, 96, 1000, 56, 256, "each"),
    (4100, 96, 72, 8, 40, "scattered"), (9000, 64, 40, 24, 3, "each"), (4096, 32, 264, 16, 4096, "each"),
    (513, 4096, 776, 48, 3, "rows"), (1000, 544, 2056, 8, 6, "one"), (2100, 256, 264, 56, 31, "scattered"),
]


@pytest.mark.parametrize("M,K,N,r,L,kind", SIZES)
def test_against_float64(M, K, N, r, L, kind):
    p = Problem(M, K, N, r, L, kind)
    H, G = p.empty(M, r), p.empty(M, r)
    Y, Yraw = guarded((M, N), torch.bfloat16)
    dX, dXraw = guarded((M, K), torch.bfloat16)
    p.forward(Y, H)
    p.back(dX, G)
    dA, dB = p.grads(H, G)
    assert canaries_intact(Yraw, (M, N), torch.bfloat16) and canaries_intact(dXraw, (M, K), torch.bfloat16)
    h, h_size = p.low(p.X, p.A)
    g, g_size = p.low(p.dY, p.B.transpose(1, 2))
    agree(H, h, (K + 8) * U32 * h_size, 0.0)
    agree(G, g, (N + 8) * U32 * g_size, 0.0)
    y, y_off = p.high(h, h_size, p.B.transpose(1, 2), p.Yb, K + 8)
    x, x_off = p.high(g, g_size, p.A, p.dXb, N + 8)
    agree(Y, y, y_off * (1 + HALF_BF16), HALF_BF16)
    agree(dX, x, x_off * (1 + HALF_BF16), HALF_BF16)
    ids = p.adapter_of.cpu().numpy()
    X, dY, Hf, Gf = to_f64(p.X), to_f64(p.dY), to_f64(H), to_f64(G)
    for a in range(L):
        mine = np.flatnonzero(ids == a)
        s = float(p.scales[a])
        tol = (len(mine) + 9) * U32                                    # (three bf16 hold an fp32 value)
        agree(dA[a], s * Gf[mine].T @ X[mine], s * tol * (np.abs(Gf[mine]).T @ np.abs(X[mine])), 2 * U32)
        agree(dB[a], s * dY[mine].T @ Hf[mine], s * tol * (np.abs(dY[mine]).T @ np.abs(Hf[mine])), 2 * U32)


@pytest.mark.parametrize("M", [6, 300])
def test_in_place_without_h_and_the_same_bits_again(M):
    p = Problem(M, 512, 520, 16, 3, "scattered")
    H = p.empty(M, 16)
    Y = p.forward(H=H)
    again = p.Yb.clone()
    p.forward(again, base=again)
    assert torch.equal(Y, again)
    dX, G = p.back(), p.empty(M, 16)
    again = p.dXb.clone()
    p.back(again, G, base=again)
    assert torch.equal(dX, again)
    bare = (p.adapter_of < 0) | (p.adapter_of >= 3)
    assert torch.equal(Y[bare], p.Yb[bare]) and torch.equal(dX[bare], p.dXb[bare]) and (H[bare] == 0).all() and (G[bare] == 0).all()
    # H and G formed again, and gradients added up
    first, twice = p.grads(H, G), p.grads(H, G)
    assert torch.equal(first[0], twice[0]) and torch.equal(first[1], twice[1])
    dA, dB = p.grads(None, None)
    ids, X, dY = p.adapter_of.cpu().numpy(), np.abs(to_f64(p.X)), np.abs(to_f64(p.dY))
    h_size, g_size = p.low(p.X, p.A)[1], p.low(p.dY, p.B.transpose(1, 2))[1]
    for a in range(3):                                                 # H and G may differ by twice what either may be off, their products by the sums' rounding
        mine, s = np.flatnonzero(ids == a), float(p.scales[a])
        agree(dA[a], first[0][a], 2 * s * ((520 + 8) * U32 + (len(mine) + 9) * U32) * (g_size[mine].T @ X[mine]), 0.0)
        agree(dB[a], first[1][a], 2 * s * ((512 + 8) * U32 + (len(mine) + 9) * U32) * (dY[mine].T @ h_size[mine]), 0.0)
    p.grads(H, G, twice[0], twice[1], accumulate=1)
    assert torch.equal(twice[0], 2 * first[0]) and torch.equal(twice[1], 2 * first[1])


@pytest.mark.parametrize("M", [8, 400])
def test_what_is_not_finite_stays_with_its_own(M):
    """An adapter of infinities and NaN beside others in the same tile, and a token of NaN among others of its adapter."""
    p = Problem(M, 256, 264, 16, 4, "each")
    clean = p.forward().clone(), p.back().clone(), *(t.clone() for t in p.grads(None, None))
    p.A[1, 3, 7], p.A[1, 0, 9], p.B[1, 5, 2] = float("nan"), float("inf"), float("-inf")
    p.X[2, 11] = float("nan")                                          # a token of adapter 2
    Y, dX, (dA, dB) = p.forward(), p.back(), p.grads(None, None)
    others = p.adapter_of != 1
    others[2] = False
    assert torch.equal(Y[others], clean[0][others]) and torch.isnan(Y[2]).all()
    mine = p.adapter_of == 1
    assert torch.isnan(Y[mine]).all() and not torch.isfinite(dX[mine][:, 9]).any()
    others[2] = True                                                   # (its dY is a number)
    assert torch.equal(dX[others], clean[1][others])
    for a in (0, 3):
        assert torch.equal(dA[a], clean[2][a]) and torch.equal(dB[a], clean[3][a])
    assert torch.isnan(dA[2][:, 11]).all() and torch.isfinite(dA[2][:, :11]).all()


@pytest.mark.parametrize("M", [8, 400])
def test_infinite_where_the_sum_is(M):
    p = Problem(M, 64, 40, 8, 2, "each")
    p.B[1, 3] = 0.0
    p.B[1, 3, 0] = float("inf")
    Y, H = torch.empty_like(p.Yb), p.empty(M, 8)
    p.forward(Y, H)
    mine = p.adapter_of == 1
    want = torch.where(H[mine][:, 0] > 0, float("inf"), float("-inf"))
    assert torch.equal(Y[mine][:, 3].float(), want) and torch.isfinite(Y[mine][:, 4:]).all()


def test_nothing_to_do_and_no_adapters():
    d = ql.adapters_desc(64, 40, 8, 3)
    ws = torch.empty(ql.qlora_adapters_workspace_bytes(d, 0), dtype=torch.uint8, device="cuda")
    none = lambda *s, **k: torch.empty(s, device="cuda", **k)  # noqa: E731
    X, dY, ids = none(0, 64, dtype=torch.bfloat16), none(0, 40, dtype=torch.bfloat16), none(0, dtype=torch.int32)
    A, B, s = none(3, 8, 64, dtype=torch.bfloat16), none(3, 40, 8, dtype=torch.bfloat16), none(3)
    ql.qlora_adapters_fwd(d, 0, X, ids, A, B, s, dY, dY, None, ws)
    dA, dB = torch.ones(3, 8, 64, device="cuda"), torch.ones(3, 40, 8, device="cuda")
    ql.qlora_adapters_bwd_lora(d, 0, X, dY, ids, A, B, s, None, None, dA, dB, 1, ws)
    assert (dA == 1).all() and (dB == 1).all()
    ql.qlora_adapters_bwd_lora(d, 0, X, dY, ids, A, B, s, None, None, dA, dB, 0, ws)
    assert (dA == 0).all() and (dB == 0).all()
    for M in (5, 300):                                                 # an empty set of adapters
        p = Problem(M, 64, 40, 8, 1, "one")
        e = ql.adapters_desc(64, 40, 8, 0)
        Y = torch.empty_like(p.Yb)
        ql.qlora_adapters_fwd(e, M, p.X, p.adapter_of, p.A[:0], p.B[:0], p.scales[:0], p.Yb, Y, None, p.ws)
        assert torch.equal(Y, p.Yb)


@pytest.mark.parametrize("M", [6, 300])
def test_captured_replayed_for_another_batch_on_another_stream(M):
    p = Problem(M, 512, 264, 24, 5, "rows")
    H, Y, G, dX = p.empty(M, 24), torch.empty_like(p.Yb), p.empty(M, 24), torch.empty_like(p.dXb)
    dA, dB = p.empty(5, 24, 512), p.empty(5, 264, 24)

    def step():
        p.forward(Y, H)
        p.back(dX, G)
        p.grads(H, G, dA, dB)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    p.adapter_of.copy_(orders("scattered", M, 5, torch.Generator().manual_seed(9)))
    p.X.neg_()
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (Y, H, dX, G, dA, dB)]
    step()
    for a, b in zip(got, (Y, H, dX, G, dA, dB)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("M", [6, 300, 900])
def test_everything_rewritten_in_stream_right_before_the_calls(M):
    """What a call reads is written by the kernels just before it, over and over, and so is the workspace by the calls themselves."""
    p, other = Problem(M, 512, 264, 16, 5, "rows"), Problem(M, 512, 264, 16, 5, "scattered", seed=7)
    names = ("X", "dY", "A", "B", "scales", "Yb", "dXb", "adapter_of")

    def results(q):
        H, G = q.empty(M, 16), q.empty(M, 16)
        Y, dX = q.forward(H=H), q.back(G=G)
        return [Y, H, dX, G, *q.grads(H, G), *q.grads(None, None)]
    want = []
    for q in (p, other):
        torch.cuda.synchronize()
        want.append(results(q))
        torch.cuda.synchronize()
    sources = [{n: getattr(q, n).clone() for n in names} for q in (p, other)]
    got = []
    for i in range(12):
        for n in names:
            getattr(p, n).copy_(sources[i % 2][n])
        got.append(results(p))
    for i, result in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(result, want[i % 2])), i


def test_two_streams_at_once():
    problems = [Problem(M, 1024, 520, 16, 4, "rows", seed) for seed, M in enumerate((5, 400, 64, 2000))]
    want = [p.forward().clone() for p in problems]
    streams = [torch.cuda.Stream() for _ in problems]
    torch.cuda.synchronize()
    out = [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for p, s, o in zip(problems, streams, out):
            p.forward(o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_a_long_pool_of_adapters():
    """Matrices beyond 2^31 bytes into the pool."""
    L, K, N, r = 300, 4096, 8, 64
    d = ql.adapters_desc(K, N, r, L * 30)
    A = torch.zeros((L * 30, r, K), dtype=torch.bfloat16, device="cuda")
    B = torch.zeros((L * 30, N, r), dtype=torch.bfloat16, device="cuda")
    A[-1], B[-1] = 1.0 / 64, 1.0 / 64
    scales = torch.ones(L * 30, device="cuda")
    for M in (3, 257):
        X, base = torch.ones((M, K), dtype=torch.bfloat16, device="cuda"), torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
        ids = torch.full((M,), L * 30 - 1, dtype=torch.int32, device="cuda")
        ids[1] = 0
        ws = torch.empty(ql.qlora_adapters_workspace_bytes(d, M), dtype=torch.uint8, device="cuda")
        Y = torch.empty_like(base)
        ql.qlora_adapters_fwd(d, M, X, ids, A, B, scales, base, Y, None, ws)
        assert (Y[0] == 64.0).all() and (Y[1] == 0).all() and (Y[2:] == 64.0).all()    # 64 x 64 / 64


def test_as_many_tokens_as_there_may_be():
    """2^20 tokens, whose hidden states begin beyond 2^32 elements: the last ones are right, and what the gradients sum up comes from all."""
    M, K, N, r, L = 1 << 20, 4128, 8, 8, 3
    d = ql.adapters_desc(K, N, r, L)
    X, dY = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda"), torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    X[:, 0], X[-40:] = 1.0, 0.5
    dY[:, 1], dY[-40:] = 0.5, 1.0
    A, B = (torch.full(s, 2.0 ** -9, dtype=torch.bfloat16, device="cuda") for s in ((L, r, K), (L, N, r)))
    scales = torch.full((L,), 2.0, device="cuda")
    ids = (torch.arange(M, device="cuda") // 1000 % L).int()
    ids[-5:] = 1
    ws = torch.empty(ql.qlora_adapters_workspace_bytes(d, M), dtype=torch.uint8, device="cuda")
    Y, H, G = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda"), torch.empty((M, r), device="cuda"), torch.empty((M, r), device="cuda")
    ql.qlora_adapters_fwd(d, M, X, ids, A, B, scales, Y, Y, H, ws)
    assert (H[:-40] == 2.0 ** -9).all() and (H[-40:] == K * 2.0 ** -10).all()
    assert (Y[:-40] == 2.0 ** -14).all() and (Y[-40:] == torch.tensor(K * 2.0 ** -15).bfloat16().item()).all()
    dX = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    ql.qlora_adapters_bwd_input(d, M, dY, ids, A, B, scales, dX, dX, G, ws)
    assert (G[:-40] == 2.0 ** -10).all() and (G[-40:] == 2.0 ** -6).all()
    assert (dX[-40:] == 2.0 ** -11).all() and (dX[-1000:-40] == 2.0 ** -15).all() and (dX[::1001] >= 2.0 ** -15).all()
    dA, dB = torch.empty((L, r, K), device="cuda"), torch.empty((L, N, r), device="cuda")
    ql.qlora_adapters_bwd_lora(d, M, X, dY, ids, A, B, scales, H, G, dA, dB, 0, ws)
    n, last = torch.bincount(ids, minlength=L).double(), torch.bincount(ids[-40:], minlength=L).double()
    # every addition is off by 2^-23 of the sum at most (cut off rather than rounded), and there are M / 16 in a chain at most
    near = lambda got, want: torch.testing.assert_close(got.double(), want.expand_as(got), rtol=2.0 ** -23 * M / 16, atol=0.0)  # noqa: E731
    near(dA[:, :, 0], (2.0 * ((n - last) * 2.0 ** -10 + last * 2.0 ** -7))[:, None])
    near(dA[:, :, 1:], (2.0 * last * 2.0 ** -7)[:, None, None])
    near(dB[:, 1], (2.0 * ((n - last) * 2.0 ** -10 + last * K * 2.0 ** -10))[:, None])
    near(dB[:, 2:], (2.0 * last * K * 2.0 ** -10)[:, None, None])
