"""Cross entropy of the head from the hidden states on the GPU against float64 (computed on the GPU by torch): sizes of every kind, labels that are
missing, logits of any size, tokens that are almost certain."""
import pytest
import torch

import paper_2306_08162_b200 as ql
from gpu_util import agree, canaries_intact, guarded

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -23           # a step of the fp32 sums of products, which may be cut off rather than rounded
HALF_BF16 = 2.0 ** -8
LOSS = 2.0 ** -16          # exponentials (2^-22 each, arguments below 128 rounded to 2^-17 at most), their sums and the logarithm


def problem(T, V, D, missing=0.0, seed=0, near=2.0, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed + T + V + D)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    head = (randn(V, D) / D ** 0.5).bfloat16()
    labels = torch.randint(0, V, (T,), device="cuda", generator=gen)
    hidden = (std * randn(T, D) + near * torch.rand((T, 1), device="cuda", generator=gen) * head[labels].float() * 4).bfloat16()
    gone = torch.rand((T,), device="cuda", generator=gen) < missing
    labels[gone] = torch.tensor([-1, V, -100, 2 ** 31 - 1], device="cuda")[torch.arange(T, device="cuda") % 4][gone]
    d_loss = torch.rand((T,), device="cuda", generator=gen) - 0.3
    return hidden, head, labels.int(), d_loss


def run(hidden, head, labels, d_loss=None, d_hidden=None, ws=None, stream=None):
    T, D = hidden.shape
    size = ql.qlora_head_loss_workspace_bytes(T, head.shape[0], D, d_loss is not None)
    if ws is None:
        ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")            # (NaN wherever it is read unwritten)
    loss = torch.full((T,), float("nan"), device="cuda")
    if d_loss is not None and d_hidden is None:
        d_hidden = torch.full_like(hidden, float("nan"))
    ql.qlora_head_loss(hidden, head, labels, loss, ws, d_loss=d_loss, d_hidden=d_hidden, stream=stream)
    return loss, d_hidden


def check(hidden, head, labels, d_loss, loss, grad=None, rows=slice(None)):
    h, w, V, D = hidden[rows].double(), head.double(), head.shape[0], head.shape[1]
    z = h @ w.t()
    off_z = ((D / 16 + 16) * U32 * (h.abs() @ w.abs().t())).amax(1)                  # (a product's sum takes D / 16 steps)
    lab = labels[rows].long()
    known = (lab >= 0) & (lab < V)
    at = lab.clamp(0, V - 1)[:, None]
    rest = z.scatter(1, at, float("-inf"))
    m = rest.amax(1, keepdim=True).clamp_min(-1e300)
    others = (rest - m).exp().sum(1).log() + m.squeeze(1)                           # log of the sum without the label
    odds = others - z.gather(1, at).squeeze(1)
    want = torch.where(known, torch.nn.functional.softplus(odds, threshold=1000), 0.0)
    # a loss moves with the odds by at most (1 - p) <= min(1, loss), in proportion to it where it is small
    agree(loss[rows], want.cpu().numpy(), ((2 * off_z + LOSS * (1 + odds.abs().clamp_max(1000))) * want.clamp_max(1.0) + 1e-38).cpu().numpy(), LOSS)
    if grad is None:
        return
    wrong = (-torch.nn.functional.softplus(-odds, threshold=1000)).exp()             # 1 - p of the label
    share = torch.where(rest > float("-inf"), (rest - others[:, None]).exp() * wrong[:, None], 0.0)
    f = torch.where(known, d_loss[rows].double(), 0.0)[:, None]
    dh = f * (share @ w - wrong[:, None] * w[at.squeeze(1)])
    size = f.abs() * (share @ w.abs() + wrong[:, None] * w[at.squeeze(1)].abs())
    off = size * (HALF_BF16 + 4 * off_z + (V / 16 + 64) * U32 + 4 * LOSS)[:, None]   # probabilities as bf16, their products' sums over the vocabulary
    agree(grad[rows], dh.cpu().numpy(), (off * (1 + HALF_BF16) + 1e-38).cpu().numpy(), HALF_BF16)


SIZES = [(1, 1, 64, 0.0), (1, 300, 64, 0.0), (3, 257, 72, 0.0), (16, 5000, 512, 0.2), (129, 4096, 200, 0.0), (256, 4097, 136, 0.0), (257, 9001, 256, 0.5),
         (300, 12345, 328, 1.0), (700, 50021, 128, 0.33), (1500, 255, 1000, 0.1), (2049, 4100, 72, 0.0), (2500, 300, 64, 0.0), (5000, 9000, 64, 0.1), (2304, 12300, 264, 0.0),
         (70, 600, 8200, 0.0), (20000, 300, 72, 0.2)]


@pytest.mark.parametrize("T,V,D,missing", SIZES)
def test_loss_alone(T, V, D, missing):
    hidden, head, labels, _ = problem(T, V, D, missing)
    loss, _ = run(hidden, head, labels)
    assert ql.qlora_device_status() == 0
    check(hidden, head, labels, None, loss)


@pytest.mark.parametrize("T,V,D,missing", SIZES)
def test_loss_and_gradient(T, V, D, missing):
    hidden, head, labels, d_loss = problem(T, V, D, missing)
    out, raw = guarded((T, D), torch.bfloat16)
    loss, grad = run(hidden, head, labels, d_loss, out)
    assert ql.qlora_device_status() == 0 and canaries_intact(raw, (T, D), torch.bfloat16)
    check(hidden, head, labels, d_loss, loss, grad)


def test_a_model_of_7b():
    hidden, head, labels, d_loss = problem(2048, 32000, 4096, 0.1, near=3.0)
    loss, grad = run(hidden, head, labels, d_loss)
    check(hidden, head, labels, d_loss, loss, grad, slice(0, None, 37))
    alone, _ = run(hidden, head, labels)
    check(hidden, head, labels, None, alone, None, slice(0, None, 37))


def test_exact_logits():
    """Hidden states and weights whose products are whole numbers: what is left is the error of exponentials, sums and logarithm."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    T, V, D = 300, 6000, 1024
    head = torch.randint(-1, 2, (V, D), device="cuda", generator=gen).bfloat16()
    hidden = (torch.randint(0, 64, (T, D), device="cuda", generator=gen) == 0).bfloat16()
    labels = torch.randint(0, V, (T,), device="cuda", generator=gen).int()
    for d_loss in (None, torch.ones(T, device="cuda")):
        loss, _ = run(hidden, head, labels, d_loss)
        want = torch.nn.functional.cross_entropy(hidden.double() @ head.double().t(), labels.long(), reduction="none")
        agree(loss, want.cpu().numpy(), 0.0, 2.0 ** -18)


@pytest.mark.parametrize("T", [5, 600])
def test_tokens_that_are_almost_certain(T):
    """The label's logit up to 80 above all others: losses down to 1e-34 and their gradients keep their digits."""
    V, D = 3000, 64
    hidden, head, labels, d_loss = problem(T, V, D, near=0.0, std=0.1)
    head[:, 0] = 0.0
    head[1000, 0] = 8.0
    hidden[:, 0] = torch.linspace(0, 10, T, device="cuda").bfloat16()
    labels = torch.full((T,), 1000, dtype=torch.int32, device="cuda")
    loss, grad = run(hidden, head, labels, d_loss)
    assert float(loss.min()) < 1e-28 and float(loss.min()) > 0
    check(hidden, head, labels, d_loss, loss, grad)
    check(hidden, head, labels, None, run(hidden, head, labels)[0])


@pytest.mark.parametrize("scale", [30.0, 1e4, 3e8])
def test_logits_of_any_size(scale):
    hidden, head, labels, d_loss = problem(700, 5000, 64, 0.1)
    hidden = (hidden.float() * scale).bfloat16()
    h = hidden.double()
    loss, grad = run(hidden, head, labels, d_loss)
    z = h @ head.double().t()
    known = (labels >= 0) & (labels < 5000)
    want = torch.nn.functional.cross_entropy(z, labels.long().clamp(0, 4999), reduction="none") * known
    # losses of this size follow the logits' own rounding
    off = 2 * (64 / 16 + 16) * U32 * (h.abs() @ head.double().abs().t()).amax(1) + LOSS
    agree(loss, want.cpu().numpy(), off.cpu().numpy(), LOSS)
    assert torch.isfinite(grad.float()).all()
    agree(run(hidden, head, labels)[0], want.cpu().numpy(), off.cpu().numpy(), LOSS)


@pytest.mark.parametrize("T,which", [(40, slice(None)), (1100, slice(300, 700, 7))])
def test_far_above_the_first_logits(T, which):
    """Tokens whose largest logits lie hundreds above those of the first 256 entries, among others that are not so."""
    V, D = 9000, 128
    hidden, head, labels, d_loss = problem(T, V, D, 0.1)
    head[:, 3] = 0.0
    head[:256, 3] = -8.0
    head[5000, 3] = 2.0
    hidden[:, 3] = 0.0
    hidden[which, 3] = 30.0                                                          # -240 at the beginning, 60 at one place
    loss, grad = run(hidden, head, labels, d_loss)
    assert ql.qlora_device_status() == 0
    check(hidden, head, labels, d_loss, loss, grad)
    twice = run(hidden, head, labels, d_loss)
    assert torch.equal(loss, twice[0]) and torch.equal(grad, twice[1])
    check(hidden, head, labels, None, run(hidden, head, labels)[0])


def test_what_is_not_finite_stays_with_its_token():
    hidden, head, labels, d_loss = problem(520, 5000, 256)
    clean = run(hidden, head, labels, d_loss)
    hidden[7, 5], hidden[300, 0], hidden[511, 9] = float("nan"), float("inf"), float("-inf")
    loss, grad = run(hidden, head, labels, d_loss)
    bad = torch.zeros(520, dtype=torch.bool, device="cuda")
    bad[[7, 300, 511]] = True
    assert torch.isnan(loss[bad]).all() and torch.isnan(grad[bad].float()).all()
    assert torch.equal(loss[~bad], clean[0][~bad]) and torch.equal(grad[~bad], clean[1][~bad])
    alone, _ = run(hidden, head, labels)
    assert torch.isnan(alone[bad]).all() and torch.isfinite(alone[~bad]).all()
    labels[bad] = -1                                                                 # without a label they are nobody's
    loss, grad = run(hidden, head, labels, d_loss)
    assert (loss[bad] == 0).all() and (grad[bad] == 0).all() and torch.isfinite(grad.float()).all()


def test_gradient_in_place_zero_upstream_and_the_same_bits():
    hidden, head, labels, d_loss = problem(777, 6000, 264, 0.3)
    d_loss[::5] = 0.0
    loss, grad = run(hidden, head, labels, d_loss)
    assert (grad[::5] == 0).all()
    ws = torch.randint(0, 256, (ql.qlora_head_loss_workspace_bytes(777, 6000, 264, True),), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        again = hidden.clone()
        loss2, _ = run(again, head, labels, d_loss, again, ws)
        assert torch.equal(loss, loss2) and torch.equal(grad, again)


def test_no_token_at_all():
    hidden, head, labels, d_loss = problem(4, 300, 64)
    none = hidden[:0]
    loss, grad = run(none, head, labels[:0], d_loss[:0])
    assert loss.numel() == 0
    labels[:] = -1
    loss, grad = run(hidden, head, labels, d_loss)
    assert (loss == 0).all() and (grad == 0).all()


@pytest.mark.parametrize("T,V", [(40, 9000), (900, 5000)])
def test_captured_and_replayed_for_another_batch(T, V):
    hidden, head, labels, d_loss = problem(T, V, 192, 0.2)
    ws = torch.zeros(ql.qlora_head_loss_workspace_bytes(T, V, 192, True), dtype=torch.uint8, device="cuda")
    loss, grad = torch.empty(T, device="cuda"), torch.empty_like(hidden)
    call = lambda: ql.qlora_head_loss(hidden, head, labels, loss, ws, d_loss=d_loss, d_hidden=grad)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for missing in (0.7, 0.0, 0.3):
        other = problem(T, V, 192, missing, seed=int(10 * missing) + 1)
        hidden.copy_(other[0])
        labels.copy_(other[2])
        graph.replay()
        torch.cuda.synchronize()
        got = loss.clone(), grad.clone()
        call()
        assert torch.equal(got[0], loss) and torch.equal(got[1], grad)
        check(hidden, head, labels, d_loss, loss, grad)


def test_several_at_once_on_their_own_streams():
    problems = [problem(T, V, D, 0.1) for T, V, D in ((30, 9000, 512), (600, 20000, 256), (2100, 5000, 256), (300, 40000, 128))]
    want = [run(*p) for p in problems]
    streams = [torch.cuda.Stream() for _ in problems]
    spaces = [torch.zeros(ql.qlora_head_loss_workspace_bytes(p[0].shape[0], p[1].shape[0], p[0].shape[1], True), dtype=torch.uint8, device="cuda") for p in problems]
    losses, grads = [torch.zeros_like(w[0]) for w in want], [torch.zeros_like(w[1]) for w in want]
    torch.cuda.synchronize()
    for _ in range(10):
        for p, s, ws, a, b in zip(problems, streams, spaces, losses, grads):
            ql.qlora_head_loss(p[0], p[1], p[2], a, ws, d_loss=p[3], d_hidden=b, stream=s)
    torch.cuda.synchronize()
    assert ql.qlora_device_status() == 0
    for w, a, b in zip(want, losses, grads):
        assert torch.equal(w[0], a) and torch.equal(w[1], b)


def test_the_gradient_is_that_of_differences():
    """Against differences of the loss itself, along directions that change it enough to be seen."""
    hidden, head, labels, _ = problem(64, 2000, 64, near=1.0)
    one = torch.ones(64, device="cuda")
    _, grad = run(hidden, head, labels, one)
    gen = torch.Generator(device="cuda").manual_seed(1)
    step = (2.0 ** -4) * torch.randint(-1, 2, hidden.shape, device="cuda", generator=gen).float()
    up, down = (hidden.float() + step).bfloat16(), (hidden.float() - step).bfloat16()
    change = (run(up, head, labels)[0] - run(down, head, labels)[0]).double()
    moved = up.double() - down.double()
    want = (grad.double() * moved).sum(1)
    # the logits move by |moved . w| / 2 about the middle: second-order terms cancel but for the middle's own shift, third-order ones are below its cube
    reach = (moved / 2 @ head.double().t()).abs().amax(1)
    middle = ((up.double() + down.double()) / 2 - hidden.double()).abs() @ head.double().abs().amax(0)
    rounding = 2 * HALF_BF16 * (grad.double().abs() * moved.abs()).sum(1) + 2 * HALF_BF16 * moved.abs().sum(1) * head.double().abs().amax()
    assert ((change - want).abs() <= reach ** 3 + 4 * reach * middle + rounding + 1e-5).all()


@pytest.mark.parametrize("missing", [0.0, 0.4])
def test_hidden_states_beyond_2_31_elements(missing):
    T, V, D = 530000, 300, 4104
    head = problem(1, V, D)[1]
    gen = torch.Generator(device="cuda").manual_seed(3)
    hidden = torch.empty((T, D), dtype=torch.bfloat16, device="cuda")
    for part in hidden.split(50000):
        part.copy_(torch.randn(part.shape, device="cuda", generator=gen))
    labels = torch.randint(0, V, (T,), device="cuda", generator=gen)
    labels[torch.rand(T, device="cuda", generator=gen) < missing] = -1
    labels, d_loss = labels.int(), torch.rand(T, device="cuda", generator=gen)
    loss, grad = run(hidden, head, labels, d_loss)
    assert ql.qlora_device_status() == 0
    for rows in (slice(0, 40), slice(265000, 265040), slice(T - 400, T)):
        check(hidden, head, labels, d_loss, loss, grad, rows)
