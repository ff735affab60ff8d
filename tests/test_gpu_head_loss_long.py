"""The head's logits at long contractions: sums that are exact, and sums of random terms, whose expected cut-off is taken back.  A logit is read out of a
loss: with a second entry of zeros the loss is log(1 + exp(-z)), which is -z to 2^-36 for z below -25."""
import pytest
import torch

import paper_2306_08162_b200 as ql
from gpu_util import agree
from test_gpu_head_loss import run

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -23
CUT_OFF = 1.0e-9           # of a logit per feature, up to 16384 of them


def logits(hidden, row, gradient):
    """hidden . row as the kernel has it, with the value in 64 bits."""
    head = torch.stack([row, torch.zeros_like(row)])
    labels = torch.zeros(len(hidden), dtype=torch.int32, device="cuda")
    loss, _ = run(hidden, head, labels, torch.ones(len(hidden), device="cuda") if gradient else None)
    assert ql.qlora_device_status() == 0
    return -loss.double(), hidden.double() @ row.double()


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("D", [64, 4096, 8192, 16384, 65536, 1 << 18, 1 << 20])
def test_sums_that_are_exact(D, gradient):
    """One feature, and 64 of them in every token's own places: whole numbers, of which nothing is cut off."""
    T = 200 if D <= 65536 else 24
    gen = torch.Generator(device="cuda").manual_seed(D)
    row = torch.randint(0, 2, (D,), device="cuda", generator=gen) * 2.0 - 1.0
    hidden = torch.zeros((T, D), device="cuda")
    at = torch.randint(0, D, (T, 64), device="cuda", generator=gen)
    hidden.scatter_(1, at, -row[at])
    hidden[::3] = 0.0
    hidden[::3, D // 2 + 5] = -row[D // 2 + 5] * (30 + torch.arange(len(hidden[::3]), device="cuda") % 64)
    got, want = logits(hidden.bfloat16(), row.bfloat16(), gradient)
    assert (want <= -25).all()
    # a reference up to 28 away, the scale, a difference, a product, a logarithm, and log 2 again: eight roundings at most, of values up to |z| + 28
    agree(got, want.cpu().numpy(), (CUT_OFF * min(D, 16384) * want.abs() + 8 * STEP * (want.abs() + 28)).cpu().numpy(), 0.0)


@pytest.mark.parametrize("D", [2048, 4096, 8192, 16384])
def test_sums_of_random_terms_are_right_on_average(D):
    """Random terms around a drift to -60: what the sums lose is expected, and no more than a quarter of it is left."""
    T = 2048
    gen = torch.Generator(device="cuda").manual_seed(D)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    row = randn(D)
    hidden = (12 / D ** 0.5 * randn(T, D) - 60 * row / row.square().sum()).bfloat16()
    got, want = logits(hidden, row.bfloat16(), False)
    far = want < -25
    assert far.sum() > T // 2
    off = ((got - want) / want)[far]
    # (off's standard deviation over the tokens is below CUT_OFF * D, so that of its mean over a thousand is below a thirtieth of it)
    assert off.abs().mean() < CUT_OFF * D and off.mean().abs() < CUT_OFF * D / 4
