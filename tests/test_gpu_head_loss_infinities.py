"""Infinite logits: the label's alone, another's, all of them.  Losses and gradients are those of the formula in 64 bits (through the
logarithm of the softmax), infinities and NaN among them."""
import pytest
import torch

import paper_2306_08162_b200 as ql
from gpu_util import agree
from test_gpu_head_loss import HALF_BF16, LOSS, U32, problem, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("T,V,D,row", [(64, 5000, 128, 3), (300, 5000, 128, 4500), (600, 600, 72, 0), (20, 2, 64, 1)])
def test_a_row_of_the_head_with_an_infinity(T, V, D, row, sign):
    hidden, head, labels, d_loss = problem(T, V, D, seed=4)
    hidden[:, 5] = torch.where(hidden[:, 5] >= 0, 0.5, -0.5).bfloat16()
    labels[::3] = row                                                                # the label's own logit, or that of an entry like any other
    d_loss[::7] = 0.0
    bare = head.clone()
    bare[row] = 0.0
    head[row, 5] = sign * float("inf")
    h, w, at, f = hidden.double(), head.double(), labels.long(), d_loss.double()[:, None]
    z = h @ w.t()
    assert torch.isinf(z[:, row]).all() and torch.isfinite(z[:, torch.arange(V, device="cuda") != row]).all()
    log_p = torch.log_softmax(z, 1)                                                  # (NaN where infinity meets infinity)
    want_loss, p = -log_p.gather(1, at[:, None]).squeeze(1), log_p.exp()
    want = f * (p @ w - w[at])
    want = torch.where(f == 0, 0.0, want)
    above = z[:, row] > 0
    assert torch.isnan(want_loss[above]).all() and torch.isnan(want[above & (d_loss != 0)]).all()
    below = ~above & (labels == row)
    assert torch.isposinf(want_loss[below]).all() and torch.isfinite(want_loss[~above & (labels != row)]).all()
    # how far off the others may be: logits by D / 16 + 16 steps, weights by that and by the rounding of P (the infinite row has none)
    off_z = ((D / 16 + 16) * U32 * (h.abs() @ bare.double().abs().t())).amax(1)
    off_loss = 2 * off_z + LOSS * (1 + want_loss.abs())
    size = f.abs() * (torch.nan_to_num(p) @ bare.double().abs() + bare.double()[at].abs() + head.double().nan_to_num(posinf=0.0, neginf=0.0)[at].abs())
    off = size * (HALF_BF16 + 4 * off_z + (V / 16 + 64) * U32 + 4 * LOSS)[:, None] * (1 + HALF_BF16) + 1e-38
    loss, grad = run(hidden, head, labels, d_loss)
    assert ql.qlora_device_status() == 0
    agree(loss, want_loss, off_loss.nan_to_num(posinf=0.0).cpu().numpy(), LOSS)
    agree(grad, want, off.cpu().numpy(), HALF_BF16)
    agree(run(hidden, head, labels)[0], want_loss, off_loss.nan_to_num(posinf=0.0).cpu().numpy(), LOSS)


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_one_entry_and_an_infinite_hidden_value(value):
    hidden, head, labels, d_loss = problem(4, 1, 64)
    hidden[1, 9] = value
    loss, grad = run(hidden, head, labels, torch.ones_like(d_loss))
    assert torch.isnan(loss[1]) and torch.isnan(grad[1].float()).all()
    others = torch.tensor([0, 2, 3], device="cuda")
    assert (loss[others] == 0).all() and (grad[others] == 0).all()
    alone, _ = run(hidden, head, labels)
    assert torch.isnan(alone[1]) and (alone[others] == 0).all()


def test_every_logit_minus_infinity():
    hidden, head, labels, d_loss = problem(6, 700, 64)
    head[:, 9] = 1.0
    hidden[2, 9] = float("-inf")
    loss, grad = run(hidden, head, labels, torch.ones_like(d_loss))
    assert torch.isnan(loss[2]) and torch.isnan(grad[2].float()).all()
    alone, _ = run(hidden, head, labels)
    assert torch.isnan(alone[2]) and torch.isfinite(alone[[0, 1, 3, 4, 5]]).all()
