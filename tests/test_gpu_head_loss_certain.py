"""Tokens that are almost certain, with the label anywhere in the vocabulary, among the first entries (which the reference comes from) as well: their
small losses and gradients keep their digits."""
import pytest
import torch

import paper_2306_08162_b200 as ql
from test_gpu_head_loss import check, problem, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("label", [0, 100, 255, 256, 2999])
@pytest.mark.parametrize("T", [5, 600])
def test_the_label_up_to_80_above_all_others(T, label):
    V, D = 3000, 64
    hidden, head, labels, d_loss = problem(T, V, D, near=0.0, std=0.1)
    head[:, 0] = 0.0
    head[label, 0] = 8.0
    hidden[:, 0] = torch.linspace(0, 10, T, device="cuda").bfloat16()
    labels = torch.full((T,), label, dtype=torch.int32, device="cuda")
    loss, grad = run(hidden, head, labels, d_loss)
    assert ql.qlora_device_status() == 0
    assert 0 < float(loss.min()) < 1e-28
    check(hidden, head, labels, d_loss, loss, grad)
    check(hidden, head, labels, None, run(hidden, head, labels)[0])


@pytest.mark.parametrize("V,label", [(1, 0), (2, 1), (256, 7), (3000, 7)])
def test_a_label_of_any_size_above_the_first_others(V, label):
    """500 above them, which is computed twice: a loss of 0, and no NaN."""
    hidden, head, labels, d_loss = problem(40, V, 64, near=0.0, std=0.1)
    head[:, 0] = 0.0
    head[label, 0] = 50.0
    hidden[:, 0] = 10.0
    hidden[::4, 0] = 0.125                                                           # and some that are ordinary
    labels = torch.full((40,), label, dtype=torch.int32, device="cuda")
    loss, grad = run(hidden, head, labels, d_loss)
    assert ql.qlora_device_status() == 0
    check(hidden, head, labels, d_loss, loss, grad)
