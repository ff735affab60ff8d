"""Blocks of tokens that are done again (a logit far above those of the first 256 entries) in some chunks of 2048 rows and not in others."""
import pytest
import torch

import paper_2306_08162_b200 as ql
from test_gpu_head_loss import check, problem, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,V,D,blocks", [(6144, 32000, 512, (3, 19)), (8192, 32000, 4096, (0, 16)), (6144, 50021, 2568, (2, 18)), (5000, 50021, 264, (0, 14)), (16384, 9000, 512, (5, 21, 45, 61))])
def test_the_first_and_the_third_chunk_again(T, V, D, blocks):
    hidden, head, labels, d_loss = problem(T, V, D)
    head[:, 3] = 0.0
    head[:256, 3] = -8.0
    head[V // 2:V // 2 + 9, 3] = 2.0
    hidden[:, 3] = 0.0
    for b in blocks:
        hidden[256 * b + 5:min(256 * b + 256, T):50, 3] = 30.0                       # -240 at the beginning, 60 in the middle
    loss, grad = run(hidden, head, labels, d_loss)
    assert ql.qlora_device_status() == 0
    for b in blocks:
        check(hidden, head, labels, d_loss, loss, grad, slice(256 * b, min(256 * b + 256, T)))
    check(hidden, head, labels, d_loss, loss, grad, slice(0, None, 151))
    for _ in range(6):
        again = run(hidden, head, labels, d_loss)
        assert torch.equal(loss, again[0]) and torch.equal(grad, again[1])
