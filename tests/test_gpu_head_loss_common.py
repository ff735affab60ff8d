"""The head's gradient where all rows of the head share a component, as those of trained models do: the weights of the rows add up to nothing, so the
component leaves the gradient, and the error is measured by what is left."""
import pytest
import torch

import paper_2306_08162_b200 as ql
from gpu_util import agree
from test_gpu_head_loss import HALF_BF16, LOSS, U32, run

pytestmark = pytest.mark.gpu


def problem(T, V, D, common, std, near):
    gen = torch.Generator(device="cuda").manual_seed(T + V + D)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    own = randn(V, D) / D ** 0.5
    head = (own + common * randn(D) / D ** 0.5).bfloat16()
    labels = torch.randint(0, V, (T,), device="cuda", generator=gen)
    hidden = (std * randn(T, D) + near * torch.rand((T, 1), device="cuda", generator=gen) * own[labels]).bfloat16()
    return hidden, head, labels.int(), torch.rand((T,), device="cuda", generator=gen) + 0.1


@pytest.mark.parametrize("common", [0.0, 5.0, 20.0])
@pytest.mark.parametrize("T,V,D,std,near", [(256, 4000, 512, 4.0, 8.0), (40, 12000, 256, 3.0, 4.0), (600, 9001, 200, 1.0, 0.0)])
def test_what_all_rows_share_cancels(T, V, D, std, near, common):
    hidden, head, labels, d_loss = problem(T, V, D, common, std, near)
    _, grad = run(hidden, head, labels, d_loss)
    assert ql.qlora_device_status() == 0
    h, w, at = hidden.double(), head.double(), labels.long()[:, None]
    z = h @ w.t()
    off_z = ((D / 16 + 16) * U32 * (h.abs() @ w.abs().t())).amax(1, keepdim=True)    # (a product's sum takes D / 16 steps)
    p = torch.softmax(z, 1)
    wrong = 1 - p.gather(1, at)
    q = torch.softmax(z.scatter(1, at, float("-inf")), 1)                            # of the others, among themselves
    middle = q @ w
    dh = d_loss[:, None].double() * wrong * (middle - w[at.squeeze(1)])
    spread = torch.stack([q[t] @ (w - middle[t]).abs() for t in range(T)])           # sum_v q_v |W_v - middle|
    # a weight off by d_v in relation moves the row by q_v (d_v - mean d) W_v, which is q_v d_v (W_v - middle): the rounding of P, its exponent and exponential;
    # the fp32 sums over the vocabulary, cut off rather than rounded, see the rows as they are, and so do the two weights' own roundings
    off = (HALF_BF16 + 4 * off_z + 4 * LOSS) * spread + (V / 16 + 64) * U32 * (q @ w.abs() + w[at.squeeze(1)].abs())
    off = d_loss[:, None].double() * wrong * off * (1 + 2 * HALF_BF16) + (HALF_BF16 + 4 * off_z + 4 * LOSS) * dh.abs() + 1e-38
    agree(grad, dh.cpu().numpy(), off.cpu().numpy(), 0.0)
    # a token's error in relation to its gradient: no more than two roundings to bf16, P's and the result's
    assert ((grad.double() - dh).norm(dim=1) <= 2 * HALF_BF16 * dh.norm(dim=1)).all()
