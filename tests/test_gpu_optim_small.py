"""The AdamW step where one of its terms is very small beside the others (needs a B200).

Weight decay far below half a step of the weight's type: it has to be right in the mean over many weights (u = 2^-24).  A weight is rounded once, off by at
most u |w| with a sign that has nothing to do with the weight's, as the update that is rounded with it is tens of steps large and random: over
n = 2^20 weights the mean is off by u rms(w) / 1024 = 7.3e-11 of the mean |w| in standard deviation, six of them 4.4e-10.  The update's own errors are at most
24u of it, with mean |update| <= 8 lr mean |w|: 1.8e-10.  So the mean change towards zero is off by less than 1e-9 of the mean |w|."""
import numpy as np
import pytest
import torch

import paper_2306_08162_b200 as ql
from gpu_util import to_f64
from test_gpu_optim import Model

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("on_device", [False, True])
@pytest.mark.parametrize("lr", [2.0 ** -20, 2.0 ** -19, 2.0 ** -18, 2.0 ** -16])
def test_small_weight_decay_in_the_mean(lr, bits, master, on_device):
    m = Model([1 << 20], param="bf16" if master else "fp32", bits=bits, master=master, seed=41, weight_decay=0.01)
    if bits == 8:                                                  # (roots of a hundredth of the gradients' size and more: updates of the size of lr)
        m.v[0].copy_(m.v[0].float().clamp_min(32.0).to(m.v[0].dtype))
        m.v_scale[0].add_(0.01)
    else:
        m.v[0].add_(0.1)
    (want, _, _, _), = m.expected(50, lr)
    weights = (m.master or m.param)[0]
    before = to_f64(weights)
    rate, step = (torch.tensor([lr], device="cuda"), torch.tensor([50], dtype=torch.int32, device="cuda")) if on_device else (lr, 50)
    ql.qlora_adamw(m.desc, rate, step)
    size = np.abs(before).mean()
    assert np.abs(want - before * (1 - lr * 0.01)).mean() <= 8 * lr * size
    assert abs((np.sign(before) * (to_f64(weights) - want)).mean()) <= 1e-9 * size
