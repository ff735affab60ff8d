"""The AdamW step where one of its terms is very small beside the others (needs a B200).

Weight decay far below half a step of the weight's type: it has to be right in the mean over many weights (u = 2^-24).  A weight is rounded once, off by at
most u |w| with a sign that has nothing to do with the weight's, as the update that is rounded with it is tens of steps large and random: over
n = 2^20 weights the mean is off by u rms(w) / 1024 = 7.3e-11 of the mean |w| in standard deviation, six of them 4.4e-10.  The update's own errors are at most
24u of it, with mean |update| <= 8 lr mean |w|: 1.8e-10.  So the mean change towards zero is off by less than 1e-9 of the mean |w|.

Gradients whose squares are near fp32's smallest numbers, or below its normal range: v = beta2 v + (1 - beta2) g^2 >= 5e-39 is formed with three roundings, each of u
relatively and 2^-150 (4.2e-7 / 3 = 2.4u of 5e-39) absolutely, so v is off by at most 11u and its root by 5.5u; this comes on top of what the step has with
ordinary gradients (24u of the update, 4u of the moments' terms, 8u of the scales)."""
import numpy as np
import pytest
import torch

import paper_2306_08162_b200 as ql
from gpu_util import to_f64
from oracle import qlora_oracle as orc
from test_gpu_optim import Model

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


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


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("fresh", [True, False])
@pytest.mark.parametrize("sizes", [[3000], [256, 77, 2048]], ids=str)
def test_gradients_near_the_smallest_numbers(sizes, fresh, bits):
    """Updates are of the size of the rate whatever the gradients' size, as eps is far smaller still; a root above zero has a code above zero."""
    lr, step = 1e-2, 1 if fresh else 30
    m = Model(sizes, param="fp32", bits=bits, fresh=fresh, seed=43, eps=1e-30, weight_decay=0.0)
    for j in range(len(sizes)):
        m.grad[j].copy_(torch.where(m.grad[j] < 0, -1e-18, 1e-18) * (1 + torch.rand_like(m.grad[j])))
        if bits == 8:
            m.v[j].copy_(m.v[j].float().clamp_min(0.0 if fresh else 32.0).to(m.v[j].dtype))
            m.m_scale[j].mul_(1e-18)
            m.v_scale[j].mul_(1e-18)
        else:
            m.m[j].mul_(1e-18)
            m.v[j].mul_(1e-36)
    want, before = m.expected(step, lr), [to_f64(t) for t in m.param]
    ql.qlora_adamw(m.desc, lr, step)
    for j, (w, mj, v, terms) in enumerate(want):
        assert v.min() >= 4.9e-39
        off = 30 * U * np.abs(w - before[j]) + 4 * U * terms + 4 * U * np.abs(before[j])
        assert (np.abs(to_f64(m.param[j]) - w) <= off + U * (np.abs(w) + off)).all()
        if bits == 32:
            assert (np.abs(to_f64(m.v[j]) - v) <= 11 * U * v).all()
            continue
        place = np.arange(sizes[j])
        codes, scales = orc.held_in_8_bits(np.sqrt(v), orc.dither(place, step)[1], True)
        got = to_f64(m.v[j].float())
        assert (np.abs(to_f64(m.v_scale[j]) - scales) <= 14 * U * scales).all() and (got > 0).all()
        assert np.mean(got != codes) <= 2.0 ** -10 + 1.5 / sizes[j]
        assert (np.abs(got - codes) <= np.maximum(orc.e4m3_step(got), orc.e4m3_step(codes))).all()
