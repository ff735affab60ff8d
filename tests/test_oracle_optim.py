"""Pins for the oracle's AdamW step, its 8-bit states and the clipping factor: CPU only."""
import math

import numpy as np
import torch

from oracle import qlora_oracle as orc


def test_step_by_hand_and_against_an_independent_implementation():
    # the first step from zero moments is lr * g / (|g| + eps), whatever the betas
    w, m, v = orc.adamw_step([1.0], [0.25], [0.0], [0.0], 1, 0.1, 0.9, 0.999, 1e-8, 0.0)
    assert abs(w[0] - (1.0 - 0.1 * 0.25 / (0.25 + 1e-8))) < 1e-12 and abs(m[0] - 0.025) < 1e-15 and abs(v[0] - 0.0000625) < 1e-15
    rng = np.random.default_rng(1)
    p = torch.nn.Parameter(torch.from_numpy(rng.standard_normal(50)))
    opt = torch.optim.AdamW([p], lr=3e-3, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    w, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for step in range(1, 6):
        g = rng.standard_normal(50)
        p.grad = torch.from_numpy(g.copy())
        opt.step()
        w, m, v = orc.adamw_step(w, g, m, v, step, 3e-3, 0.8, 0.95, 1e-6, 0.1)
        assert np.allclose(w, p.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_clipping_factor():
    g = [np.array([3.0]), np.array([[0.0, 4.0]])]
    assert orc.grad_norm(g, 1.0, 0.0) == (5.0, 1.0)
    assert orc.grad_norm(g, 0.5, 10.0) == (2.5, 0.5)
    assert orc.grad_norm(g, 2.0, 1.0) == (10.0, 0.2)
    norm, f = orc.grad_norm([np.array([np.inf])], 1.0, 1.0)
    assert math.isinf(norm) and math.isnan(f)


def test_e4m3_neighbours_and_their_chance():
    codes = torch.arange(0, 0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()      # 0 .. 448
    assert np.array_equal(orc.dithered_e4m3(codes, np.zeros(codes.size)), codes) and np.array_equal(orc.dithered_e4m3(-codes, np.full(codes.size, 2 ** 20 - 1)), -codes)
    rng = np.random.default_rng(2)
    x = np.exp(rng.uniform(math.log(2.0 ** -11), math.log(448.0), 2000))
    lo, hi = orc.dithered_e4m3(x, np.zeros(x.size)), orc.dithered_e4m3(x, np.full(x.size, 2 ** 20 - 1))
    at = np.searchsorted(codes, x, side="right") - 1
    assert np.array_equal(lo, codes[at]) and np.array_equal(hi, codes[np.minimum(at + 1, codes.size - 1)])
    # over the steps the mean is the value: 4000 draws of a step of size u have a deviation of at most u / 2 / sqrt(4000)
    for value in (0.003, 0.77, 100.0):
        mean = np.mean([orc.dithered_e4m3(value, orc.dither(np.array([1234]), step)[0][0]) for step in range(1, 4001)])
        assert abs(mean - value) < 5 * orc.e4m3_step(value) / 2 / math.sqrt(4000)
    for r in orc.dither(np.arange(100000), 7):                                   # uniform over places: 5 deviations of the mean and of each of 16 bins
        assert r.min() >= 0 and r.max() < 2 ** 20 and abs(r.mean() / 2 ** 20 - 0.5) < 5 * math.sqrt(1 / 12 / 1e5)
        assert np.abs(np.bincount(r >> 16, minlength=16) - 6250).max() < 5 * math.sqrt(6250)


def test_blocks_in_8_bits():
    rng = np.random.default_rng(3)
    x = rng.standard_normal(700) * np.repeat([1e-3, 1e-6, 0.0], 256)[:700]
    r = orc.dither(np.arange(700), 3)[0]
    codes, scales = orc.held_in_8_bits(x, r)
    assert scales.shape == (3,) and scales[2] == 0 and (codes[512:] == 0).all()
    held = codes * np.repeat(scales, 256)[:700]
    assert (np.abs(held - x) <= np.repeat(scales, 256)[:700] * orc.e4m3_step(codes) * 1.0000001).all()
    u = np.abs(x)
    u[0], u[1] = 1e-12, 0.0
    codes, scales = orc.held_in_8_bits(u, r, root=True)
    assert codes[0] == 2.0 ** -9 and codes[1] == 0.0
