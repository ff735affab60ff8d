"""Pins for the oracle's log probabilities, entropies, alternatives and their gradient: CPU only."""
import math

import numpy as np

from oracle import qlora_oracle as orc
from helpers import rel_err


def test_against_plain_loops_and_closed_forms():
    rng = np.random.default_rng(5)
    T, V, c = 4, 11, 1.7
    z = rng.standard_normal((T, V)) * 2
    tokens = np.array([3, -1, 10, 11])
    out = orc.token_logprobs(z, tokens, c, k=3)
    for t in range(T):
        e = [math.exp(c * v) for v in z[t]]
        p = [v / sum(e) for v in e]
        assert abs(out["entropy"][t] + sum(v * math.log(v) for v in p)) < 1e-12
        want = math.log(p[tokens[t]]) if 0 <= tokens[t] < V else 0.0
        assert abs(out["logprobs"][t] - want) < 1e-12
        assert abs(out["stats"][t, 0] - max(z[t])) == 0 and abs(c * out["stats"][t, 0] + out["stats"][t, 1] - math.log(sum(e))) < 1e-12
        order = sorted(range(V), key=lambda j: (-z[t, j], j))[:3]
        assert list(out["top_ids"][t]) == order and np.allclose(out["top_logprobs"][t], [math.log(p[j]) for j in order], atol=1e-12)
    uniform = orc.token_logprobs(np.zeros((1, 8)), [2], 0.5, k=8)
    assert abs(uniform["entropy"][0] - math.log(8)) < 1e-12 and abs(uniform["logprobs"][0] + math.log(8)) < 1e-12
    assert list(uniform["top_ids"][0]) == list(range(8))                     # ties by place


def test_masked_empty_and_broken_rows():
    inf = np.inf
    z = np.array([[0.0, -inf, 1.0, -inf], [-inf] * 4, [0.0, np.nan, 1.0, -inf], [0.0, inf, 1.0, 2.0], [-0.0, 0.0, -1.0, 0.0]])
    out = orc.token_logprobs(z, [1, 0, 2, 2, 3], 1.0, k=4)
    assert out["logprobs"][0] == -inf and out["logprobs"][1] == -inf and np.isnan(out["logprobs"][2:4]).all()
    assert out["entropy"][1] == 0.0 and np.isfinite(out["entropy"][0])
    assert out["top_ids"].tolist() == [[2, 0, 1, 3], [0, 1, 2, 3], [1, 2, 0, 3], [1, 3, 2, 0], [0, 1, 3, 2]]
    grad = orc.token_logprobs_backward(z, [0, 0, 2, 2, -1], 1.0, np.ones(5), np.array([1.0, 1.0, 0.0, 0.0, 0.0]))
    assert np.isfinite(grad[0]).all() and grad[0, 1] == 0 and (grad[1] == 0).all() and np.isnan(grad[2:4]).all() and (grad[4] == 0).all()


def test_gradient_by_central_differences():
    rng = np.random.default_rng(6)
    T, V, c, eps = 3, 9, 0.6, 1e-5
    z, tokens = rng.standard_normal((T, V)), np.array([4, 0, -1])
    gl, gh = rng.standard_normal(T), rng.standard_normal(T)

    def total(x):
        out = orc.token_logprobs(x, tokens, c)
        return (gl * out["logprobs"]).sum() + (gh * out["entropy"]).sum()
    num = np.zeros_like(z)
    for idx in np.ndindex(*z.shape):
        up, dn = z.copy(), z.copy()
        up[idx] += eps
        dn[idx] -= eps
        num[idx] = (total(up) - total(dn)) / (2 * eps)
    assert rel_err(orc.token_logprobs_backward(z, tokens, c, gl, gh), num) < 1e-7
    assert np.allclose(orc.token_logprobs_backward(z, tokens, c, gl, gh).sum(axis=1), 0, atol=1e-12)     # a shift of a row changes nothing


def test_agrees_with_the_training_loss():
    rng = np.random.default_rng(7)
    z, labels = rng.standard_normal((5, 16)), np.array([0, 15, -1, 7, 3])
    loss, grad = orc.lrec_loss(z, z, labels, 0.0, 1.0)
    out = orc.token_logprobs(z, labels, 1.0)
    assert np.allclose(loss, -out["logprobs"], atol=1e-12)
    assert np.allclose(grad, orc.token_logprobs_backward(z, labels, 1.0, -np.ones(5), None), atol=1e-12)
