"""Pins for the oracle's adapters of many requests: CPU only."""
import numpy as np

from oracle import qlora_oracle as orc
from helpers import rel_err


def problem(seed=3, M=7, K=6, N=5, r=2, L=3):
    rng = np.random.default_rng(seed)
    n = rng.standard_normal
    return dict(X=n((M, K)), dY=n((M, N)), adapter_of=np.array([2, -1, 0, 0, L, 2, 1])[:M], A=n((L, r, K)), B=n((L, N, r)), scales=n(L) + 2.0), n((M, N)), n((M, K))


def test_one_adapter_is_the_layer_with_a_zero_weight():
    p, base, _ = problem()
    p["adapter_of"] = np.zeros(7, int)
    Y, H = orc.adapters_forward(p["X"], p["adapter_of"], p["A"], p["B"], p["scales"], 0 * base)
    want, want_H = orc.forward(p["X"], np.zeros((5, 6)), p["A"][0], p["B"][0], 2 * p["scales"][0])
    assert rel_err(Y, want) < 1e-12 and rel_err(H, want_H) < 1e-12


def test_tokens_without_an_adapter_and_loops():
    p, base, _ = problem()
    Y, H = orc.adapters_forward(p["X"], p["adapter_of"], p["A"], p["B"], p["scales"], base)
    assert (Y[1] == base[1]).all() and (Y[4] == base[4]).all() and (H[[1, 4]] == 0).all()
    for t in (0, 2, 6):
        a = p["adapter_of"][t]
        for n in range(5):
            want = base[t, n] + sum(p["scales"][a] * p["B"][a, n, j] * sum(p["A"][a, j, k] * p["X"][t, k] for k in range(6)) for j in range(2))
            assert abs(Y[t, n] - want) < 1e-12


def test_gradients_are_those_of_differences():
    p, base, dx_base = problem()
    dX, _, dA, dB = orc.adapters_backward(p["X"], p["dY"], p["adapter_of"], p["A"], p["B"], p["scales"], 0 * dx_base)
    loss = lambda: float((orc.adapters_forward(p["X"], p["adapter_of"], p["A"], p["B"], p["scales"], base)[0] * p["dY"]).sum())  # noqa: E731
    for name, grad in (("X", dX), ("A", dA), ("B", dB)):
        x = p[name]
        for at in [tuple(np.random.default_rng(i).integers(0, x.shape)) for i in range(12)]:
            keep, h = x[at], 1e-5
            x[at] = keep + h
            up = loss()
            x[at] = keep - h
            down = loss()
            x[at] = keep
            assert abs((up - down) / (2 * h) - grad[at]) < 1e-7
