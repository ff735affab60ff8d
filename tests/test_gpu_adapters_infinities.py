"""Infinities and NaN in what the adapters' gradients are formed from: they reach their own columns and ranks, the others keep their bits."""
import pytest
import torch

import paper_2306_08162_b200 as ql
from test_gpu_adapters import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,r,kind", [(8, 16, "each"), (400, 16, "each"), (1300, 8, "rows"), (1300, 16, "one"), (700, 64, "one"), (700, 24, "each")])
def test_finite_columns_and_ranks_keep_their_bits(M, r, kind):
    p = Problem(M, 288, 264, r, 3, kind)
    H, G = p.empty(M, r), p.empty(M, r)
    p.forward(H=H)
    p.back(G=G)
    clean = p.grads(H, G)
    a = int(p.adapter_of[5])
    a = a if a >= 0 else int(p.adapter_of.max())
    t = int(torch.nonzero(p.adapter_of == a)[-1])
    p.X[t, 3], p.X[t, 70], p.dY[t, 9], p.dY[t, 200] = float("inf"), float("nan"), float("-inf"), float("nan")
    dA, dB = p.grads(H, G)
    for got, want, axis, columns in ((dA, clean[0], 2, (3, 70)), (dB, clean[1], 1, (9, 200))):
        odd = torch.zeros(got.shape[axis], dtype=torch.bool, device="cuda")
        odd[list(columns)] = True
        got, want = got.movedim(axis, 2), want.movedim(axis, 2)                      # [adapter, rank, column]
        assert torch.equal(got[..., ~odd], want[..., ~odd])
        others = torch.arange(3, device="cuda") != a
        assert torch.equal(got[others], want[others])
        assert torch.isnan(got[a][:, columns[1]]).all()
    # an infinity keeps its sign: G's for dA, the opposite of H's for dB
    assert torch.equal(dA[a][:, 3], G[t].sign() * float("inf")) and torch.equal(dB[a][9], -H[t].sign() * float("inf"))
    # of one rank of G and H
    G[t, 2], H[t, 5] = float("inf"), float("nan")
    p.X[t, 3], p.X[t, 70], p.dY[t, 9], p.dY[t, 200] = 1.0, -1.0, 2.0, 0.5
    clean = p.grads(torch.nan_to_num(H), torch.nan_to_num(G, posinf=1.0))
    dA, dB = p.grads(H, G)
    rank = torch.arange(r, device="cuda")
    assert torch.equal(dA[:, rank != 2], clean[0][:, rank != 2]) and torch.equal(dB[..., rank != 5], clean[1][..., rank != 5])
    assert not torch.isfinite(dA[a, 2]).any() and torch.isnan(dB[a][:, 5]).all()
    assert ql.qlora_device_status() == 0
