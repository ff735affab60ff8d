"""Log probabilities of rows masked by -inf: an infinity has to be that infinity, and a number a number, at every place.  Tolerances of finite
numbers: S = (V / 256 + 64) u for log s, S + 4u |log p| for log probabilities, 25 S for entropies (the mean of c |z - max| is below 24), u = 2^-24."""
import numpy as np
import pytest
import torch

import paper_2306_08162_b200 as ql
from oracle import qlora_oracle as orc
from gpu_util import agree, to_f64

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("got,want", [([-3.0, 0.0], [-INF, 0.0]), ([INF, 0.0], [-INF, 0.0]), ([NAN, 0.0], [-INF, 0.0]), ([-INF, 0.0], [-3.0, 0.0]), ([0.0, 0.0], [NAN, 0.0]),
                                      ([0.0, NAN], [0.0, 0.0]), ([0.0, 1.1], [0.0, 1.0])])
def test_the_comparison_tells_infinities_from_numbers(got, want):
    agree(want, want, 0.0, 0.0)
    agree(torch.tensor(want), np.array(want), 0.01, 0.01)
    with pytest.raises(AssertionError):
        agree(got, want, 0.01, 0.01)


@pytest.mark.gpu
@pytest.mark.parametrize("c", [0.05, 1.0, 30.0, 1e7])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,V,k", [(3000, 331, 20), (40, 1000, 20), (170, 7000, 64), (20, 20011, 0), (20, 20011, 20), (300, 40000, 20), (460, 12001, 5), (460, 20011, 0), (460, 40000, 20)])
def test_masked_rows(T, V, k, dtype, c):
    """All but none, 1, 5 or half of a row masked; the tokens in turn masked and not; alternatives behind the last unmasked one."""
    c = float(np.float32(c))
    gen = torch.Generator(device="cuda").manual_seed(T + V)
    z = (torch.randn((T, V), device="cuda", generator=gen) * min(3.0, 3.0 / c)).to(DTYPES[dtype])
    tokens = torch.randint(0, V, (T,), device="cuda", generator=gen).int()
    rows = torch.arange(0, 12, device="cuda") * (T // 12)
    for i, t in enumerate(rows.tolist()):
        kept = (0, 1, 5, V // 2)[i % 4]
        first = (i * 97) % (V - kept + 1)
        masked = torch.ones(V, dtype=torch.bool, device="cuda")
        masked[first:first + kept] = False
        z[t, masked] = -INF
        tokens[t] = first if i % 3 == 0 and kept else (first + kept) % V
    out = dict(logprobs=torch.full((T,), 3.0, device="cuda"), entropy=torch.full((T,), 3.0, device="cuda"), stats=torch.full((T, 3), 3.0, device="cuda"))
    if k:
        out["top_ids"], out["top_logprobs"] = torch.full((T, k), -7, dtype=torch.int32, device="cuda"), torch.full((T, k), 3.0, device="cuda")
    ql.qlora_token_logprobs(z, tokens, c, out["logprobs"], entropy=out["entropy"], top_ids=out.get("top_ids"), top_logprobs=out.get("top_logprobs"), stats=out["stats"])
    want = orc.token_logprobs(to_f64(z[rows]), tokens[rows].cpu().numpy(), c, k)
    S = (V / 256 + 64) * U
    agree(out["logprobs"][rows], want["logprobs"], S, 4 * U)
    agree(out["entropy"][rows], want["entropy"], 25 * S, 4 * U)
    agree(out["stats"][rows][:, 0], want["stats"][:, 0], 0.0, 0.0)
    agree(out["stats"][rows][:, 1], want["stats"][:, 1], S, 4 * U)
    assert np.isneginf(want["logprobs"]).any() and np.isneginf(want["stats"][:, 1]).any()
    if k:
        assert np.array_equal(out["top_ids"][rows].cpu().numpy(), want["top_ids"])
        agree(out["top_logprobs"][rows], want["top_logprobs"], S, 4 * U)
        assert np.isneginf(want["top_logprobs"]).any()
