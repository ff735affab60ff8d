"""The log probabilities of a text: row t of the logits goes with token t + 1, so the tokens begin one element into their tensor."""
import pytest
import torch

import paper_2306_08162_b200 as ql
from paper_2306_08162_b200 import build as qbuild

OK = 0x1000                     # aligned and non-NULL; never dereferenced because something else is refused first


def test_tokens_between_elements_are_refused():
    qbuild.build_library()
    lib = ql.library()
    for by in (1, 2, 3):
        assert lib.qlora_token_logprobs(4, 100, 100, 0, OK, OK + by, 1.0, 0, OK, None, None, None, None, 0) == -3
        assert lib.qlora_token_logprobs_bwd(4, 100, 100, 0, OK, OK + by, 1.0, OK, OK, None, 100, 2 * OK, 0) == -3


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V,k", [(2, 1000, 0), (40, 20011, 5), (300, 515, 5), (3100, 331, 0)])
def test_next_tokens_of_a_text(T, V, k, dtype):
    """As with a copy of the tokens; the gradient too, into the logits' place of a tensor of all T rows."""
    gen = torch.Generator(device="cuda").manual_seed(T + V)
    z = torch.randn((T, V), device="cuda", generator=gen).to(dtype)
    text = torch.randint(0, V, (T + 3,), device="cuda", generator=gen).int()
    gl = torch.randn(T - 1, device="cuda", generator=gen)
    for first in (1, 2, 3):
        results = []
        for tokens in (text[first:first + T - 1], text[first:first + T - 1].clone()):
            lp, ent, stats = torch.empty(T - 1, device="cuda"), torch.empty(T - 1, device="cuda"), torch.empty((T - 1, 3), device="cuda")
            ids, top = (torch.empty((T - 1, k), dtype=torch.int32, device="cuda"), torch.empty((T - 1, k), device="cuda")) if k else (None, None)
            ql.qlora_token_logprobs(z[:-1], tokens, 0.8, lp, entropy=ent, top_ids=ids, top_logprobs=top, stats=stats)
            dz = torch.zeros_like(z)
            ql.qlora_token_logprobs_bwd(z[:-1], tokens, 0.8, stats, gl, None, dz[:-1])
            assert (dz[-1] == 0).all()
            results.append([t for t in (lp, ent, stats, ids, top, dz) if t is not None])
        assert all(torch.equal(a, b) for a, b in zip(*results))
        want = torch.log_softmax(z[:-1].double() * 0.8, 1).gather(1, text[first:first + T - 1].long()[:, None])[:, 0]
        # (0.8 is rounded to fp32, off by 2^-25, of the difference to the maximum: below 8 here; the sums as in the other tests of these kernels)
        assert ((results[0][0].double() - want).abs() <= (V / 256 + 64 + 8) * 2.0 ** -24 + 4 * 2.0 ** -24 * want.abs()).all()
