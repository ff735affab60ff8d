"""The operators as a fine-tuning program runs them: layer forward to logits, log probabilities and entropies, their gradient in place of the
logits, the layer's backward, the LoRA gradients, the clipping factor and the AdamW step -- and the next forward on the updated pair.  Every
stage against the 64-bit oracle on the stage's own device inputs (tolerances: those of the layer's parity tests; the optimizer's own
test has the tight ones)."""
import numpy as np
import pytest
import torch

import paper_2306_08162_b200 as ql
import qlora_inputs as qi
from oracle import qlora_oracle as orc
from gpu_util import GpuLayer, to_f64
from helpers import REL_TOL, rel_err

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [5, 200])
@pytest.mark.parametrize("bits", [32, 8])
def test_step(M, bits):
    K, V, r = 256, 1000, 8
    layer = qi.make_layer(K=K, N=V, bits=4, group_size=64, r=r, alpha=16.0, M=M, seed=61)
    gl = GpuLayer(layer)
    W = orc.dequant(orc.pack(layer["codes"], 4), layer["scales"], layer["zeros"], 4, 64)
    X64 = to_f64(gl.X)
    tokens = torch.from_numpy(np.random.default_rng(3).integers(-1, V, size=M).astype(np.int32)).cuda()
    f32 = lambda *s: torch.zeros(s, dtype=torch.float32, device="cuda")  # noqa: E731
    dA, dB, H, G = f32(r, K), f32(V, r), f32(M, r), f32(M, r)
    Y, dX = torch.empty((M, V), dtype=torch.bfloat16, device="cuda"), torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
    lp, ent, stats = f32(M), f32(M), f32(M, 3)
    masters = [gl.A.float(), gl.B.float()]
    if bits == 32:
        states = dict(m=[f32(r, K), f32(V, r)], v=[f32(r, K), f32(V, r)])
    else:
        e4 = lambda *s: torch.zeros(s, device="cuda").to(torch.float8_e4m3fn)  # noqa: E731
        blocks = [-(-r * K // 256), -(-r * V // 256)]
        states = dict(m=[e4(r, K), e4(V, r)], v=[e4(r, K), e4(V, r)], m_scale=[f32(b) for b in blocks], v_scale=[f32(b) for b in blocks])
    opt = ql.adamw_desc([gl.A, gl.B], [dA, dB], master=masters, **states)
    norm, ws = f32(2), torch.empty(ql.GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    d_lp, d_ent = torch.full((M,), -1.0 / M, device="cuda"), torch.full((M,), -0.1 / M, device="cuda")
    for step in range(1, 4):
        A64, B64 = to_f64(gl.A), to_f64(gl.B)
        ql.qlora_fwd(gl.desc, M, gl.X, gl.Q, gl.scales, gl.zeros, gl.A, gl.B, Y, H, gl.ws)
        assert rel_err(to_f64(Y), orc.forward(X64, W, A64, B64, 16.0)[0]) <= REL_TOL
        Y64 = to_f64(Y)
        ql.qlora_token_logprobs(Y, tokens, 1.0, lp, entropy=ent, stats=stats)
        want = orc.token_logprobs(Y64, tokens.cpu().numpy(), 1.0)
        assert np.abs(to_f64(lp) - want["logprobs"]).max() < 1e-4 and np.abs(to_f64(ent) - want["entropy"]).max() < 1e-4
        ql.qlora_token_logprobs_bwd(Y, tokens, 1.0, stats, d_lp, d_ent, Y)                  # in place: the logits become their gradient
        want = orc.token_logprobs_backward(Y64, tokens.cpu().numpy(), 1.0, to_f64(d_lp), to_f64(d_ent))
        assert rel_err(to_f64(Y), want) <= REL_TOL
        dY64 = to_f64(Y)
        ql.qlora_bwd_input(gl.desc, M, Y, gl.Q, gl.scales, gl.zeros, gl.A, gl.B, dX, G, gl.ws)
        ql.qlora_bwd_lora(gl.desc, M, gl.X, Y, gl.A, gl.B, H, G, dA, dB, 0, gl.ws)
        _, wA, wB, _ = orc.backward(X64, dY64, W, A64, B64, 16.0)
        assert rel_err(to_f64(dA), wA) <= REL_TOL and rel_err(to_f64(dB), wB) <= REL_TOL
        ql.qlora_grad_norm(opt, 1.0, 0.01, norm, ws)
        factor = orc.grad_norm([to_f64(dA), to_f64(dB)], 1.0, 0.01)[1]
        assert abs(norm[1].item() - factor) <= 1e-6 * factor
        held = []
        for j, n in enumerate((r * K, r * V)):
            m, v = to_f64(states["m"][j].float()).ravel(), to_f64(states["v"][j].float()).ravel()
            if bits == 8:
                m, v = m * np.repeat(to_f64(states["m_scale"][j]), 256)[:n], (v * np.repeat(to_f64(states["v_scale"][j]), 256)[:n]) ** 2
            held.append(orc.adamw_step(to_f64(masters[j]).ravel(), to_f64((dA, dB)[j]).ravel(), m, v, step, 1e-3, 0.9, 0.999, 1e-8, 0.0, factor)[0])
        ql.qlora_adamw(opt, 1e-3, step, norm)
        torch.cuda.synchronize()
        for j, (w, p) in enumerate(zip(masters, (gl.A, gl.B))):
            assert np.abs(to_f64(w).ravel() - held[j]).max() <= 1e-3 * 1e-4 and torch.equal(p, w.bfloat16())
    assert ql.qlora_device_status() == 0
