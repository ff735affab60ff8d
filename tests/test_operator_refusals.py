"""Refusals of the log-probability and optimizer calls: on the host, before anything is launched, so these run without a GPU."""
import ctypes

import pytest
import torch

from paper_2306_08162_b200 import build as qbuild

OK = 0x1000                     # aligned and non-NULL; never dereferenced because something else is refused first


@pytest.fixture(scope="module")
def ql():
    qbuild.build_library()
    import paper_2306_08162_b200 as mod
    mod.library()
    return mod


def test_token_logprobs_arguments(ql):
    call = ql.library().qlora_token_logprobs

    def status(T=4, V=100, ld=100, dtype=0, logits=OK, tokens=OK, c=1.0, k=0, lp=OK, ent=None, ids=None, top=None, stats=None):
        return call(T, V, ld, dtype, logits, tokens, c, k, lp, ent, ids, top, stats, 0)
    assert status(T=-1) == -1 and status(V=-1) == -1 and status(ld=99) == -1
    assert status(V=0) == -2 and status(V=(1 << 24) + 1, ld=1 << 25) == -2
    assert status(dtype=3) == -2 and status(dtype=-1) == -2
    for c in (0.0, -1.0, float("nan"), float("inf")):
        assert status(c=c) == -1
    assert status(k=-1) == -1 and status(k=65, ids=OK) == -2 and status(V=8, ld=8, k=9, ids=OK) == -2
    assert status(k=4) == -1 and status(ids=OK) == -1                       # alternatives without a place for them, and the reverse
    assert status(logits=None) == -1 and status(tokens=None) == -1 and status(lp=None) == -1
    assert status(logits=OK + 1) == -3 and status(dtype=2, logits=OK + 2) == -3 and status(lp=OK + 4) == -3 and status(stats=OK + 8) == -3
    assert status(T=0, logits=None) == 0                                    # nothing to do


def test_token_logprobs_bwd_arguments(ql):
    call = ql.library().qlora_token_logprobs_bwd

    def status(T=4, V=100, ld=100, dtype=0, logits=OK, tokens=OK, c=1.0, stats=OK, gl=OK, gh=None, gld=100, out=2 * OK):
        return call(T, V, ld, dtype, logits, tokens, c, stats, gl, gh, gld, out, 0)
    assert status(T=-1) == -1 and status(ld=99) == -1 and status(gld=99) == -1 and status(c=0.0) == -1
    assert status(V=0) == -2 and status(dtype=3) == -2
    assert status(logits=None) == -1 and status(stats=None) == -1 and status(out=None) == -1 and status(tokens=None) == -1
    assert status(gl=None) == -1                                            # no gradient at all
    # over the logits in part: at another stride, a row further, a few columns further, over the last row's end
    big = 1 << 20
    assert status(ld=128, out=OK) == -1 and status(logits=big, out=big + 200) == -1 and status(logits=big, out=big + 16) == -1
    assert status(logits=big, ld=256, gld=256, out=big + 2 * (256 + 99)) == -1 and status(logits=big, ld=256, gld=256, out=big - 2 * 99) == -1
    assert status(logits=big, ld=128, gld=300, out=big - 2 * (3 * 300 + 99)) == -1 and status(T=1, logits=big, out=big + 198) == -1
    assert status(logits=big, ld=1 << 60, gld=1 << 61, out=big + 1000) == -1 and status(logits=big, ld=1 << 62, gld=1 << 62, out=big + 198) == -1
    # beside them in one buffer, or right behind: nothing wrong with that (what is refused, later on, is an address)
    assert status(logits=big, ld=256, gld=256, out=big + 2 * 128, gl=OK + 4) == -3 and status(logits=big, out=big + 2 * 400, gl=OK + 4) == -3
    assert status(out=2 * OK + 1) == -3 and status(dtype=2, logits=OK + 2) == -3 and status(gl=OK + 4) == -3
    assert status(T=0, logits=None) == 0


def adam(ql, n=8, **kw):
    array = (ql.binding._AdamwTensor * 1)()
    for t in array:
        t.param, t.grad, t.m, t.v, t.n = OK, OK, OK, OK, n
    fields = dict(n_tensors=1, tensors=array, param_type=0, grad_type=2, state_type=2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)
    fields.update(kw)
    d = ql.binding._AdamwDesc(**fields)
    d.keep = array
    return d, array


def test_adamw_arguments(ql):
    lib = ql.library()

    def status(d, lr=1e-3, step=1, lr_dev=None, step_dev=None, norm=None):
        return lib.qlora_adamw(ctypes.byref(d), lr, step, lr_dev, step_dev, norm, 0)

    def changed(**kw):
        d, array = adam(ql)
        for key, value in kw.items():
            setattr(array[0], key, value)
        return status(d)
    d, _ = adam(ql)
    assert lib.qlora_adamw(None, 1e-3, 1, None, None, None, 0) == -1
    assert status(d, step=0) == -1 and status(d, lr=float("nan")) == -1 and status(d, lr=float("inf")) == -1
    assert status(d, lr_dev=OK + 4) == -3 and status(d, step=0, step_dev=OK + 4) == -3 and status(d, norm=OK + 8) == -3
    for kw in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=1e-60), dict(weight_decay=-1.0),
               dict(n_tensors=-1), dict(tensors=None)):
        assert status(adam(ql, **kw)[0]) == -1, kw
    for kw in (dict(param_type=3), dict(grad_type=3), dict(state_type=0)):
        assert status(adam(ql, **kw)[0]) == -2, kw
    assert changed(n=-1) == -1 and changed(param=None) == -1 and changed(grad=None) == -1 and changed(m=None) == -1 and changed(v=None) == -1
    assert changed(n=(1 << 40) + 1) == -2
    assert changed(m_scale=OK) == -1                                        # scales with 32-bit states
    assert changed(param=OK + 2) == -3 and changed(grad=OK + 4) == -3 and changed(master=OK + 4) == -3
    d, array = adam(ql, state_type=3)
    assert status(d) == -1                                                  # 8-bit states without scales
    array[0].m_scale, array[0].v_scale = OK + 4, OK + 2                     # (scales may begin at any float)
    assert status(d) == -3
    d, array = adam(ql, param_type=2)
    array[0].master = OK
    assert status(d) == -1                                                  # master weights of fp32 parameters
    d, array = adam(ql, n=0)
    assert status(d) == 0 and status(adam(ql, n_tensors=0)[0]) == 0         # nothing to do, nothing launched


def test_grad_norm_arguments(ql):
    lib = ql.library()
    need = ql.GRAD_NORM_WORKSPACE_BYTES

    def status(d, prescale=1.0, max_norm=1.0, out=OK, ws=OK, size=need):
        return lib.qlora_grad_norm(ctypes.byref(d), prescale, max_norm, out, ws, size, 0)
    d, array = adam(ql)
    nan = float("nan")
    assert status(d, prescale=nan) == -1 and status(d, max_norm=nan) == -1 and status(d, out=None) == -1
    assert status(d, out=OK + 4) == -3 and status(d, ws=OK + 8) == -3
    assert status(d, ws=None) == -4 and status(d, size=need - 1) == -4
    array[0].grad = None
    assert status(d) == -1


def test_descriptor_of_the_optimizer_step(ql):
    """adamw_desc checks its lists once: sizes, types, overlaps -- and that the tensors are on a GPU, which these are not."""
    f = lambda n, t=torch.float32: torch.zeros(n, dtype=t)  # noqa: E731
    bf, e4 = torch.bfloat16, torch.float8_e4m3fn

    def refused(match, *lists, **kw):
        with pytest.raises(ValueError, match=match):
            ql.adamw_desc(*lists, **kw)
    refused("on one CUDA device", [f(300, bf)], [f(300)], [f(300)], [f(300)])
    refused("2 tensors in m", [f(300, bf)], [f(300)], [f(300), f(300)], [f(300)])
    refused("299 elements", [f(300, bf)], [f(299)], [f(300)], [f(300)])
    refused("not supported", [f(300, torch.float64)], [f(300)], [f(300)], [f(300)])
    refused("not supported", [f(300, bf), f(8)], [f(300), f(8)], [f(300), f(8)], [f(300), f(8)])          # one call, one type
    refused("m_scale and v_scale", [f(300, bf)], [f(300)], [f(300, e4)], [f(300, e4)])
    refused("m_scale and v_scale", [f(300, bf)], [f(300)], [f(300)], [f(300)], m_scale=[f(2)], v_scale=[f(2)])
    refused("1 elements", [f(300, bf)], [f(300)], [f(300, e4)], [f(300, e4)], m_scale=[f(2)], v_scale=[f(1)])
    refused("on one CUDA device", [f(300, bf)], [f(300)], [f(300, e4)], [f(300, e4)], m_scale=[f(2)], v_scale=[f(2)])
    refused("no master", [f(300)], [f(300)], [f(300)], [f(300)], master=[f(300)])
    refused("contiguous", [f(300, bf)], [f(600)[::2]], [f(300)], [f(300)])
    p = f(300, bf)
    refused("overlap", [p, p], [f(300), f(300)], [f(300), f(300)], [f(300), f(300)])
    m = f(400)
    refused("overlap", [f(300, bf)], [f(300)], [m[:300]], [m[100:]])
    refused("gradient overlaps", [f(300, bf)], [m[100:]], [m[:300]], [f(300)])
    g = f(300)
    refused("on one CUDA device", [f(300, bf), f(300, bf)], [g, g], [f(300), f(300)], [f(300), f(300)])   # a shared gradient is only read


def test_tensors_of_the_host_are_refused(ql):
    z, t, out = torch.zeros(3, 16), torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    with pytest.raises(ValueError, match="current CUDA device"):
        ql.qlora_token_logprobs(z, t, 1.0, out)
    with pytest.raises(ValueError, match="current CUDA device"):
        ql.qlora_token_logprobs_bwd(z, t, 1.0, torch.zeros(3, 3), out, None, torch.zeros(3, 16))
    with pytest.raises(ValueError, match="dense rows"):
        ql.qlora_token_logprobs(torch.zeros(16, 3).t(), t, 1.0, out)
    with pytest.raises(ValueError, match="torch.int32"):
        ql.qlora_token_logprobs(z, t.long(), 1.0, out)
    with pytest.raises(ValueError, match=r"\[3\] is needed"):
        ql.qlora_token_logprobs(z, t, 1.0, torch.zeros(4))
    with pytest.raises(ValueError, match="not supported"):
        ql.qlora_token_logprobs(z.double(), t, 1.0, out)
    with pytest.raises(ValueError, match="shape and the type"):
        ql.qlora_token_logprobs_bwd(z, t, 1.0, torch.zeros(3, 3), out, None, torch.zeros(3, 15))
    with pytest.raises(TypeError, match="adamw_desc"):
        ql.qlora_adamw(None, 1e-3, 1, stream=0)
