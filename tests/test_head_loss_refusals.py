"""Refusals of the head's cross entropy: on the host, before anything is launched, so these run without a GPU."""
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


BAD_SIZES = [(dict(T=-1), -1), (dict(V=-1), -1), (dict(D=-8), -1), (dict(V=0), -2), (dict(V=(1 << 24) + 1), -2), (dict(D=56), -2), (dict(D=100), -2),
             (dict(D=(1 << 20) + 8), -2), (dict(T=1 << 30, V=1 << 24), -2), (dict(T=(1 << 24) + 1), -2), (dict(T=2 ** 31 - 1, V=1), -2)]


@pytest.mark.parametrize("change,status", BAD_SIZES)
def test_sizes(ql, change, status):
    size = {**dict(T=4, V=100, D=64), **change}
    out = ctypes.c_size_t()
    assert ql.library().qlora_head_loss_workspace_bytes(size["T"], size["V"], size["D"], 1, out) == status
    assert ql.library().qlora_head_loss(size["T"], size["V"], size["D"], *[OK] * 7, 1 << 40, None) == status


def test_workspace_bytes(ql):
    lib, out = ql.library(), ctypes.c_size_t()
    assert lib.qlora_head_loss_workspace_bytes(4, 100, 64, 1, None) == -1 and lib.qlora_head_loss_workspace_bytes(4, 100, 64, 2, out) == -1
    alone, both = ql.qlora_head_loss_workspace_bytes(2048, 32000, 4096, False), ql.qlora_head_loss_workspace_bytes(2048, 32000, 4096, True)
    assert 0 < alone < both < 2048 * 32000 * 2                                       # less than the logits would take
    assert ql.qlora_head_loss_workspace_bytes(0, 100, 64, True) > 0


def test_arguments(ql):
    call = ql.library().qlora_head_loss

    def status(T=4, V=100, D=64, hidden=OK, head=OK, labels=OK, d_loss=None, loss=OK, d_hidden=None, ws=OK, size=1 << 40):
        return call(T, V, D, hidden, head, labels, d_loss, loss, d_hidden, ws, size, None)
    for missing in ("hidden", "head", "labels", "loss"):
        assert status(**{missing: None}) == -1
    assert status(d_loss=OK) == -1 and status(d_hidden=64 * OK) == -1                # the gradient takes both
    assert status(d_loss=OK, d_hidden=OK + 16) == -1                                 # overlaps the hidden states
    assert status(d_loss=OK + 8, d_hidden=64 * OK) == -1                             # overlaps the losses
    for off in ("hidden", "head", "ws"):
        assert status(**{off: OK + 8}) == -3
    assert status(d_loss=OK, d_hidden=64 * OK + 8) == -3
    assert status(labels=OK + 2) == -3 and status(loss=OK + 1) == -3 and status(d_loss=OK + 2, d_hidden=64 * OK) == -3
    assert status(ws=None) == -4 and status(size=1000) == -4
    assert status(T=0, hidden=None) == 0                                             # nothing to do


@pytest.mark.skipif(torch.cuda.is_available(), reason="what a host without a GPU sees")
def test_binding_without_a_gpu(ql):
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ql.qlora_head_loss(x, x, torch.zeros(4, dtype=torch.int32), torch.zeros(4), None)
    with pytest.raises(ValueError):
        ql.qlora_head_loss(x[0], x, torch.zeros(4, dtype=torch.int32), torch.zeros(4), None)


@pytest.mark.gpu
def test_binding_refuses_other_shapes_types_and_devices(ql):
    t = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
    half = dict(dtype=torch.bfloat16)
    right = dict(hidden=t(4, 64, **half), head=t(100, 64, **half), labels=t(4, dtype=torch.int32), loss=t(4), ws=t(ql.qlora_head_loss_workspace_bytes(4, 100, 64, True), dtype=torch.uint8),
                 d_loss=t(4), d_hidden=t(4, 64, **half))

    def call(**change):
        a = {**right, **change}
        ql.qlora_head_loss(a["hidden"], a["head"], a["labels"], a["loss"], a["ws"], d_loss=a["d_loss"], d_hidden=a["d_hidden"])
    call()
    for name, wrong in dict(hidden=t(4, 64), head=t(100, 128, **half), labels=t(4, dtype=torch.int64), loss=t(3), d_loss=t(5), d_hidden=t(4, 64)).items():
        with pytest.raises(ValueError):
            call(**{name: wrong})
        with pytest.raises(ValueError):
            call(**{name: right[name].cpu()})
    with pytest.raises(ValueError):
        call(ws=right["ws"].cpu())
    with pytest.raises(ValueError):
        call(hidden=t(64, 4, **half).t())
    for change in (dict(ws=right["ws"][:1024]), dict(d_loss=None), dict(d_hidden=None)):
        with pytest.raises(ql.QloraError):
            call(**change)
    buffer = t(5, 64, **half)
    with pytest.raises(ql.QloraError):
        call(hidden=buffer[:4], d_hidden=buffer[1:])
