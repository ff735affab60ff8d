"""Refusals of the calls on adapters of many requests: on the host, before anything is launched, so these run without a GPU."""
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


BAD = [(dict(K=33), -2), (dict(K=0), -2), (dict(N=0), -2), (dict(N=12), -2), (dict(r=0), -2), (dict(r=12), -2), (dict(r=72), -2), (dict(n_adapters=65536), -2),
       (dict(K=-32), -1), (dict(N=-8), -1), (dict(r=-8), -1), (dict(n_adapters=-1), -1)]


def made(ql, **kw):
    return ql.adapters_desc(**{**dict(K=64, N=40, r=8, n_adapters=3), **kw})


@pytest.mark.parametrize("change,status", BAD)
def test_descriptor(ql, change, status):
    lib, d = ql.library(), made(ql, **change)
    size = ctypes.c_size_t()
    assert lib.qlora_adapters_workspace_bytes(d, 4, size) == status
    assert lib.qlora_adapters_fwd(d, 4, *[OK] * 9, 1 << 30, None) == status
    assert lib.qlora_adapters_bwd_input(d, 4, *[OK] * 9, 1 << 30, None) == status
    assert lib.qlora_adapters_bwd_lora(d, 4, *[OK] * 10, 0, OK, 1 << 30, None) == status


def test_workspace_bytes(ql):
    d, size = made(ql), ctypes.c_size_t()
    assert ql.library().qlora_adapters_workspace_bytes(d, -1, size) == -1 and ql.library().qlora_adapters_workspace_bytes(None, 4, size) == -1
    assert ql.library().qlora_adapters_workspace_bytes(d, 4, None) == -1
    assert ql.qlora_adapters_workspace_bytes(d, 1000) >= 2 * 1000 * 8 * 4 and ql.qlora_adapters_workspace_bytes(d, 0) > 0


@pytest.mark.parametrize("name", ["qlora_adapters_fwd", "qlora_adapters_bwd_input"])
def test_products_arguments(ql, name):
    d, call = made(ql), getattr(ql.library(), name)

    def status(M=4, X=OK, ids=OK, A=OK, B=OK, s=OK, base=OK, out=16 * OK, low=None, ws=OK, size=1 << 20, desc=d):
        return call(desc, M, X, ids, A, B, s, base, out, low, ws, size, None)
    assert status(desc=None) == -1 and status(M=-1) == -1
    for missing in ("X", "ids", "A", "B", "s", "base", "out"):
        assert status(**{missing: None}) == -1
    for off in ("X", "A", "B", "base", "low", "ws"):
        assert status(**{off: OK + 8}) == -3
    assert status(out=16 * OK + 8) == -3 and status(ids=OK + 2) == -3 and status(s=OK + 1) == -3
    assert status(out=OK + 16) == -1 and status(base=OK + 16, out=OK) == -1        # they overlap
    assert status(X=32 * OK, base=32 * OK + 64, out=32 * OK + 64) == -1             # the input is overwritten
    assert status(ws=None) == -4 and status(size=100) == -4
    assert status(M=0, X=None) == 0                                                # nothing to do


def test_gradients_arguments(ql):
    d, call = made(ql), ql.library().qlora_adapters_bwd_lora

    def status(M=4, X=OK, dY=OK, ids=OK, A=OK, B=OK, s=OK, H=OK, G=OK, dA=OK, dB=OK, add=0, ws=OK, size=1 << 20, desc=d):
        return call(desc, M, X, dY, ids, A, B, s, H, G, dA, dB, add, ws, size, None)
    assert status(desc=None) == -1 and status(M=-1) == -1 and status(add=2) == -1 and status(add=-1) == -1
    for missing in ("X", "dY", "ids", "s", "dA", "dB"):
        assert status(**{missing: None}) == -1
    assert status(H=None, A=None) == -1 and status(G=None, B=None) == -1
    for off in ("X", "dY", "A", "B", "H", "G", "dA", "dB", "ws"):
        assert status(**{off: OK + 8}) == -3
    assert status(ws=None) == -4 and status(size=100) == -4
    assert status(desc=made(ql, n_adapters=0), dA=None) == 0


def test_binding_refuses_what_is_not_a_descriptor_or_not_on_the_gpu(ql):
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        ql.qlora_adapters_fwd(ql.desc(4, 32, 64, 40, 8, 16.0), 4, x, None, None, None, None, None, None, None, None)
    if not torch.cuda.is_available():
        with pytest.raises(ValueError):
            ql.qlora_adapters_fwd(made(ql), 4, x, None, None, None, None, None, None, None, None)


@pytest.mark.gpu
def test_binding_refuses_other_shapes_types_and_devices(ql):
    d = made(ql)
    t = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
    half, ints = dict(dtype=torch.bfloat16), dict(dtype=torch.int32)
    right = dict(X=t(4, 64, **half), ids=t(4, **ints), A=t(3, 8, 64, **half), B=t(3, 40, 8, **half), s=t(3), base=t(4, 40, **half), Y=t(4, 40, **half), H=t(4, 8),
                 ws=t(ql.qlora_adapters_workspace_bytes(d, 4), dtype=torch.uint8))

    def call(**change):
        a = {**right, **change}
        ql.qlora_adapters_fwd(d, 4, a["X"], a["ids"], a["A"], a["B"], a["s"], a["base"], a["Y"], a["H"], a["ws"])
    call()
    for name, wrong in dict(X=t(4, 32, **half), ids=t(5, **ints), A=t(3, 8, 64), B=t(3, 8, 40, **half), s=t(2), base=t(4, 40), Y=t(3, 40, **half), H=t(4, 16)).items():
        with pytest.raises(ValueError):
            call(**{name: wrong})
        with pytest.raises(ValueError):
            call(**{name: right[name].cpu()})
    with pytest.raises(ValueError):
        call(ws=right["ws"].cpu())
    with pytest.raises(ValueError):
        call(X=t(64, 4, **half).t())
    with pytest.raises(ql.QloraError):
        call(ws=right["ws"][:64])
    buffer = t(5, 40, **half)
    with pytest.raises(ql.QloraError):
        call(base=buffer[:4], Y=buffer[1:])
