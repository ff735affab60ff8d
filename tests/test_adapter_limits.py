"""The longest features of the calls on adapters: refused on the host beyond them, before anything is launched (an adapter's matrix is counted in 32 bits,
steps of 2^14 included)."""
import ctypes

import pytest

from test_adapter_refusals import OK, made, ql  # noqa: F401


@pytest.mark.parametrize("change,status", [(dict(K=1 << 24, N=1 << 24, r=64), 0), (dict(K=(1 << 24) + 32), -2), (dict(N=(1 << 24) + 8), -2), (dict(N=(1 << 25) - 8, r=64), -2), (dict(K=2 ** 31 - 32), -2),
                                           (dict(N=2 ** 31 - 8), -2)])
def test_features(ql, change, status):  # noqa: F811
    lib, d, size = ql.library(), made(ql, **change), ctypes.c_size_t()
    assert lib.qlora_adapters_workspace_bytes(d, 4, size) == status
    if status != 0:
        assert lib.qlora_adapters_fwd(d, 4, *[OK] * 9, 1 << 60, None) == status
        assert lib.qlora_adapters_bwd_input(d, 4, *[OK] * 9, 1 << 60, None) == status
        assert lib.qlora_adapters_bwd_lora(d, 4, *[OK] * 10, 0, OK, 1 << 60, None) == status
