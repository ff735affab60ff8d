"""The waits of the head's cross entropy that run out: they set their own bit of the status word, and the call is right afterwards."""
import time

import pytest
import torch

import paper_2306_08162_b200 as ql
from test_gpu_head_loss import check, problem, run

pytestmark = pytest.mark.gpu


def test_waits_that_run_out_are_reported_and_cleared():
    hidden, head, labels, d_loss = problem(300, 9000, 256)
    assert ql.qlora_device_status() == 0
    t0 = time.perf_counter()
    ql.qlora_selftest_bounded_wait(2000)
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 1.0                                            # they ended by themselves
    for clear in (False, True):
        with pytest.raises(ql.QloraError, match="0x3") as e:
            ql.qlora_device_status(clear=clear)
        assert e.value.status == -6
    assert ql.qlora_device_status() == 0
    loss, grad = run(hidden, head, labels, d_loss)
    assert ql.qlora_device_status() == 0
    check(hidden, head, labels, d_loss, loss, grad)
