"""GPU: the time limit of every kind of bounded wait.

The check runs three waits one after the other on a barrier that nothing
completes. Each may overrun its limit by one round of attempts: at most 256,
each suspended for a time that is the hardware's choice, taken to be below a
millisecond.
"""
import pytest
import torch

from paper_2607_05722_gb300 import nld
from test_gpu_kv4 import VER, Attn, _lib, check, f32_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("limit_ms", [2, 20])
def test_each_wait_keeps_its_limit(orc, limit_ms):
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    nld.nld_check_wait_timeout(1000)  # loads the kernel
    torch.cuda.synchronize()
    nld.nld_device_error(clear=True)
    start.record()
    nld.nld_check_wait_timeout(limit_ms * 1_000_000)
    end.record()
    torch.cuda.synchronize()
    assert nld.nld_device_error(clear=True) == nld.NLD_DEVERR_WAIT_TIMEOUT
    assert 3 * limit_ms <= start.elapsed_time(end) <= 3 * (limit_ms + 256)
    # the context is in order: an attention call of the kernel whose waits were checked
    c = Attn(60, (16, 2, 128), 16, [300, 40], 8)
    out, lse = c.run(VER)
    check(out, lse, *c.oracle(orc, VER), size=float(abs(f32_of(c.v)).max()))
