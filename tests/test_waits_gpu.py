"""The bounded waits of the kernels: on a barrier, and for a count in shared memory."""
import pytest
import torch

from paper_2407_18121_b200 import binding as ec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("limit_us", [1500, 20000])
def test_both_kinds_of_wait_run_out(limit_us):
    """One after the other: the kernel takes two limits, reports, and leaves the context usable."""
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    ec.ec_selftest_wait_timeout(ws, 10)                        # loads the kernel
    torch.cuda.synchronize()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    ec.ec_selftest_wait_timeout(ws, limit_us)
    b.record()
    assert ec.ec_device_status(ws) == ec.EC_ERR_TIMEOUT
    torch.cuda.synchronize()
    assert a.elapsed_time(b) * 1000 >= 2 * limit_us * 0.99
    assert (torch.ones(4, device="cuda") + 1).tolist() == [2.0] * 4
