"""The dispatch filter and kernels that are launched between its blocks."""
import threading

import pytest
import torch

from paper_2604_17861_amd import model as M
from paper_2604_17861_amd import runtime as R
from paper_2604_17861_amd.dispatch import GpuosMode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("launch", ("norm", "cache", "torch"))
def test_a_block_that_begins_behind_a_kernel_in_flight_reads_its_result(launch):
    """Some milliseconds of work on PyTorch's stream between two blocks; the second block's first operation reads the last of what
    it writes."""
    x = torch.randn(16384, 16, 128, device="cuda")
    small = torch.randn(4, 16, 128, device="cuda")
    slots = torch.arange(16384, dtype=torch.int32, device="cuda")
    cache = torch.zeros(256, 64, 16, 128, dtype=torch.int8, device="cuda")
    scales = torch.zeros(256, 64, 16, 1, device="cuda")
    pages = torch.arange(256, dtype=torch.int32, device="cuda")[None]
    M.cache_store(x, slots, cache, scales)

    def work(out):
        for _ in range(30):
            if launch == "norm":
                M.norm_rope(x, out=out)
            elif launch == "cache":
                M.cache_load(cache, scales, pages, None, 16384, out=out[None])
            else:
                torch.mul(x, 2.0, out=out)
        return out[-4:]

    want = torch.relu(work(torch.zeros_like(x))).cpu()
    assert (want > 0).any()
    outs = [torch.zeros_like(x) for _ in range(3)]
    torch.cuda.synchronize()
    mode = GpuosMode(idle_exit_ms=50)
    try:
        for out in outs:
            with mode:
                torch.relu(small)                        # the filter knows of nothing in flight behind this
            last = work(out)
            with mode:
                y = torch.relu(last)
            assert torch.equal(y.cpu(), want)
        assert mode.stats["redirected"] == 6, mode.stats
    finally:
        mode.close()


def test_a_call_from_another_thread_passes_a_filter_by_and_ends():
    x = torch.randn(40, 4, 64, device="cuda")
    want = M.norm_rope(x)
    torch.cuda.synchronize()
    mode, got = GpuosMode(idle_exit_ms=50), []
    try:
        with mode:
            other = threading.Thread(target=lambda: got.append(M.norm_rope(x)))
            other.start()
            other.join(60)
            assert not other.is_alive() and len(got) == 1 and mode in R.active_filters
        torch.cuda.synchronize()
        assert torch.equal(got[0], want)
    finally:
        mode.close()
