"""A second context behind work on streams of PyTorch's: if its worker's stream lies on the hardware queue of the first one's worker, it
waits for that worker's idle exit, and no longer.  (In a file that runs late: it makes streams.)"""
import time

import numpy as np
import pytest
import torch

from gpu_helpers import DevicePools, compare_with_oracle
from paper_2604_17861_amd import runtime as R
from paper_2604_17861_amd import streams as S

pytestmark = pytest.mark.gpu


def test_a_second_context_waits_for_the_firsts_idle_exit_at_most():
    side = torch.cuda.Stream()
    host, device = torch.empty(1 << 22, pin_memory=True), torch.zeros(1 << 22, device="cuda")
    torch.cuda.synchronize()
    with R.Runtime(0, idle_exit_ms=2000, wait_timeout_ms=20000):
        with torch.cuda.stream(side):                        # (copies beside a worker: after these two contexts have shared a queue)
            for _ in range(50):
                host.copy_(device, non_blocking=True)
        side.synchronize()
    streams = [S.config1(n_tasks=300, numel=5000, seed=k) for k in (1, 2)]
    pools = [DevicePools(s) for s in streams]
    for _ in range(2):
        with R.Runtime(64, workgroups_per_cu=1, idle_exit_ms=1000, wait_timeout_ms=20000) as a:
            t0 = time.perf_counter()
            with R.Runtime(64, workgroups_per_cu=1, idle_exit_ms=1000, wait_timeout_ms=20000) as b:
                took = time.perf_counter() - t0
                print("the second context took %.3f s" % took, flush=True)
                assert took < 5.0
                for rt, s, p in ((b, streams[1], pools[1]), (a, streams[0], pools[0])):
                    rt.start_worker()                        # (as a program does that has waited: nothing where it is running)
                    rt.register_table(s.table)
                    first = rt.submit(p.tasks, 0, 50)
                    rt.wait()
                    assert np.all(rt.completions(first, 50)["status"] == 0)
        for s, p in zip(streams, pools):
            assert compare_with_oracle(s, p.download(), first=0, count=50)["max_ulp"] == 0
