"""Cache operators as kernels beside a resident worker at its default size: each starts at once, not when the worker has left; and on
tensors that a dispatch filter's tasks are working on."""
import time

import pytest
import torch

from paper_2604_17861_amd import model as M
from paper_2604_17861_amd import runtime as R
from paper_2604_17861_amd.dispatch import GpuosMode
from test_zzy_gpu_cache import E2M1, E4M3, I8, attend_inputs, caches_of
from test_gpu_model import BF16, F16, F32, _let_go, laid, normal, up  # noqa: F401

pytestmark = pytest.mark.gpu


def calls_of_every_kernel():
    made = []
    for dtype in (F32, F16, BF16):
        gen = torch.Generator().manual_seed(2)
        for layout in ("plain", "strided"):
            q, k, v = (laid(normal(gen, 40, 4, 64, dtype=dtype), layout) for _ in range(3))
            slots, table, mine = up(torch.arange(40, dtype=torch.int32)), up(torch.rand(40, 64, generator=gen)), [up(c) for c in caches_of(3, 16, 4, 64, 1, I8)]
            made.append(("append %s %s" % (dtype, layout), lambda q=q, k=k, v=v, slots=slots, mine=mine, table=table: (M.cache_append_qkv(q, k, v, slots, *mine, table), *mine)))
        for fmt in (E2M1, I8, E4M3):
            for d in (64, 72, 128, 200, 256):
                for groups in (1, d // 32) if d % 32 == 0 else (1,):
                    for longest in (100, 1100):
                        q, caches, pages, lengths = attend_inputs((1, 1, 4, 4, d, groups, 16, longest, None, 0, "plain"), dtype, fmt)
                        a = (up(q), *[up(c) for c in caches], up(pages), None, longest)
                        made.append(("attention %s %s %d %d %d" % (dtype, fmt, d, groups, longest), lambda a=a: (M.cache_attention(*a),)))
        q, caches, pages, _ = attend_inputs((1, 1, 1, 1, 64, 1, 64, 40000, None, 0, "plain"), dtype, I8)
        a = (up(q), *[up(c) for c in caches], up(pages), None, 40000)
        made.append(("a wide join %s" % dtype, lambda a=a: (M.cache_attention(*a),)))
    return made


def test_every_kernel_starts_beside_the_default_worker():
    made = calls_of_every_kernel()
    want = [[o.clone() for o in call()] for what, call in made]
    done = torch.cuda.Event()
    torch.cuda.synchronize()
    got = []
    with R.Runtime(0, idle_exit_ms=8000, wait_timeout_ms=20000) as rt:
        assert rt.peek_queue().workgroups == 3 * int(R.device_info(0)["compute_units"])
        t0 = time.perf_counter()
        for what, call in made:
            got.append(call())
            done.record()
            while not done.query():
                assert time.perf_counter() - t0 < 5.0, "%s has not started" % what
                time.sleep(0.0002)
        assert rt.worker_alive() and time.perf_counter() - t0 < 5.0
    torch.cuda.synchronize()
    for (what, call), now, was in zip(made, got, want):
        for o, w in zip(now, was):
            assert bool(((o == w) | (torch.isnan(o.float()) & torch.isnan(w.float()))).all()), what


def test_a_dispatch_filters_tasks_are_waited_for():
    q, caches, pages, lengths = attend_inputs((2, 1, 4, 4, 64, 1, 16, 60, (60, 33), 0, "plain"), F32, I8)
    x, mine, table, n = up(q), [up(c) for c in caches], up(pages), up(lengths)
    want = M.cache_attention(x * 0.5 + 0.25, *mine, table, n, 60) * 2.0
    mode = GpuosMode(wait_timeout_ms=20000, idle_exit_ms=5000)
    try:
        for _ in range(5):
            with mode:
                y = x * 0.5 + 0.25
                got = M.cache_attention(y, *mine, table, n, 60) * 2.0
            assert torch.equal(got, want)
    finally:
        mode.close()
