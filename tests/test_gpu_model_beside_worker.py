"""Model operators as kernels beside a resident worker at its default size: each starts at once, not when the worker has left."""
import time

import pytest
import torch

from paper_2604_17861_amd import model as M
from paper_2604_17861_amd import runtime as R
from test_gpu_model import BF16, F16, F32, _let_go, cache_of, normal, rope_inputs, up  # noqa: F401

pytestmark = pytest.mark.gpu


def tasks_of_every_variant():
    """(what, descriptors, outputs)."""
    made = []
    every = lambda t: torch.stack((t, t), -1).flatten(-2)[..., ::2]
    for dtype in (F32, F16, BF16):
        gen, x, g, table, p = rope_inputs((300, 4, 64), 64, dtype, dtype, "each", 21)
        x, g, table, p, dz = up(x), up(g), up(table), up(p), up(normal(gen, 300, 4, 64, dtype=dtype))
        for name, pairs, dout, rows in (("halves", False, dz, x), ("pairs", True, dz, x), ("elements", False, dz[:1, :1, :1].expand_as(dz), every(x))):
            out, dx, partial, dg = up(torch.zeros_like(dz)), up(torch.zeros_like(dz)), up(torch.zeros(64, 37)), up(torch.zeros(64))
            made.append(("rotation, %s" % name, (M.norm_rope_task(up(rows), g, table, p, out, pairs=pairs),), (out,)))
            made.append(("gradient, %s" % name, (M.norm_rope_grad_task(up(dout), x, g, table, p, dx, partial, pairs=pairs), M.gamma_sum_task(partial, dg)), (dx, partial, dg)))
        for name, rows in (("vectors", x), ("elements", every(x))):
            _, _, cache, scales = cache_of(20, 16, 4, 64, 1, torch.int8, "plain")
            made.append(("store, %s" % name, (M.cache_store_task(up(rows), up(torch.arange(300, dtype=torch.int32)), up(cache), up(scales)),), (cache, scales)))
            back = up(every(torch.zeros(2, 100, 4, 64, dtype=dtype)) if name == "elements" else torch.zeros(2, 100, 4, 64, dtype=dtype))
            pages = up(torch.arange(14, dtype=torch.int32).reshape(2, 7))
            made.append(("read back, %s" % name, (M.cache_load_task(cache, scales, pages, None, back),), (back,)))
        logits = up(normal(gen, 40, 9000, dtype=dtype))
        history, params = up(torch.randint(0, 9000, (40, 500), generator=gen, dtype=torch.int32)), up(torch.rand(40, 3, generator=gen) + 0.5)
        for name, into in (("vectors", dtype), ("elements", F32 if dtype != F32 else F16)):
            out = up(torch.zeros(40, 9000, dtype=into))
            made.append(("penalties, %s" % name, (M.penalty_task(logits, out, history, None, params),), (out,)))
    return made


def test_every_kernel_starts_beside_the_default_worker():
    made = tasks_of_every_variant()
    for what, tasks, outs in made:
        for o in outs:
            o.zero_()                                        # (of a cache only what is stored is written)
    for what, tasks, outs in made:
        M.launch(*tasks)
    want = [[o.clone() for o in outs] for what, tasks, outs in made]
    for what, tasks, outs in made:
        for o in outs:
            o.zero_()
    done = torch.cuda.Event()
    torch.cuda.synchronize()
    with R.Runtime(0, idle_exit_ms=8000, wait_timeout_ms=20000) as rt:
        M.register(rt)
        assert rt.peek_queue().workgroups == 3 * int(R.device_info(0)["compute_units"])
        t0 = time.perf_counter()
        for what, tasks, outs in made:
            M.launch(*tasks)
            done.record()
            while not done.query():
                assert time.perf_counter() - t0 < 5.0, "%s has not started" % what
                time.sleep(0.0002)
        assert rt.worker_alive() and time.perf_counter() - t0 < 5.0
    torch.cuda.synchronize()
    for (what, tasks, outs), was in zip(made, want):
        for o, w in zip(outs, was):
            assert bool((o == w).all()), what
