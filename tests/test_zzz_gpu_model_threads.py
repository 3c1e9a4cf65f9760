"""Model operators from several threads, each on a stream of its own, with every thread's end looked at.  (Behind the tests that have no
streams of their own: see test_zzz_gpu_model_streams.py.)"""
import threading

import pytest
import torch

from paper_2604_17861_amd import model as M
from test_gpu_model import F16, _let_go, cache_of, normal, rope_inputs  # noqa: F401

pytestmark = pytest.mark.gpu


def in_threads(n, work):
    """work(k) in n threads; what they return, or what one of them raised."""
    results, raised = [None] * n, []

    def run(k):
        try:
            results[k] = work(k)
        except BaseException as e:                           # (a thread's exception ends the thread only)
            raised.append(e)
    threads = [threading.Thread(target=run, args=(k,)) for k in range(n)]
    [t.start() for t in threads]
    [t.join(60) for t in threads]
    assert not any(t.is_alive() for t in threads)
    if raised:
        raise raised[0]
    return results


def test_threads_and_streams_of_their_own_give_the_same_and_all_end():
    gen, x, g, table, p = rope_inputs((300, 8, 128), 128, F16, F16, "each", 6)
    x, g, table, p, dz = x.cuda(), g.cuda(), table.cuda(), p.cuda(), normal(gen, 300, 8, 128, dtype=F16).cuda()
    logits, history, params = normal(gen, 9, 5001).cuda(), torch.randint(0, 5001, (9, 77), generator=gen, dtype=torch.int32).cuda(), torch.rand(9, 3, generator=gen).cuda() + 0.5
    _, _, cache, scales = cache_of(5, 64, 8, 128, 1, torch.int8, "plain")
    pages = torch.arange(5, dtype=torch.int32, device="cuda")[None]

    def once():
        return (*M.norm_rope_backward(dz, x, g, table, p), M.norm_rope(x, g, table, p), M.penalize_logits(logits, history=history, params=params),
                M.cache_load(cache, scales, pages, None, 300, dtype=F16))
    want = once()
    torch.cuda.synchronize()

    def work(k):
        stream, rounds = torch.cuda.Stream(), 0
        with torch.cuda.stream(stream):
            for _ in range(20):
                if k == 0:
                    M._plans.clear()                         # (as a full table of plans does)
                got = once()
                stream.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want))
                rounds += 1
        return rounds
    assert in_threads(4, work) == [20] * 4
