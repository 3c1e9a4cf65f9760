"""Cache operators on streams of their own, in threads and in graphs.  Runs last, as the model operators' like it: PyTorch makes all its streams
with the first one."""
import threading

import pytest
import torch

import cache_reference as ref
from paper_2604_17861_amd import model as M
from test_zzy_gpu_cache import E2M1, I8, attend_inputs, caches_of, close
from test_gpu_model import BF16, F16, _let_go, normal, same, up  # noqa: F401

pytestmark = pytest.mark.gpu


def a_step(longest, fmt, seed):
    """Inputs of a decoding step whose attention is in pieces where `longest` is long."""
    gen = torch.Generator().manual_seed(seed)
    b, hq, hk, d, page = 3, 8, 4, 128, 16
    per = -(-longest // page)
    caches = caches_of(b * per + 1, page, hk, d, 4, fmt, "plain", gen)
    t = dict(qkv=normal(gen, b, hq + 2 * hk, d, dtype=BF16), table=torch.rand(longest, d, generator=gen),
             lengths=torch.tensor([longest, longest // 2, 7], dtype=torch.int32), pages=torch.randperm(b * per, generator=gen).to(torch.int32).reshape(b, per))
    t["positions"] = t["lengths"] - 1
    last = t["positions"].long()
    t["slots"] = (t["pages"].long().gather(1, (last // page)[:, None])[:, 0] * page + last % page).to(torch.int32)
    return t, caches


def step(g, caches, longest):
    x = g["qkv"]
    q = M.cache_append_qkv(x[:, :8], x[:, 8:12], x[:, 12:], g["slots"], *caches, g["table"], g["positions"])
    return q, M.cache_attention(q, *caches, g["pages"], g["lengths"], longest)


def test_two_graphs_of_steps_replayed_in_turn_on_new_values():
    """The second step's attention is in pieces; its workspace is its graph's own."""
    made = []
    for longest, fmt in ((300, I8), (2500, E2M1), (2500, E2M1)):
        t, caches = a_step(longest, fmt, longest + len(made))
        g, mine = {k: up(v) for k, v in t.items()}, [up(c) for c in caches]
        step(g, mine, longest)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = step(g, mine, longest)
        made.append((graph, captured, g, mine, longest, t))
    for k in range(4):
        for graph, captured, g, mine, longest, t in made:
            t["qkv"] = normal(torch.Generator().manual_seed(60 + k), *g["qkv"].shape, dtype=BF16)
            t["lengths"] = torch.tensor([longest - k, 9 + k, 7], dtype=torch.int32)
            g["qkv"].copy_(t["qkv"])
            g["lengths"].copy_(t["lengths"])
        for graph, *_ in made:                               # (one behind the other, nothing waited for)
            graph.replay()
        torch.cuda.synchronize()
        for graph, captured, g, mine, longest, t in made:
            got = [c.clone() for c in captured]
            for a, b in zip(got, step(g, mine, longest)):
                assert torch.equal(a, b)
            if k == 3:
                close(got[1][:, None], got[0].cpu()[:, None], [c.cpu() for c in mine], t["pages"], t["lengths"], longest, 128 ** -0.5, 0)


def test_streams_threads_and_repetition_give_the_same():
    t, caches = a_step(2500, E2M1, 4)
    g, mine = {k: up(v) for k, v in t.items()}, [up(c) for c in caches]
    want = step(g, mine, 2500)
    torch.cuda.synchronize()
    bad = []

    def work(side):
        s = torch.cuda.Stream() if side else torch.cuda.current_stream()
        try:
            with torch.cuda.stream(s), torch.no_grad():
                for _ in range(20):
                    got = M.cache_attention(want[0], *mine, g["pages"], g["lengths"], 2500)
                    s.synchronize()
                    if not torch.equal(got, want[1]):
                        bad.append("other values")
        except Exception as e:                               # (of a thread nobody else hears)
            bad.append(e)
    threads = [threading.Thread(target=work, args=(k > 0,)) for k in range(4)]
    [x.start() for x in threads]
    [x.join(60) for x in threads]
    assert not bad and not any(x.is_alive() for x in threads)


def test_rows_of_another_stream_than_the_current_one():
    """What was made on one stream is used on another behind an event, and its memory given back at once."""
    q, caches, pages, lengths = attend_inputs((2, 1, 8, 4, 128, 1, 16, 1200, (1200, 800), 0, "plain"), F16, I8)
    mine, table, n = [up(c) for c in caches], up(pages), up(lengths)
    want = M.cache_attention(up(q), *mine, table, n, 1200)
    side = torch.cuda.Stream()
    for _ in range(5):
        x = up(q) * 1.0
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = M.cache_attention(x, *mine, table, n, 1200)
            x.record_stream(side)
        del x
        torch.empty(1 << 20, device="cuda").fill_(1.0)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
