"""Model operators on streams of their own and in graphs.  The last file of the tests: PyTorch makes all its streams with the first one, and
a worker of a context that is created then may share a hardware queue with the stream that a test's other kernels are on."""
import threading

import pytest
import torch

import model_reference as ref
from paper_2604_17861_amd import model as M
from test_gpu_model import BF16, F16, F32, _let_go, cache_of, check, decode_step, normal, rope_inputs  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_decode_step_in_a_graph_replayed_on_new_values():
    t, page, length = decode_step()
    g = {k: v.cuda() for k, v in t.items()}
    values, scales, kc, ks = cache_of(9, page, 4, 64, 1, torch.float8_e4m3fn, "plain")
    _, _, vc, vs = cache_of(9, page, 4, 64, 1, torch.float8_e4m3fn, "plain")

    def step():
        q, k = M.norm_rope_qk(g["q"], g["k"], g["g"], g["g"], g["table"], g["positions"])
        M.cache_store_kv(k, g["v"], g["slots"], kc, ks, vc, vs)
        kb, vb = M.cache_load_kv(kc, ks, vc, vs, g["pages"], g["lengths"], length, dtype=BF16)
        return q, kb, vb, M.penalize_logits(g["logits"], history=g["history"], params=g["params"])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(4):
        for name in ("q", "k", "v", "logits"):
            g[name].copy_(normal(torch.Generator().manual_seed(50 + k), *g[name].shape, dtype=g[name].dtype).cuda())
        graph.replay()
        torch.cuda.synchronize()
        got = [c.clone() for c in captured]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
        z, size = ref.norm_rope(g["q"].cpu(), t["g"], t["table"], t["positions"], 1e-6, False)
        check(got[0], z, size, 16)


def test_a_captured_training_step_beside_an_eager_one_of_the_same_values():
    gen, x, g, table, p = rope_inputs((33, 4, 64), 64, BF16, F32, "each", 4)
    leaves = [x.cuda().requires_grad_(), g.cuda().requires_grad_()]
    table, p = table.cuda(), p.cuda()
    dz = normal(gen, 33, 4, 64, dtype=BF16).cuda()
    eager = M.norm_rope(*leaves, table, p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        inner = [t.detach().requires_grad_() for t in leaves]      # (leaves of its own: a graph's gradients are its own)
        torch.autograd.grad(M.norm_rope(*inner, table, p), inner, dz)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = torch.autograd.grad(M.norm_rope(*inner, table, p), inner, dz)
    want = torch.autograd.grad(eager, leaves, dz)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, want):
            assert torch.equal(a, b)


def test_streams_threads_and_repetition_give_the_same():
    gen, x, g, table, p = rope_inputs((300, 8, 128), 128, F16, F16, "each", 6)
    x, g, table, p, dz = x.cuda(), g.cuda(), table.cuda(), p.cuda(), normal(gen, 300, 8, 128, dtype=F16).cuda()
    want = M.norm_rope_backward(dz, x, g, table, p)
    torch.cuda.synchronize()
    bad = []

    def work():
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = M.norm_rope_backward(dz, x, g, table, p)
                s.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    bad.append(1)
    threads = [threading.Thread(target=work) for _ in range(3)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not bad
