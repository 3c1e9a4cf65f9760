"""Attention whose results go where its queries are, against the same into memory of its own."""
import pytest
import torch

from paper_2604_17861_amd import model as M
from test_gpu_model import BF16, F16, F32, _let_go, laid, up  # noqa: F401
from test_zzy_gpu_cache import E2M1, E4M3, I8, attend_inputs, close, on_gpu

pytestmark = pytest.mark.gpu

CASES = [
    # b, s, hq, hk, d, groups, page, longest, lengths, window, cache
    (2, 3, 6, 3, 64, 1, 16, 100, (100, 2), 0, "plain"),
    (1, 9, 8, 2, 128, 4, 16, 200, None, 30, "heads"),
    (2, 1, 5, 1, 136, 1, 7, 100, (77, 100), 0, "plain"),
    (2, 4, 6, 2, 192, 3, 16, 90, (90, 2), 0, "heads"),          # (of the second sequence two queries see nothing)
    (1, 40, 4, 2, 256, 8, 64, 129, None, 17, "plain"),
    (3, 1, 8, 4, 256, 1, 16, 1300, (1300, 600, 9), 0, "plain"),  # in pieces
]


@pytest.mark.parametrize("fmt", (E2M1, I8, E4M3))
@pytest.mark.parametrize("dtype", (F32, F16, BF16))
@pytest.mark.parametrize("case", CASES)
def test_in_place_is_the_same(case, dtype, fmt):
    longest, window = case[7], case[9]
    q, caches, pages, lengths = attend_inputs(case, dtype, fmt)
    rest = (*[on_gpu(c) for c in caches], up(pages), up(lengths), longest)
    want = M.cache_attention(up(q), *rest, window=window)
    close(want, q, caches, pages, lengths, longest, q.shape[-1] ** -0.5, window)
    for layout in ("plain", "fused", "strided"):
        x = laid(q, layout)
        version = x._version
        assert M.cache_attention(x, *rest, window=window, out=x) is x and x._version == version + 1
        assert torch.equal(x, want), layout


@pytest.mark.parametrize("d", (128, 200, 256))
def test_in_place_of_more_workgroups_than_run_at_a_time(d):
    """2,048 (of 128 elements 1,024) workgroups; the last begin behind the first ones' end."""
    q, caches, pages, _ = attend_inputs((1, 2048, 8, 2, d, 1, 64, 2100, None, 0, "plain"), BF16, I8)
    rest = (*[up(c) for c in caches], up(pages), None, 2100)
    want = M.cache_attention(up(q), *rest)
    assert bool(torch.isfinite(want).all())
    for _ in range(5):
        x = up(q)
        M.cache_attention(x, *rest, out=x)
        assert torch.equal(x, want)


def test_in_place_in_a_graph():
    q, caches, pages, _ = attend_inputs((2, 3, 4, 2, 256, 1, 16, 90, None, 0, "plain"), F16, E2M1)
    rest = (*[up(c) for c in caches], up(pages), None, 90)
    x, source = up(q), up(q)
    M.cache_attention(x, *rest, out=x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.copy_(source)
        M.cache_attention(x, *rest, out=x)
    for k in range(4):
        source.copy_(up(q) * (1.0 - 0.25 * k))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, M.cache_attention(source, *rest))
