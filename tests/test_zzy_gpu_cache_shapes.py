"""Attention where its ways of sharing out work meet: a head for each wavefront with windows, numbers of heads that are no multiple of four,
pages of one place, wide joins of heads above 128, several tiles of queries with pieces."""
import pytest
import torch

from paper_2604_17861_amd import model as M
from test_gpu_model import BF16, F16, F32, _let_go, up  # noqa: F401
from test_zzy_gpu_cache import E2M1, E4M3, I8, attend_inputs, close, on_gpu

pytestmark = pytest.mark.gpu

CASES = [
    # b, s, hq, hk, d, groups, page, longest, lengths, window, cache
    (2, 2, 8, 4, 128, 1, 16, 1500, (1500, 800), 600, "plain"),       # a head for each wavefront, a window
    (1, 3, 10, 5, 64, 1, 16, 900, None, 700, "plain"),               # five heads: three wavefronts of eight have none
    (2, 1, 3, 3, 128, 4, 32, 700, (700, 1), 0, "plain"),
    (1, 1, 6, 6, 256, 1, 16, 1100, None, 0, "plain"),
    (1, 2, 10, 10, 72, 1, 5, 800, (799,), 0, "plain"),
    (2, 1, 8, 4, 128, 1, 1, 900, (900, 513), 0, "plain"),            # pages of one place
    (1, 4, 16, 4, 64, 2, 1, 700, None, 600, "heads"),
    (1, 20, 4, 1, 64, 1, 16, 1500, (1400,), 0, "plain"),             # five tiles of queries, pieces
    (1, 9, 8, 4, 200, 1, 64, 1200, None, 0, "heads"),
    (1, 1, 2, 1, 256, 8, 128, 40000, None, 0, "plain"),              # more pieces than a wavefront joins
    (1, 1, 1, 1, 136, 1, 64, 36000, (35000,), 0, "heads"),
]


@pytest.mark.parametrize("fmt", (E2M1, I8, E4M3))
@pytest.mark.parametrize("dtype", (F32, F16, BF16))
@pytest.mark.parametrize("case", CASES)
def test_attention(case, dtype, fmt):
    longest, window = case[7], case[9]
    q, caches, pages, lengths = attend_inputs(case, dtype, fmt, seed=7)
    got = M.cache_attention(up(q), *[on_gpu(c) for c in caches], up(pages), up(lengths), longest, window=window)
    close(got, q, caches, pages, lengths, longest, q.shape[-1] ** -0.5, window)


@pytest.mark.parametrize("d", (64, 128, 256))
def test_lengths_below_zero_and_past_the_longest(d):
    """A length below 0 counts as 0, one over `longest` as it; so do the ends of the integers."""
    q, caches, pages, _ = attend_inputs((5, 2, 4, 4, d, 1, 16, 600, None, 0, "plain"), F16, I8)
    mine = [up(c) for c in caches]
    odd = torch.tensor([-1, -2 ** 31, 2 ** 31 - 1, 601, 1], dtype=torch.int32)
    plain = torch.tensor([0, 0, 600, 600, 1], dtype=torch.int32)
    got, want = (M.cache_attention(up(q), *mine, up(pages), up(n), 600) for n in (odd, plain))
    assert torch.equal(got, want) and bool((got[:2] == 0).all()) and bool((got[4, 0] == 0).all())
    close(got, q, caches, pages, plain, 600, d ** -0.5, 0)
