"""Attention where scores leave the numbers."""
import pytest
import torch

from paper_2604_17861_amd import model as M
from test_gpu_model import BF16, F16, F32, _let_go, up  # noqa: F401
from test_zzy_gpu_cache import E2M1, E4M3, I8, attend_inputs, close, on_gpu

pytestmark = pytest.mark.gpu

CASES = [
    # b, s, hq, hk, d, groups, page, longest, lengths, window, cache
    (2, 3, 6, 3, 64, 1, 16, 100, (100, 2), 0, "plain"),          # (of the second sequence a query sees nothing)
    (2, 3, 4, 1, 128, 4, 16, 200, (2, 150), 30, "heads"),
    (2, 3, 4, 2, 256, 1, 7, 100, (2, 77), 0, "plain"),
    (3, 2, 8, 4, 128, 1, 16, 1300, (1300, 600, 1), 0, "plain"),  # in pieces, a head for each wavefront
    (2, 2, 2, 1, 64, 2, 16, 1300, (1300, 1), 700, "heads"),      # in pieces
    (1, 1, 1, 1, 128, 1, 128, 40000, None, 0, "plain"),          # more pieces than a wavefront joins
]


@pytest.mark.parametrize("fmt", (E2M1, I8, E4M3))
@pytest.mark.parametrize("dtype", (F32, F16, BF16))
@pytest.mark.parametrize("case", CASES)
def test_a_query_all_of_whose_scores_are_minus_infinity(case, dtype, fmt):
    """A softmax has no value there; what sees nothing gets zeros all the same."""
    longest, window = case[7], case[9]
    q, caches, pages, lengths = attend_inputs(case, dtype, fmt)
    code = caches[0].view(torch.uint8)
    code[..., 0] = (code[..., 0] & 0xf0) | 3 if fmt == E2M1 else 7          # of every key the first element is above 0
    q[:, -2:, 0, 0] = -float("inf")                                         # two queries' first head
    got = M.cache_attention(up(q), *[on_gpu(c) for c in caches], up(pages), up(lengths), longest, window=window)
    o = close(got, q, caches, pages, lengths, longest, q.shape[-1] ** -0.5, window)
    for i in range(case[0]):
        n = longest if lengths is None else int(lengths[i])
        for j in range(max(0, case[1] - 2), case[1]):
            if n - case[1] + j >= 0:
                assert bool(torch.isnan(got[i, j, 0]).all())
            else:
                assert bool((got[i, j, 0] == 0).all())
    assert bool(torch.isfinite(o[:, :, 1:]).all())


def test_scores_that_leave_the_range():
    """Products of numbers that sum to less than fp32's least one are -inf; a row beside them that does not has all of the weight."""
    q, caches, pages, lengths = attend_inputs((2, 1, 4, 2, 64, 1, 16, 50, (50, 33), 0, "plain"), F32, I8)
    caches[0].copy_(torch.ones_like(caches[0]))
    caches[1].fill_(1e38)
    q.fill_(-1.0)
    ask = lambda: M.cache_attention(up(q), *[up(c) for c in caches], up(pages), up(lengths), 50, scale=1.0).cpu()
    assert bool(torch.isnan(ask()).all())
    caches[1][pages[0, 1], 4] = 1.0                          # row 20 of the first sequence
    got = ask()                                              # (three parts of a weight, their sums, a division: fewer than eight roundings of 2^-24)
    want = (caches[2][pages[0, 1], 4].float() * caches[3][pages[0, 1], 4])
    assert bool(torch.isnan(got[1]).all())
    assert bool(((got[0, 0].unflatten(0, (2, 2)) - want[:, None]).abs() <= want[:, None].abs() * 2.0 ** -21).all())
