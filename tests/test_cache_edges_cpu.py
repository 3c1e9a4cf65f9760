"""Descriptors of the cache operators at the edges of what they take, without a GPU."""
import pytest

from paper_2604_17861_amd import runtime as R
from test_cache_cpu import BF16, C, E2M1, F16, F32, I32, I8, NO, op


def attention(b=1, s=1, hq=4, hk=2, d=256, page=16, longest=100, q=4096, out=8192, dtype=BF16, fmt=I8, pages=8, heads_first=False, alpha=0.1):
    w = d // 2 if fmt == E2M1 else d
    width = -(-longest // page)
    codes, scales = ((hk * page * w, w, page * w, 1), (hk * page, 1, page, 1)) if heads_first else ((page * hk * w, hk * w, w, 1), (page * hk, hk, 1, 1))
    cache, sc = op(fmt, *codes), op(F32, *scales)
    rows = (s * hq * d if b > 1 else 0, hq * d, d, 1)
    return C._pack(2, 0, (b, s, hq, hk, d, pages, page, 1, width, longest, 0),
                   (op(dtype, *rows, ptr=q), cache, sc, cache, sc, op(I32, width, 1), NO, op(dtype, *rows, ptr=out)), alpha)


@pytest.mark.parametrize("d", (136, 192, 256))
def test_attention_in_place_above_128_elements_asks_for_a_workspace(d):
    """Two workgroups read such a query, and each stores half of its result."""
    task = attention(d=d, s=5, out=4096)
    need = 4 * 5 * 4 * (d + 2)
    for at, n in ((0, 0), (0, need), (4096, need - 1), (4100, need)):
        with pytest.raises(R.GpuosError) as e:
            R.launch_cache(task, at, n)
        assert e.value.status == R.E_NOMEM


def test_attention_in_place_of_more_queries_than_a_grid_of_the_second_launch_takes():
    assert R.cache_workspace(attention(hq=1, hk=1, s=2 ** 26)) == 0 and R.cache_workspace(attention(hq=1, hk=1, s=2 ** 26 - 8, out=4096)) == 0
    with pytest.raises(R.GpuosError) as e:
        R.cache_workspace(attention(hq=1, hk=1, s=2 ** 26, out=4096))
    assert e.value.status == R.E_INVAL


@pytest.mark.parametrize("kw", (dict(hk=4, hq=4, d=128, longest=2048), dict(hk=8, hq=8, longest=2048), dict(hk=8, hq=8, b=64, d=128, longest=4096), dict(hk=8, hq=16, s=3, d=64, longest=700)))
def test_a_workspace_depends_on_sizes_alone(kw):
    """Heads behind places or before them, any dtype of the queries, any format."""
    kw = dict(kw, pages=2 ** 20)
    found = {(dtype, fmt, first): R.cache_workspace(attention(dtype=dtype, fmt=fmt, heads_first=first, **kw)) for dtype in (F32, F16, BF16) for fmt in (E2M1, I8) for first in (False, True)}
    assert len(set(found.values())) == 1 and found[BF16, I8, False] > 0, found


def test_a_workspace_holds_the_pieces_of_either_layout():
    """In a head for each wavefront four heads of 2,048 rows are 16 pieces of 128 rows; otherwise they are four of 512, and what is asked for is enough."""
    for first in (False, True):
        assert R.cache_workspace(attention(hk=4, hq=4, d=128, longest=2048, heads_first=first)) == 16 * 4 * 130 * 4
