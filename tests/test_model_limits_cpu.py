"""Descriptors at the limits of their integers, without a GPU."""
import pytest

from paper_2604_17861_amd import runtime as R
from test_model_cpu import BF16, F16, F32, I8, I32, NO, grad, load, op, penalty, plan, rope, store

MOST, STRIDE = 2 ** 31 - 1, 2 ** 32 - 1


@pytest.mark.parametrize("b,v,row,last", [
    (4, MOST, STRIDE, STRIDE), (2, MOST, 1, STRIDE), (2, MOST, STRIDE, STRIDE), (MOST, 2, STRIDE, 1), (MOST, 1, STRIDE, 1), (MOST, 1, 2 ** 15, 1),
    (2 ** 14 + 1, 2, STRIDE, 2 ** 14), (2 ** 14 + 1, 2, STRIDE, 2 ** 14 + 1), (2 ** 30 + 1, 1, 2 ** 16, 1), (2 ** 30 + 2, 1, 2 ** 16, 1), (2, 4096, STRIDE, STRIDE)])
def test_an_operand_spans_2_to_the_46_elements_at_most(b, v, row, last):
    """Some of these spans are close to 2^63 in one dim, so that all dims together are over what 64 bits hold."""
    x = op(F32, row, last)
    got = penalty(b=b, v=v, n=0, x=x, out=x, history=NO, prompts=NO, params=NO, bias=NO, allowed=NO)
    assert isinstance(got, tuple) if (b - 1) * row + (v - 1) * last <= 2 ** 46 else got == R.E_INVAL


@pytest.mark.parametrize("sizes", [(1, 1, MOST, 1), (2, 1, MOST // 2, 2), (1, MOST, 1, 512), (3, 5, MOST // 15, 2)])
def test_rows_as_far_apart_as_strides_go(sizes):
    b, s, h, d = sizes
    x = op(BF16, STRIDE, STRIDE, STRIDE, STRIDE)
    assert rope(b=b, s=s, h=h, d=d, r=0, table=NO, positions=NO, gamma=NO, x=x, out=x) == R.E_INVAL


def test_a_sum_of_no_shares_needs_no_memory_for_them():
    """A tensor without elements has no address."""
    none = lambda parts, **kw: plan("GAMMA_SUM", (64, parts), (op(F32, parts, 1, ptr=0), op(BF16, 1, **kw)))
    assert all(p["chunks"] >= 1 and p["vectors"] == 0 for p in none(0))
    assert none(1) == R.E_INVAL and none(0, ptr=0) == R.E_INVAL


def test_what_has_no_elements_needs_no_address():
    """Tasks without rows, and caches without pages, as empty tensors describe them."""
    at = lambda dtype, *stride: op(dtype, *stride, ptr=0)
    rows = at(BF16, 768, 256, 64, 1)
    empty = [plans for n in (dict(b=0), dict(s=0), dict(h=0)) for plans in (
        rope(x=rows, out=rows, positions=NO, **n), grad(x=rows, dx=rows, dout=rows, partial=NO, positions=NO, **n))]
    empty += [store(s=0, x=at(BF16, 256, 128, 64, 1), slots=at(I32, 1, 1)), load(b=0, table=at(I32, 2, 1), lengths=NO, out=at(F16, 3840, 128, 64, 1)), load(l=0, out=at(F16, 128, 128, 64, 1)),
              store(h=0, x=at(BF16, 64, 64, 64, 1), cache=at(I8, 64, 64, 64, 1), scales=at(F32, 1, 1, 1, 1)),
              penalty(b=0, x=at(F32, 1000, 1), out=at(F32, 1000, 1), history=NO, prompts=NO, params=NO), penalty(v=0, x=at(F32, 1, 1), out=at(F32, 1, 1)),
              plan("GAMMA_SUM", (0, 5), (at(F32, 5, 1), at(BF16, 1)))]
    assert all(p["vectors"] == 2 and p["chunks"] == 1 for plans in empty for p in plans)
    none = dict(pages=0, cache=at(I8, 2048, 128, 64, 1), scales=at(F32, 32, 2, 1, 1))
    assert isinstance(store(**none), tuple) and isinstance(load(**none), tuple)
    # with elements they do
    for bad in (store(cache=at(I8, 2048, 128, 64, 1)), load(scales=at(F32, 32, 2, 1, 1)), load(pages=0, table=NO, **{k: none[k] for k in ("cache", "scales")}),
                store(pages=0, x=NO), load(pages=0, out=NO), rope(x=rows), rope(out=rows), penalty(x=at(F32, 1000, 1))):
        assert bad == R.E_INVAL
