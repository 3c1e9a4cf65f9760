"""Descriptors at the limits of their integers, without a GPU."""
import pytest

from paper_2604_17861_amd import runtime as R
from test_model_cpu import BF16, F32, NO, op, penalty, plan, rope

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
