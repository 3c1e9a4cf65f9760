"""Arguments of the model operators that contradict each other, on the CPU."""
import pytest
import torch

from paper_2604_17861_amd import model as M
from test_model_autograd_cpu import PAGES, a_cache, launched  # noqa: F401


@pytest.mark.parametrize("seen", (False, True))
def test_an_output_has_the_length_and_the_dtype_that_are_named(launched, seen):
    (kc, ks), (vc, vs) = a_cache(), a_cache()
    if seen:                                                 # (plans of the calls that are right)
        M.cache_load(kc, ks, PAGES, None, 3)
        M.cache_load(kc, ks, PAGES, None, 3, out=torch.zeros(1, 3, 2, 8))
    done = len(launched)
    out = lambda *shape, dtype=torch.float16: torch.zeros(shape, dtype=dtype)
    fits = out(1, 3, 2, 8)
    for bad, named in ((out(1, 4, 2, 8), None), (out(1, 2, 2, 8), None), (out(2, 3, 2, 8), None), (out(1, 3, 2, 8, 1), None), (out(1, 3, 1, 8), None), (out(3, 2, 8), None),
                       (fits, torch.float32), (fits, torch.bfloat16), (out(1, 3, 2, 8, dtype=torch.int32), None), (out(1, 3, 2, 8, dtype=torch.float64), torch.float64)):
        for call in (lambda: M.cache_load(kc, ks, PAGES, None, 3, dtype=named, out=bad), lambda: M.cache_load_kv(kc, ks, vc, vs, PAGES, None, 3, dtype=named, out=(None, bad)),
                     lambda: M.cache_load_kv(kc, ks, vc, vs, PAGES, None, 3, dtype=named, out=(bad, out(1, 3, 2, 8)))):
            with pytest.raises(ValueError):
                call()
    assert len(launched) == done
    assert M.cache_load(kc, ks, PAGES, None, 3, out=fits) is fits and M.cache_load(kc, ks, PAGES, None, 3, dtype=torch.float16, out=fits) is fits
    k, v = M.cache_load_kv(kc, ks, vc, vs, PAGES, None, 3, out=(None, fits))
    assert k.dtype == torch.float32 and v is fits
    assert M.cache_load(kc, ks, PAGES, None, 3).dtype == torch.float32 and M.cache_load(kc, ks, PAGES, None, 3, dtype=torch.bfloat16).dtype == torch.bfloat16
    assert len(launched) == done + 5


def test_two_results_have_two_outputs(launched):
    """One short, the second tensor was left out of the launch; one over, it was ignored."""
    x, o = torch.randn(3, 2, 8), torch.zeros(3, 2, 8)
    (kc, ks), (vc, vs) = a_cache(), a_cache()
    rows = torch.zeros(1, 3, 2, 8)
    for n in (0, 1, 3):
        for call in (lambda: M.norm_rope_qk(x, x, out=(o,) * n), lambda: M.cache_load_kv(kc, ks, vc, vs, PAGES, None, 3, out=(rows,) * n)):
            with pytest.raises(ValueError, match="2 entries"):
                call()
    assert not launched
    M.norm_rope_qk(x, x, out=(o, None))
    M.cache_load_kv(kc, ks, vc, vs, PAGES, None, 3, out=[rows, torch.zeros(1, 3, 2, 8)])
    assert launched == [2, 2]
