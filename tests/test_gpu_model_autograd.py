"""Model operators and autograd on the GPU: what they write counts as written, and what would lose a derivative is refused."""
import pytest
import torch

from paper_2604_17861_amd import model as M
from test_gpu_model import _let_go, cache_of  # noqa: F401

pytestmark = pytest.mark.gpu


def test_stored_rows_count_as_written():
    _, _, kc, ks = cache_of(2, 4, 2, 8, 1, torch.int8, "heads")
    _, _, vc, vs = cache_of(2, 4, 2, 8, 1, torch.int8, "plain")
    x, slots = torch.randn(3, 2, 8, device="cuda"), torch.tensor([0, 5, 2], dtype=torch.int32, device="cuda")
    scores = torch.randn(2, 4, 2, 1, device="cuda", requires_grad=True)
    for saved, call in ((ks, lambda: M.cache_store(x, slots, kc, ks)), (vs, lambda: M.cache_store_kv(x, x, slots, kc, ks, vc, vs))):
        product = scores * saved
        call()
        with pytest.raises(RuntimeError, match="inplace"):
            product.sum().backward()
    with pytest.raises(ValueError):
        M.cache_store(x, slots, kc, ks.clone().requires_grad_())
