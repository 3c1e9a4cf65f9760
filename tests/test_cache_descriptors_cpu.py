"""The cache operators' module and its descriptors, which are public: without a GPU."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2604_17861_amd import model as M

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("first", ("_cache", "model"))
def test_either_module_may_be_imported_first(first):
    code = "from paper_2604_17861_amd import %s\nfrom paper_2604_17861_amd import model, _cache\nassert model.cache_attention is _cache.cache_attention and _cache.M is model" % first
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True, timeout=300)


def test_descriptors_are_public_and_check_their_tensors():
    q, cache, scales, n = torch.zeros(3, 4, 8), torch.zeros(2, 4, 2, 8, dtype=torch.int8), torch.ones(2, 4, 2, 1), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="k is a tensor on a GPU"):
        M.cache_append_task(q, q, q, n, cache, scales, cache, scales, out=q)
    with pytest.raises(ValueError, match="q is a tensor on a GPU"):
        M.cache_attention_task(q, cache, scales, cache, scales, n[:, None], n, 4, q)
