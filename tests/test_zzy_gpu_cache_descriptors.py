"""The cache operators' descriptors as what a program makes and launches itself; what goes wrong inside a call."""
import pytest
import torch

from paper_2604_17861_amd import model as M
from paper_2604_17861_amd import _binding as B
from paper_2604_17861_amd import runtime as R
from paper_2604_17861_amd import streams as S
from test_gpu_model import BF16
from test_zzy_gpu_cache import E2M1, attend_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,longest", ((64, 90), (128, 1300), (256, 90), (256, 1300)))
def test_descriptors_do_what_the_functions_do(d, longest):
    q, caches, pages, lengths = (t if t is None or isinstance(t, list) else t.cuda() for t in attend_inputs((2, 3, 8, 4, d, 1, 16, longest, (longest, 9), 0, "plain"), BF16, E2M1))
    caches = [c.cuda() for c in caches]
    k, v = (torch.randn(2, 3, 4, d, device="cuda").bfloat16() for _ in range(2))
    slots = (pages[:, :1] * 16 + torch.tensor([3, 4, 5], device="cuda")).to(torch.int32)
    mine, table, into = [c.clone() for c in caches], torch.rand(3, d, device="cuda"), torch.empty_like(q)
    turned = M.cache_append_qkv(q, k, v, slots, *caches, table)
    want = M.cache_attention(turned, *caches, pages, lengths, longest)
    stream = torch.cuda.current_stream()

    def run(task, least=0):
        assert isinstance(task, bytes) and len(task) == S.CACHE_TASK_BYTES
        space = torch.empty(max(least, R.cache_workspace(task)), dtype=torch.uint8, device="cuda")
        R.launch_cache(task, space.data_ptr(), space.numel(), stream.device_index, stream.cuda_stream)
        torch.cuda.synchronize()
    run(M.cache_append_task(q, k, v, slots, *mine, table, out=into))
    assert torch.equal(into, turned) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(mine, caches))
    out = torch.empty_like(q)
    run(M.cache_attention_task(into, *mine, pages, lengths, longest, out))
    assert torch.equal(out, want)
    run(M.cache_attention_task(into, *mine, pages, lengths, longest, into), 4 * 2 * 3 * 8 * (d + 2))      # in place
    assert torch.equal(into, want)


def test_no_memory_is_an_error_of_its_own():
    x = torch.zeros(1, device="cuda").expand(2 ** 44)        # (64 TB: refused at once)
    with pytest.raises(torch.OutOfMemoryError):
        B.like(x)
