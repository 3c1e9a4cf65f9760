"""Model operators on the GPU round their arithmetic: what they write counts as written for autograd, what would lose a derivative is refused,
tensors without elements are nothing to do."""
import pytest
import torch
from torch.autograd import forward_ad
from torch.fx.experimental.proxy_tensor import make_fx

import model_reference as ref
from paper_2604_17861_amd import model as M
from test_gpu_model import BF16, F32, ROUTES, _let_go, cache_of, check, normal, rope_inputs, run, up  # noqa: F401

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


def test_traces_and_tangents_are_refused():
    x = torch.randn(3, 2, 8, device="cuda")
    want = M.norm_rope(x)
    for trace in (lambda: make_fx(lambda t: M.norm_rope(t))(x), lambda: make_fx(lambda t: M.norm_rope(t), pre_dispatch=True)(x),
                  lambda: torch.jit.trace(lambda t: M.norm_rope(t), x, check_trace=False)):
        with pytest.raises(ValueError, match="traced"):
            trace()
    with forward_ad.dual_level():
        with pytest.raises(ValueError, match="forward-mode"):
            M.norm_rope(forward_ad.make_dual(x, torch.ones_like(x)))
    assert torch.equal(M.norm_rope(x), want)


@pytest.mark.parametrize("route", ROUTES)
def test_the_sums_of_no_shares_are_zeros(route):
    partial = up(torch.empty(70, 0))
    out = torch.full((70,), 7.0, device="cuda")
    run(route, M.gamma_sum_task(partial, out))
    assert (out == 0).all()


def test_a_gradient_through_complex_numbers():
    """The loss is that of the imaginary part alone, whose gradient comes back lazily negated."""
    x, zero = torch.randn(30, 2, 64, device="cuda"), torch.zeros(30, 2, 64, device="cuda")
    grads = []
    for loss in (lambda z: torch.complex(zero, z).conj().abs().sum(), lambda z: z.abs().sum()):
        leaf = x.clone().requires_grad_()
        loss(M.norm_rope(leaf, eps=0.1)).backward()
        grads.append(leaf.grad)
    # The gradients at z are 1 or -1 either way, off by two half steps (of |z| and z / |z|).  dx = r (u - x r^2 mean(u x)) has terms of
    # r (1 + |x| r mean(|x| r)) <= 10 ** 0.5 * (1 + 64 ** 0.5) < 29, and 56 roundings of them in either run.
    torch.testing.assert_close(grads[0], grads[1], rtol=0, atol=(2 + 2 * 56) * 29 * 2.0 ** -24)


@pytest.mark.parametrize("route", ROUTES)
def test_empty_tensors_in_descriptors(route):
    e, x, out = up(torch.empty(0, 2, 64)), up(torch.randn(5, 2, 64)), up(torch.zeros(5, 2, 64))
    none, some = up(torch.empty(0, dtype=torch.int32)), up(torch.zeros(3, 2, dtype=torch.int32))
    cache, scales = up(torch.empty(0, 4, 2, 64, dtype=torch.int8)), up(torch.empty(0, 4, 2, 1))
    back = up(torch.zeros(3, 7, 2, 64))
    lengths = up(torch.tensor([7, 0, 3], dtype=torch.int32))
    run(route, M.norm_rope_task(e, None, None, None, e), M.norm_rope_task(x, None, None, None, out), M.cache_store_task(e, none, cache, scales),
        M.penalty_task(up(torch.empty(0, 9)), up(torch.empty(0, 9))),
        # a cache without pages: nothing is stored, and what is read back is in no page
        M.cache_store_task(x, up(torch.arange(5, dtype=torch.int32)), cache, scales), M.cache_load_task(cache, scales, some, lengths, back))
    assert torch.equal(out, M.norm_rope(x))
    for b, n in enumerate((7, 0, 3)):
        assert torch.isnan(back[b, :n]).all() and (back[b, n:] == 0).all()
    M.cache_store(x, up(torch.arange(5, dtype=torch.int32)), cache, scales)
    assert torch.isnan(M.cache_load(cache, scales, some, None, 7)).all()


def test_gradients_that_keep_their_graph_are_the_same_and_are_not_differentiated_again():
    gen, x, g, table, p = rope_inputs((33, 4, 64), 64, BF16, F32, "each", 4)
    leaves = [x.cuda().requires_grad_(), g.cuda().requires_grad_()]
    table, p, dz = table.cuda(), p.cuda(), normal(gen, 33, 4, 64, dtype=BF16).cuda()
    want = torch.autograd.grad(M.norm_rope(*leaves, table, p), leaves, dz)
    got = torch.autograd.grad(M.norm_rope(*leaves, table, p), leaves, dz, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(RuntimeError, match="not differentiable themselves"):
        (leaves[1].sum() + got[0].float().square().sum()).backward()


@pytest.mark.parametrize("frozen", ("gamma", "x", "k"))
def test_gradients_of_some_inputs_only(frozen):
    gen, q, g, table, p = rope_inputs((70, 4, 64), 64, BF16, F32, "each", 31)
    k, dq, dk = (normal(gen, 70, n, 64, dtype=BF16) for n in (2, 4, 2))
    leaves = [t.cuda() for t in (q, k, g)]
    if frozen != "gamma":
        leaves[2].requires_grad_()
    if frozen != "x":
        leaves[0].requires_grad_()
        if frozen != "k":
            leaves[1].requires_grad_()
    zq, zk = M.norm_rope_qk(leaves[0], leaves[1], leaves[2], leaves[2], table.cuda(), p.cuda())
    torch.autograd.backward((zq, zk), (dq.cuda(), dk.cuda()))
    dgs = 0.0
    size = 0.0
    for leaf, dz, x in ((leaves[0], dq, q), (leaves[1], dk, k)):
        dx, s, dg, gs = ref.norm_rope_grad(dz, x, g, table, p, 1e-6, False)
        dgs, size = dgs + dg, size + gs
        assert (leaf.grad is None) == (not leaf.requires_grad)
        if leaf.requires_grad:
            check(leaf.grad, dx, s, 56)
    assert (leaves[2].grad is None) == (frozen == "gamma")
    if frozen != "gamma":                                    # (two sums of at most 280 rows, and their sum)
        check(leaves[2].grad, dgs, size, 56 + 280 + 256 + 8 + 4 + 1)
