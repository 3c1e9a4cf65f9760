"""What the model operators tell autograd, and what they refuse because they can not: on the CPU, with the library's launch replaced by
one that takes the descriptors and computes nothing."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from torch.autograd import forward_ad
from torch.fx.experimental.proxy_tensor import make_fx
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2604_17861_amd import model as M
from paper_2604_17861_amd import runtime as R


@pytest.fixture
def launched(monkeypatch):
    """Operators on tensors of the CPU; the number of descriptors of every launch."""
    calls, check = [], M._check
    monkeypatch.setattr(M, "_check", lambda x, what, dtypes=None, dims=None, shape=None, device=None, **kw: check(
        x, what, dtypes, dims, shape, x.device if device is None and isinstance(x, torch.Tensor) else device, **kw))
    monkeypatch.setattr(M, "_stream_of", lambda device: 0)
    monkeypatch.setattr(R, "launch_model_at", lambda tasks, n, device, stream: calls.append(n))
    monkeypatch.setattr(M, "_plans", {})
    return calls


def a_cache(groups=1):
    return torch.zeros(2, 4, 2, 8, dtype=torch.int8), torch.ones(2, 4, 2, groups)


SLOTS = torch.tensor([0, 5, 2], dtype=torch.int32)
PAGES = torch.tensor([[1]], dtype=torch.int32)


def test_stored_rows_count_as_written(launched):
    x = torch.randn(3, 2, 8)
    (kc, ks), (vc, vs) = a_cache(), a_cache()
    scores = torch.randn(2, 4, 2, 1, requires_grad=True)
    for call, tensors in ((lambda: M.cache_store(x, SLOTS, kc, ks), (kc, ks)), (lambda: M.cache_store_kv(x, x, SLOTS, kc, ks, vc, vs), (kc, ks, vc, vs))):
        before = [t._version for t in tensors]
        product = scores * ks                                # keeps the scales for the gradient
        call()
        assert all(t._version > v for t, v in zip(tensors, before))
        with pytest.raises(RuntimeError, match="inplace"):
            product.sum().backward()
    assert launched == [1, 2]


def test_scales_that_require_a_gradient_are_not_overwritten(launched):
    x = torch.randn(3, 2, 8)
    (kc, ks), (vc, vs) = a_cache(), a_cache()
    vs.requires_grad_()
    for call in (lambda: M.cache_store(x, SLOTS, vc, vs), lambda: M.cache_store_kv(x, x, SLOTS, kc, ks, vc, vs)):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    with torch.inference_mode():                             # (tensors without versions)
        M.cache_store(x, SLOTS, *a_cache())
    assert launched == [1, 2, 1]


def test_a_refused_call_has_written_nothing(launched, monkeypatch):
    x, out, bad = torch.randn(3, 2, 8), torch.zeros(3, 2, 8), torch.zeros(3, 2, 9)
    (kc, ks), rows = a_cache(), torch.zeros(1, 3, 2, 8)
    short = torch.zeros(2, dtype=torch.int32)
    calls = [(out, lambda: M.norm_rope(bad, out=out)), (out, lambda: M.norm_rope_qk(x, bad, out=(out, out))), (rows, lambda: M.cache_load(kc, kc, PAGES, None, 3, out=rows)),
             (ks, lambda: M.cache_store(x, short, kc, ks)), (out, lambda: M.penalize_logits(x, out=out))]
    for tensor, call in calls:
        with pytest.raises(ValueError):
            call()
        assert tensor._version == 0
    for tensor, call in ((out, lambda: M.norm_rope(x, out=out)), (rows, lambda: M.cache_load(kc, ks, PAGES, None, 3, out=rows)), (ks, lambda: M.cache_store(x, SLOTS, kc, ks))):
        def refuse(*args):
            raise R.GpuosError(R.E_INVAL, "gpuos_launch_model")
        with monkeypatch.context() as m:
            m.setattr(R, "launch_model_at", refuse)          # by the library
            with pytest.raises(R.GpuosError):
                call()
        assert tensor._version == 0
        call()
        assert tensor._version == 1


def test_results_that_would_be_cut_off_from_a_gradient_are_refused(launched):
    x, w, g = torch.randn(3, 2, 8), torch.randn(3, 2, 8, requires_grad=True), torch.ones(8, requires_grad=True)
    plain = g.detach()
    (kc, ks), (vc, vs) = a_cache(), a_cache()
    ws = ks.clone().requires_grad_()
    table = torch.randn(4, 8, requires_grad=True)
    logits, wl = torch.randn(2, 5), torch.randn(2, 5, requires_grad=True)
    history, params = torch.zeros(2, 3, dtype=torch.int32), torch.ones(2, 3, requires_grad=True)
    calls = [lambda: M.cache_load(kc, ws, PAGES, None, 3), lambda: M.cache_load_kv(kc, ks, vc, ws, PAGES, None, 3),
             lambda: M.cache_store(w, SLOTS, kc, ks), lambda: M.cache_store_kv(x, w, SLOTS, kc, ks, vc, vs),
             lambda: M.norm_rope_backward(w, x), lambda: M.norm_rope_backward(x, w), lambda: M.norm_rope_backward(x, x, g), lambda: M.norm_rope_backward(x, x, plain, table),
             lambda: M.norm_rope_qk_backward(x, x, x, w), lambda: M.norm_rope_qk_backward(x, x, x, x, plain, g), lambda: M.norm_rope_qk_backward(w, x, x, x),
             lambda: M.norm_rope(x, plain, table), lambda: M.norm_rope_qk(x, x, plain, plain, table), lambda: M.penalize_logits(wl),
             lambda: M.penalize_logits(logits, history=history, params=params), lambda: M.penalize_logits(logits, bias=wl)]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
    assert not launched
    with torch.no_grad():
        for call in calls:
            call()
    assert len(launched) == len(calls)


def test_backward_passes_go_through(launched):
    """The refusals are for callers: autograd's own calls are not among them."""
    q, k, g = torch.randn(3, 2, 8, requires_grad=True), torch.randn(3, 1, 8), torch.ones(8, requires_grad=True)
    zq, zk = M.norm_rope_qk(q, k, g, g)
    grads = torch.autograd.grad((zq, zk), (q, g), (torch.ones_like(zq), torch.ones_like(zk)))
    assert [t.shape for t in grads] == [q.shape, g.shape] and launched == [2, 4]
    (grad,) = torch.autograd.grad(M.norm_rope(q).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):                        # twice is refused by autograd
        grad.sum().backward()


@pytest.mark.filterwarnings("ignore::DeprecationWarning")
def test_tangents_of_forward_mode_are_refused(launched):
    x, table, g = torch.randn(3, 2, 8), torch.randn(4, 8), torch.ones(8)
    logits, bias = torch.randn(2, 5), torch.randn(5)
    kc, ks = a_cache()
    leaf = x.clone().requires_grad_()
    later = M.norm_rope(leaf)                                # a forward pass outside, its gradient inside
    rows = torch.zeros(1, 3, 2, 8)
    calls = [(x, lambda d: M.norm_rope(d)), (g, lambda d: M.norm_rope(x, d)), (table, lambda d: M.norm_rope(x, g, d)), (x, lambda d: M.norm_rope_qk(x, d)),
             (logits, lambda d: M.penalize_logits(d)), (bias, lambda d: M.penalize_logits(logits, bias=d)), (ks, lambda d: M.cache_load(kc, d, PAGES, None, 3)),
             (x, lambda d: M.cache_store(d, SLOTS, kc, ks)), (x, lambda d: M.norm_rope_backward(d, x)), (x, lambda d: M.norm_rope_backward(x, d)),
             (rows, lambda d: M.cache_load(kc, ks, PAGES, None, 3, out=d)), (x, lambda d: torch.autograd.grad(later, leaf, d, retain_graph=True))]
    done = len(launched)
    with forward_ad.dual_level():
        for t, call in calls:
            dual = forward_ad.make_dual(t, torch.ones_like(t))
            with pytest.raises(ValueError, match="forward-mode"):
                call(dual)
        with pytest.raises(ValueError, match="forward-mode"):      # both at once
            M.norm_rope(forward_ad.make_dual(leaf, torch.ones_like(leaf)))
        assert len(launched) == done
        M.norm_rope(x, g, table)                             # without a tangent
        torch.autograd.grad(later, leaf, x)
    for t, call in calls[:-1]:
        call(t)
    assert len(launched) == done + 2 + len(calls) - 1


TRACES = {"make_fx": dict(), "fake": dict(tracing_mode="fake"), "symbolic": dict(tracing_mode="symbolic"), "before dispatch": dict(pre_dispatch=True)}


@pytest.mark.filterwarnings("ignore")
@pytest.mark.parametrize("how", [*TRACES, "jit", "export", "fake tensors", "functionalize"])
@pytest.mark.parametrize("seen", (False, True))
def test_traces_are_refused(launched, how, seen):
    """A trace would hold the allocation of the results only."""
    x, logits = torch.randn(3, 2, 8), torch.randn(2, 5)
    (kc, ks) = a_cache()

    class One(torch.nn.Module):
        def __init__(self, f):
            super().__init__()
            self.f = f

        def forward(self, t):
            return self.f(t)

    def trace(f, t):
        if how in TRACES:
            return make_fx(f, **TRACES[how])(t)
        if how == "jit":
            return torch.jit.trace(f, t, check_trace=False)
        if how == "export":
            return torch.export.export(One(f), (t,), strict=False)
        if how == "functionalize":
            return torch.func.functionalize(f)(t)
        with FakeTensorMode():
            fake = torch.empty(t.shape)
        return f(fake)
    calls = [(x, lambda t: M.norm_rope(t)), (x, lambda t: M.norm_rope(t, out=t)), (logits, lambda t: M.penalize_logits(t)),
             (x, lambda t: M.norm_rope_qk(t, t)[0]), (ks, lambda t: M.cache_load(kc, t, PAGES, None, 3)), (x, lambda t: M.norm_rope_backward(t, t)[0])]
    for t, call in calls:
        if seen:
            call(t)                                          # (its plan is there)
        done = len(launched)
        with pytest.raises((ValueError, RuntimeError, AssertionError, TypeError)):      # (fake tensors and symbols by PyTorch itself)
            trace(call, t)
        assert len(launched) == done
        call(t)
        assert len(launched) == done + 1


def test_modes_that_trace_nothing_are_let_through(launched):
    class Seen(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))
    with Seen(), torch.device("cpu"):
        M.norm_rope(torch.randn(3, 2, 8))
    assert launched == [1]


def test_compiled_programs_call_the_operators(launched):
    x = torch.randn(3, 2, 8)
    program = torch.compile(lambda x: M.norm_rope(x * 2.0) + 1.0, backend="eager")
    for _ in range(3):
        program(x)
    assert len(launched) == 3
    torch._dynamo.reset()


def test_a_tensor_whose_memory_was_let_go_is_refused(launched):
    x, g = torch.randn(3, 2, 8), torch.ones(8)
    M.norm_rope(x, g)
    g.untyped_storage().resize_(0)
    with pytest.raises(ValueError, match="without memory"):
        M.norm_rope(x, g)
    assert launched == [1]


def test_gradients_that_are_lazily_negated_go_through(launched):
    """What autograd hands back through the imaginary part of a conjugate."""
    x = torch.randn(3, 2, 8, requires_grad=True)
    torch.complex(torch.zeros(3, 2, 8), M.norm_rope(x)).conj().abs().sum().backward()
    assert launched == [1, 1] and x.grad is not None


@pytest.mark.filterwarnings("ignore:Using backward")
def test_second_derivatives_raise_also_on_the_way_to_others(launched):
    x, g = torch.randn(3, 2, 8, requires_grad=True), torch.ones(8, requires_grad=True)
    other = torch.randn(3, requires_grad=True)
    dz = torch.randn(3, 2, 8)
    for leaves in ((x,), (x, g), (g,)):
        z = M.norm_rope(x, g)
        grads = torch.autograd.grad(z, leaves, dz, create_graph=True)
        assert all(t.requires_grad for t in grads)
        with pytest.raises(RuntimeError, match="not differentiable themselves"):
            (other.sum() + sum(t.square().sum() for t in grads)).backward()
    with pytest.raises(RuntimeError, match="not differentiable themselves"):      # by way of dout
        torch.autograd.functional.jvp(lambda t: M.norm_rope(t), x.detach(), dz)
    # the first ones are there all the same, and what does not need the second goes its way
    x.grad = g.grad = other.grad = None                      # (of the passes that ended on their way)
    z = M.norm_rope(x, g)
    (z.sum() + other.square().sum()).backward(create_graph=True)
    assert x.grad.shape == x.shape and g.grad.shape == g.shape and torch.equal(other.grad, 2 * other)
    x.grad = g.grad = other.grad = None
    q, k = M.norm_rope_qk(x, torch.randn(3, 1, 8), None, g)
    grads = torch.autograd.grad((q, k), (x, g), (dz, torch.ones(3, 1, 8)), create_graph=True)
    assert [t.shape for t in grads] == [x.shape, g.shape]
