"""Cache operators without a GPU: their descriptors' checks, their arguments' on tensors of the CPU with the launch replaced, what they tell
autograd and refuse, the keys of calls, and whether their kernels fit beside a worker."""
import struct

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from torch.autograd import forward_ad
from torch.fx.experimental.proxy_tensor import make_fx

import cache_reference as ref
from paper_2604_17861_amd import model as M
from paper_2604_17861_amd import _binding as B
from paper_2604_17861_amd import _cache as C
from paper_2604_17861_amd import runtime as R
from test_model_autograd_cpu import launched as _launched  # noqa: F401
from test_model_registers_cpu import kernels

F32, F16, BF16, I32, I8, E4M3, E2M1 = 0, 1, 2, 3, 4, 5, 6
NO = (0, 0, 0, 0, 0, 0)
MOST = 2 ** 31 - 1


def op(dtype, *stride, ptr=4096):
    return (ptr, *stride, *(0,) * (4 - len(stride)), dtype)


def plan(kind, sizes, operands, flags=0, alpha=1.0):
    """The workspace of a task, or the status of a refused one."""
    try:
        return R.cache_workspace(C._pack(kind, flags, sizes, operands, alpha))
    except R.GpuosError as e:
        return e.status


def append(b=2, s=3, hq=4, hk=2, d=64, r=64, places=10, pages=8, page=16, groups=1, flags=0, **kw):
    width = d // 2
    o = dict(q=op(BF16, s * hq * d, hq * d, d, 1), k=op(BF16, s * hk * d, hk * d, d, 1), v=op(BF16, s * hk * d, hk * d, d, 1), table=op(F32, r, 1), positions=op(I32, s, 1),
             slots=op(I32, s, 1), out=op(BF16, s * hq * d, hq * d, d, 1), kc=op(E2M1, page * hk * width, hk * width, width, 1), ks=op(F32, page * hk * groups, hk * groups, groups, 1))
    o.update(vc=o["kc"], vs=o["ks"])
    o.update(kw)
    return plan(1, (b, s, hq, hk, d, r, places, pages, page, groups), tuple(o.values()), flags)


def attend(b=2, s=1, hq=4, hk=2, d=64, pages=8, page=16, groups=1, width=4, longest=60, window=0, flags=0, alpha=0.1, **kw):
    w = d // 2
    o = dict(q=op(BF16, s * hq * d, hq * d, d, 1), kc=op(E2M1, page * hk * w, hk * w, w, 1), ks=op(F32, page * hk * groups, hk * groups, groups, 1))
    o.update(vc=o["kc"], vs=o["ks"], table=op(I32, width, 1), lengths=op(I32, 1), out=op(BF16, s * hq * d, hq * d, d, 1))
    o.update(kw)
    return plan(2, (b, s, hq, hk, d, pages, page, groups, width, longest, window), tuple(o.values()), flags, alpha)


def test_descriptors_that_are_taken():
    assert append() == 0 and append(flags=4) == 0 and append(r=0, table=NO, positions=NO) == 0 and append(positions=NO) == 0
    assert append(hq=0, q=NO, out=NO) == 0 and append(b=0) == 0 and append(hk=0) == 0 and append(groups=8) == 0 and append(d=2, r=2) == 0
    assert attend() == 0 and attend(lengths=NO) == 0 and attend(b=0) == 0 and attend(longest=0, table=op(I32, 4, 1, ptr=0)) == 0 and attend(window=MOST) == 0
    assert attend(groups=2) == 0 and attend(d=256, groups=8) == 0 and attend(hq=64) == 0
    # pieces: 1,024 rows of two sequences of one head are two each, of 4 queries of 64 elements with two numbers beside
    assert attend(hk=1, longest=1024, width=64) == 2 * 2 * 4 * 66 * 4
    assert attend(b=800, longest=1024, width=64) == 0 and attend(longest=1024, width=64, window=20) == 0


@pytest.mark.parametrize("bad", [
    dict(d=0), dict(d=513), dict(d=63), dict(r=63), dict(r=66), dict(r=-2), dict(places=0), dict(page=0), dict(pages=2 ** 30), dict(groups=3), dict(groups=16), dict(groups=0), dict(flags=1),
    dict(b=MOST, s=2), dict(b=2 ** 20, s=2 ** 10), dict(b=2 ** 16, s=2 ** 10, hq=64), dict(hq=-1),
    dict(q=NO), dict(k=NO), dict(v=NO), dict(out=NO), dict(slots=NO), dict(table=NO), dict(kc=NO), dict(vs=NO),
    dict(q=op(F16, 768, 256, 64, 1)), dict(v=op(F32, 384, 128, 64, 1)), dict(out=op(F32, 768, 256, 64, 1)), dict(k=op(I8, 384, 128, 64, 1)), dict(slots=op(F32, 3, 1)), dict(positions=op(F32, 3, 1)),
    dict(table=op(BF16, 64, 1)), dict(table=op(F32, 64, 2)), dict(kc=op(I8, 2048, 128, 64, 1)), dict(vc=op(E4M3, 2048, 128, 64, 1)), dict(kc=op(BF16, 1024, 64, 32, 1)), dict(ks=op(BF16, 32, 2, 1, 1)),
    dict(kc=op(E2M1, 1024, 64, 32, 2)), dict(out=op(BF16, 768, 0, 64, 1)), dict(vc=op(E2M1, 1024, 64, 0, 1)), dict(ks=op(F32, 32, 0, 1, 1)), dict(q=op(BF16, -1, 256, 64, 1)),
    dict(k=op(BF16, 2 ** 32, 128, 64, 1)), dict(q=op(BF16, 768, 256, 64, 1, ptr=4097))])
def test_descriptors_of_appending_that_are_refused(bad):
    assert append(**bad) == R.E_INVAL


@pytest.mark.parametrize("bad", [
    dict(d=0), dict(d=60), dict(d=264), dict(hk=3), dict(hk=0), dict(pages=0), dict(page=0), dict(groups=4), dict(groups=3), dict(longest=65), dict(longest=-1), dict(longest=2 ** 30 + 1, width=2 ** 27), dict(width=3), dict(window=-1), dict(flags=4),
    dict(alpha=float("nan")), dict(b=MOST, s=2), dict(b=2 ** 20, s=2 ** 6, hq=64), dict(s=2 ** 22, hq=64),
    dict(q=NO), dict(kc=NO), dict(ks=NO), dict(vc=NO), dict(vs=NO), dict(table=NO), dict(out=NO),
    dict(q=op(I32, 256, 256, 64, 1)), dict(out=op(F16, 256, 256, 64, 1)), dict(out=op(BF16, 0, 256, 64, 1)), dict(table=op(F32, 4, 1)), dict(lengths=op(F32, 1)), dict(vc=op(I8, 2048, 128, 64, 1)),
    dict(kc=op(E2M1, 1024, 64, 32, 2)), dict(ks=op(F16, 32, 2, 1, 1)), dict(out=op(BF16, 256, 256, 64, 1, ptr=4097))])
def test_descriptors_of_attention_that_are_refused(bad):
    assert attend(**bad) == R.E_INVAL


def test_a_task_of_no_operator_is_refused_and_a_workspace_has_to_be_there():
    for kind in (0, 3, 2 ** 32 - 1):
        assert plan(kind, (1,), ()) == R.E_INVAL
    task = C._pack(2, 0, (1, 1, 4, 1, 64, 100, 16, 1, 64, 1024, 0),
                   (op(BF16, 256, 256, 64, 1), op(E2M1, 512, 32, 32, 1), op(F32, 16, 1, 1, 1), op(E2M1, 512, 32, 32, 1), op(F32, 16, 1, 1, 1), op(I32, 64, 1), NO, op(BF16, 256, 256, 64, 1)), 0.1)
    need = R.cache_workspace(task)
    assert need > 0
    for at, n in ((0, need), (4096, need - 1), (4100, need)):
        with pytest.raises(R.GpuosError) as e:
            R.launch_cache(task, at, n)
        assert e.value.status == R.E_NOMEM


# ---- tensors ---------------------------------------------------------------------------------------

@pytest.fixture
def launched(_launched, monkeypatch):  # noqa: F811
    calls = []

    def launch(function, task, places, tensors, written, device, workspace, stream):
        for i in written:
            torch.autograd.graph.increment_version(tensors[i]) if not tensors[i].is_inference() else None
        calls.append(struct.unpack_from("<I", task)[0])
        return 0
    make = B.like
    monkeypatch.setattr(B, "launch", launch)
    monkeypatch.setattr(B, "like", lambda x: make(x).zero_())
    return calls


def inputs(s=3, fmt=torch.uint8):
    n = 4 if fmt == torch.uint8 else 8
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(s, h, 8, generator=gen) for h in (4, 2, 2))
    caches = [torch.zeros(2, 4, 2, n, dtype=torch.uint8).view(fmt) if i % 2 == 0 else torch.ones(2, 4, 2, 1) for i in range(4)]
    return q, k, v, torch.arange(s, dtype=torch.int32), caches, torch.ones(9, 8)


PAGES = torch.tensor([[0, 1], [1, 0], [1, 1]], dtype=torch.int32)


@pytest.mark.parametrize("seen", (False, True))
def test_arguments_that_do_not_fit_are_refused(launched, seen):
    q, k, v, slots, caches, table = inputs()
    kc, ks, vc, vs = caches
    call = lambda **kw: M.cache_append_qkv(**{**dict(q=q, k=k, v=v, slots=slots, k_cache=kc, k_scales=ks, v_cache=vc, v_scales=vs, table=table, positions=slots), **kw})
    ask = lambda **kw: M.cache_attention(**{**dict(q=q, k_cache=kc, k_scales=ks, v_cache=vc, v_scales=vs, pages=PAGES, lengths=slots, longest=8), **kw})
    if seen:                                                 # (plans of the calls that are right)
        call(), ask()
    done = len(launched)
    for bad in (dict(q=q[:2]), dict(q=q.half()), dict(q=q[..., :4]), dict(k=k.int()), dict(v=v.half()), dict(v=v[:, :1]), dict(slots=slots.long()), dict(slots=slots[:2]), dict(positions=slots[:2]),
                dict(positions=slots.float()), dict(table=table.half()), dict(table=None), dict(table=table[0]), dict(k_cache=kc[..., :3]), dict(k_cache=kc[:, :, :1]), dict(v_cache=vc.view(torch.int8)),
                dict(k_scales=ks.half()), dict(v_scales=vs[:1]), dict(k_scales=ks.expand(2, 4, 2, 3), v_scales=vs.expand(2, 4, 2, 3)), dict(out=q.half()), dict(out=q[:2]), dict(q=None, out=q), dict(q=None, k=None),
                dict(q=3), dict(k_cache=kc.float()), dict(q=torch.view_as_complex(torch.randn(3, 4, 8, 2)).conj().imag)):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(q=q[:2]), dict(q=q.int()), dict(q=q[..., :4]), dict(q=q[:, :3]), dict(q=q[0]), dict(pages=PAGES.long()), dict(pages=PAGES[0]), dict(lengths=slots[:2]), dict(lengths=slots.long()), dict(longest=9),
                dict(longest=-1), dict(window=-1), dict(k_cache=kc[..., :3]), dict(v_cache=vc[:1]), dict(v_cache=vc.view(torch.int8)), dict(k_scales=ks.double()), dict(out=q.half()), dict(out=q[:1]),
                dict(k_scales=ks.expand(2, 4, 2, 2), v_scales=vs.expand(2, 4, 2, 2)), dict(q=None), dict(k_cache=None), dict(q=torch.view_as_complex(torch.randn(3, 4, 8, 2)).conj().imag)):
        with pytest.raises(ValueError):
            ask(**bad)
    assert len(launched) == done
    for bad in (dict(k=k[:, :, :7], q=None, v=v[:, :, :7], table=None, positions=None), dict(k_scales=ks.expand(2, 4, 2, 8), v_scales=vs.expand(2, 4, 2, 8))):
        with pytest.raises((ValueError, R.GpuosError)):
            call(**bad)
    assert len(launched) == done


def test_heads_of_attention_are_multiples_of_eight_up_to_256(launched):
    for d, ok in ((8, True), (12, False), (256, True), (264, False)):
        q, cache, scales = torch.zeros(1, 1, d), torch.zeros(1, 4, 1, d, dtype=torch.int8), torch.ones(1, 4, 1, 1)
        ask = lambda: M.cache_attention(q, cache, scales, cache, scales, PAGES[:1, :1], None, 4)
        if ok:
            assert ask().shape == q.shape
        else:
            with pytest.raises(ValueError):
                ask()


def test_what_a_gradient_would_be_cut_off_from_is_refused(launched):
    q, k, v, slots, caches, table = inputs()
    for name in ("q", "k", "v", "table", "k_scales", "v_scales"):
        for fresh in (False, True):
            q, k, v, slots, caches, table = inputs()
            kw = dict(q=q, k=k, v=v, slots=slots, k_cache=caches[0], k_scales=caches[1], v_cache=caches[2], v_scales=caches[3], table=table)
            if not fresh:
                M.cache_append_qkv(**kw)
            kw[name].requires_grad_()
            done = len(launched)
            with pytest.raises(ValueError, match="gradient"):
                M.cache_append_qkv(**kw)
            assert len(launched) == done
            with torch.no_grad():
                M.cache_append_qkv(**kw)
    q, k, v, slots, caches, table = inputs()
    q.requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        M.cache_attention(q, *caches, PAGES, None, 8)
    with torch.no_grad():
        assert not M.cache_attention(q, *caches, PAGES, None, 8).requires_grad


def test_what_is_written_counts_as_written(launched):
    q, k, v, slots, caches, table = inputs()
    scores = torch.randn(2, 4, 2, 1, requires_grad=True)
    product, before = scores * caches[1], [c._version for c in caches]
    out = torch.zeros_like(q)
    M.cache_append_qkv(q, k, v, slots, *caches, table, out=out)
    assert [c._version for c in caches] == [n + 1 for n in before] and out._version == 1 and q._version == 0
    with pytest.raises(RuntimeError, match="inplace"):
        product.sum().backward()
    M.cache_attention(q, *caches, PAGES, None, 8, out=out)
    assert out._version == 2 and caches[0]._version == before[0] + 1
    with torch.inference_mode():
        M.cache_append_qkv(*(t.clone() for t in (q, k, v)), slots, *(c.clone() for c in caches), table)
    assert launched == [1, 2, 1]


def test_traces_and_tangents_are_refused(launched):
    q, k, v, slots, caches, table = inputs()
    both = (lambda q: M.cache_append_qkv(q, k, v, slots, *caches, table), lambda q: M.cache_attention(q, *caches, PAGES, None, 8))
    for f in both:
        f(q)
        done = len(launched)
        for trace in (lambda: make_fx(f)(q), lambda: torch.jit.trace(f, (q,), check_trace=False)):
            with pytest.raises((ValueError, RuntimeError)):
                trace()
        with forward_ad.dual_level(), pytest.raises(ValueError, match="forward-mode"):
            f(forward_ad.make_dual(q, torch.ones_like(q)))
        assert len(launched) == done


def test_a_compiled_program_calls_them(launched):
    q, k, v, slots, caches, table = inputs()

    def f(q):
        return M.cache_attention(M.cache_append_qkv(q * 2, k, v, slots, *caches, table), *caches, PAGES, None, 8) * 0
    assert torch.equal(torch.compile(f, backend="eager")(q), torch.zeros_like(q)) and launched == [1, 2]


def test_tensors_without_memory_are_refused():
    with FakeTensorMode():
        fake = torch.empty(3, 4, 8)
    task = C._pack(2, 0, (1, 1, 1, 1, 8, 1, 1, 1, 1, 1, 0), ())
    with pytest.raises((ValueError, RuntimeError)):
        B.launch(R.cache_launch_address(), task, bytes([0]), (fake,), b"", 0, 0, 0)


def test_keys_tell_calls_apart():
    t = torch.zeros(4, 6)
    keys = [B.key(x) for x in ((t,), (t, None), (None, t), (t, t), (t.t(),), (t[:, ::2],), (t[:, :3],), (t.half(),), (t.view(6, 4),), (t.view(24),), (t.expand(1, 4, 6),), (t.int(),),
                               (t.to("meta"),), (torch.view_as_complex(torch.zeros(4, 6, 2)).conj().imag.as_strided((4, 6), (6, 1)),))]
    assert len(set(keys)) == len(keys) and B.key((t,)) == B.key((torch.ones(4, 6),)) == keys[0]
    r = torch.zeros(4, 6, requires_grad=True)
    assert B.key((r,))[0] == 1 and B.key((r,))[1:] == keys[0][1:]
    with torch.no_grad():
        assert B.key((r,)) == keys[0]
    for bad in ((3,), ("t",), (t.to_sparse(),)):
        with pytest.raises(ValueError):
            B.key(bad)
    with pytest.raises(TypeError):
        B.key([t])


# ---- definitions, kernels ----------------------------------------------------------------------------

def test_the_definition_of_codes_of_four_bits():
    """Against the borders between codes, ties and both zeros among them."""
    y = torch.cat((torch.arange(-800, 801).float() / 128, torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0, -0.0])))
    m = y.abs()
    code = (m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0) + 8 * torch.signbit(y).int()
    assert torch.equal(ref.encode(y).int(), code.int())
    x = torch.randn(5, 64) * 3
    codes, scales = ref.quantise(x, 2, torch.uint8)
    back = ref.values(codes[None, None], scales[None, None])[0, 0]
    assert bool(((back - x).abs() <= scales.double().repeat_interleave(32, -1) * 1.0001).all())      # half of the widest step, 2


def test_every_kernel_has_room_beside_the_default_worker():
    """128 registers of every SIMD for a workgroup of 256, 64 for one of 512.  (Attention's LDS is given with the launch, 65,536 bytes at most; the source
    asserts that.)"""
    mine = {n: k for n, k in kernels().items() if "gpuos_cache_" in n}
    assert len([n for n in mine if "attend" in n]) == 72 and len([n for n in mine if "append" in n]) == 6 and len([n for n in mine if "join" in n]) == 6
    (worker,) = [k for n, k in kernels().items() if "gpuos_worker_kernel" in n]
    for name, k in mine.items():
        waves = -(-k[".max_flat_workgroup_size"] // 256)
        registers = -(-k[".vgpr_count"] // 8) * 8
        assert waves * registers <= 512 - 3 * 128, (name, registers, waves)
        assert k[".group_segment_fixed_size"] <= 160 * 1024 - 3 * worker[".group_segment_fixed_size"], name
        assert 65536 <= 160 * 1024 - 3 * worker[".group_segment_fixed_size"]
