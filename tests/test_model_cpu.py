"""Host logic of the model operators, without a GPU: which descriptors are refused, how tasks are cut into chunks, what the
binding checks, and the definitions the GPU tests compare with against autograd in 64 bits."""
import numpy as np
import pytest
import torch

import model_reference as ref
from paper_2604_17861_amd import model as M
from paper_2604_17861_amd import runtime as R
from paper_2604_17861_amd import streams as S

F32, F16, BF16, I32, I8, E4M3 = range(6)
AT = 1 << 20                       # an address that is never read


def op(dtype, *stride, ptr=AT):
    return (ptr, *stride, *(0,) * (4 - len(stride)), dtype)


def plan(name, size, operands, flags=0, n=None):
    task = M._TASK.pack(S.MODEL_OP[name], len(operands) if n is None else n, 0, flags, *size, *(0,) * (8 - len(size)),
                        *(v for o in operands for v in o), *M._NONE * (8 - len(operands)), 1e-6, 0, 0, 0)
    try:
        return R.model_plan(task, S.MODEL_IMPL[name])
    except R.GpuosError as e:
        return e.status


def rope(b=2, s=3, h=4, d=64, r=64, places=100, **change):
    o = dict(x=op(BF16, s * h * d, h * d, d, 1), gamma=op(F32, 1), table=op(F32, r, 1), positions=op(I32, s, 1), out=op(BF16, s * h * d, h * d, d, 1))
    flags = change.pop("flags", 0)
    o.update(change)
    return plan("NORM_ROPE", (b, s, h, d, r, places), tuple(o.values()), flags)


def grad(b=2, s=3, h=4, d=64, r=64, places=100, parts=5, **change):
    rows = op(BF16, s * h * d, h * d, d, 1)
    o = dict(x=rows, gamma=op(F32, 1), table=op(F32, r, 1), positions=op(I32, s, 1), dx=rows, dout=rows, partial=op(F32, parts, 1))
    o.update(change)
    return plan("NORM_ROPE_GRAD", (b, s, h, d, r, places, parts), tuple(o.values()))


def store(b=1, s=9, h=2, d=64, pages=5, page=16, groups=1, **change):
    o = dict(x=op(BF16, s * h * d, h * d, d, 1), slots=op(I32, s, 1), cache=op(I8, page * h * d, h * d, d, 1), scales=op(F32, page * h * groups, h * groups, groups, 1))
    o.update(change)
    return plan("CACHE_STORE", (b, s, h, d, pages, page, groups), tuple(o.values()))


def load(b=2, l=30, h=2, d=64, pages=5, page=16, groups=1, width=2, **change):
    o = dict(cache=op(I8, page * h * d, h * d, d, 1), scales=op(F32, page * h * groups, h * groups, groups, 1), table=op(I32, width, 1), lengths=op(I32, 1),
             out=op(F16, l * h * d, h * d, d, 1))
    o.update(change)
    return plan("CACHE_LOAD", (b, l, h, d, pages, page, groups, width), tuple(o.values()))


def penalty(b=2, v=1000, n=50, **change):
    w = (v + 31) // 32
    o = dict(x=op(F32, v, 1), out=op(F32, v, 1), history=op(I32, n, 1), prompts=op(I32, 1), params=op(F32, 3, 1), bias=op(F32, 0, 1), allowed=op(I32, w, 1))
    o.update(change)
    return plan("LOGIT_PENALTY", (b, v, n), tuple(o.values()))


NO = op(0, ptr=0)
GOOD = [lambda: rope(), lambda: rope(flags=4), lambda: rope(r=0, table=NO, positions=NO), lambda: rope(gamma=NO), lambda: rope(positions=NO),
        lambda: rope(x=op(BF16, 0, 0, 0, 1)), lambda: grad(), lambda: grad(partial=NO), lambda: grad(dout=op(BF16, 0, 0, 0, 0)),
        lambda: plan("GAMMA_SUM", (64, 5), (op(F32, 5, 1), op(BF16, 1))), lambda: store(), lambda: store(groups=8), lambda: load(), lambda: load(lengths=NO),
        lambda: load(l=32), lambda: penalty(), lambda: penalty(bias=NO, allowed=NO), lambda: penalty(n=0, history=NO, prompts=NO, params=NO),
        lambda: penalty(prompts=NO), lambda: penalty(out=op(BF16, 2000, 2))]
BAD = {
    "odd R": lambda: rope(r=63), "R over D": lambda: rope(r=66), "D of nothing": lambda: rope(d=0, r=0), "D too long": lambda: rope(d=513, r=2),
    "negative size": lambda: rope(b=-1), "too many rows": lambda: rope(b=1 << 20, s=1 << 10, h=4), "sizes that overflow": lambda: plan("NORM_ROPE", (1 << 31, 1 << 31, 1 << 31, 64, 0, 0), (op(F32, 64, 64, 64, 1), NO, NO, NO, op(F32, 64, 64, 64, 1))),
    "products that overflow": lambda: plan("NORM_ROPE", ((1 << 31) - 1,) * 3 + (64, 0, 0), (op(F32, 64, 64, 64, 1), NO, NO, NO, op(F32, 64, 64, 64, 1))),
    "no x": lambda: rope(x=NO), "no out": lambda: rope(out=NO), "no table": lambda: rope(table=NO), "no row in the table": lambda: rope(places=0),
    "integer x": lambda: rope(x=op(I32, 768, 256, 64, 1)), "8-bit out": lambda: rope(out=op(I8, 768, 256, 64, 1)), "16-bit table": lambda: rope(table=op(F16, 64, 1)),
    "table with gaps": lambda: rope(table=op(F32, 128, 2)), "float positions": lambda: rope(positions=op(F32, 3, 1)), "unknown dtype": lambda: rope(x=op(6, 768, 256, 64, 1)),
    "negative stride": lambda: rope(x=op(BF16, 768, 256, -64, 1)), "stride of 2^32": lambda: rope(x=op(BF16, 1 << 32, 256, 64, 1)),
    "out over itself": lambda: rope(out=op(BF16, 0, 256, 64, 1)), "address between elements": lambda: rope(x=op(BF16, 768, 256, 64, 1, ptr=AT + 1)),
    "unknown flag": lambda: rope(flags=8), "KEEPDIM": lambda: rope(flags=2), "pairs of a cache": lambda: plan("GAMMA_SUM", (64, 5), (op(F32, 5, 1), op(BF16, 1)), 4),
    "too few operands": lambda: plan("NORM_ROPE", (2, 3, 4, 64, 0, 0), (op(F32, 1),) * 4),
    "no parts": lambda: grad(parts=0), "too many parts": lambda: grad(parts=1025), "rows of parts that overlap": lambda: grad(partial=op(F32, 4, 1)),
    "parts with gaps": lambda: grad(partial=op(F32, 10, 2)), "16-bit parts": lambda: grad(partial=op(F16, 5, 1)), "no dout": lambda: grad(dout=NO),
    "group of 3": lambda: store(d=96, groups=32), "group of 24": lambda: store(d=96, groups=4), "groups that do not divide": lambda: store(groups=7),
    "no groups": lambda: store(groups=0), "page of nothing": lambda: store(page=0), "slots past 2^31": lambda: store(pages=1 << 20, page=1 << 12),
    "float cache": lambda: store(cache=op(F16, 2048, 128, 64, 1)), "cache with gaps": lambda: store(cache=op(I8, 4096, 256, 128, 2)),
    "16-bit scales": lambda: store(scales=op(F16, 32, 2, 1, 1)), "cache over itself": lambda: store(cache=op(I8, 0, 128, 64, 1)),
    "float slots": lambda: store(slots=op(F32, 9, 1)), "no slots": lambda: store(slots=NO), "row of 513": lambda: store(d=513),
    "length over the table": lambda: load(l=33), "float lengths": lambda: load(lengths=op(F32, 1)), "no page table": lambda: load(table=NO),
    "out over itself, read back": lambda: load(out=op(F16, 30 * 128, 128, 0, 1)),
    "history without params": lambda: penalty(params=NO), "params without history": lambda: penalty(history=NO, prompts=NO, n=0),
    "a length without history": lambda: penalty(history=NO, prompts=NO, params=NO), "prompts without history": lambda: penalty(n=0, history=NO, params=NO),
    "float history": lambda: penalty(history=op(F32, 50, 1)), "integer bias": lambda: penalty(bias=op(I32, 0, 1)), "float bits": lambda: penalty(allowed=op(F32, 32, 1)),
    "logits over themselves": lambda: penalty(out=op(F32, 0, 1)), "16-bit params": lambda: penalty(params=op(F16, 3, 1)),
}


@pytest.mark.parametrize("case", range(len(GOOD)))
def test_descriptors_that_are_taken(case):
    assert isinstance(GOOD[case](), tuple)


@pytest.mark.parametrize("what", list(BAD))
def test_descriptors_that_are_refused(what):
    assert BAD[what]() == R.E_INVAL


def test_an_unknown_implementation_is_refused():
    task = M._TASK.pack(52, 2, 0, 0, *(1,) * 8, *M._NONE * 8, 0.0, 0, 0, 0)
    for impl in (0, 1, 19, 26, 64):
        with pytest.raises(R.GpuosError) as e:
            R.model_plan(task, impl)
        assert e.value.status == R.E_BADOP


def test_empty_sizes_are_empty_tasks():
    for plans in (rope(b=0), rope(s=0), rope(h=0), store(s=0), load(b=0), load(l=0), penalty(b=0), penalty(v=0),
                  plan("GAMMA_SUM", (0, 5), (op(F32, 5, 1), op(BF16, 1)))):
        assert all(p["vectors"] == 2 and p["chunks"] == 1 for p in plans)
    assert all(p["vectors"] == 0 and p["chunks"] == 5 for p in grad(b=0))      # its shares are written all the same


def test_rows_of_sums_are_shared_out_however_short():
    """A row takes a workgroup the same time from one share to a thousand."""
    for shares in (0, 1, 7, 640, 1024):
        ring, kernel = plan("GAMMA_SUM", (128, shares), (op(F32, shares, 1), op(BF16, 1)))
        assert ring["chunks"] == 32 and kernel["chunks"] == 128


def test_chunks_cover_every_row_once_and_stay_in_their_bounds():
    rng = np.random.default_rng(0)
    for _ in range(400):
        b, s, h = (int(2 ** rng.uniform(0, k)) for k in (6, 11, 5))
        d = int(rng.integers(1, 513))
        r = 2 * int(rng.integers(0, d // 2 + 1))
        kind = rng.integers(0, 4)
        if kind == 0:
            plans = rope(b, s, h, d, r, table=op(F32, r, 1) if r else NO, positions=op(I32, s, 1) if r else NO)
        elif kind == 1:
            plans = store(b, s, h, d)
        elif kind == 2:
            plans = load(b, s, h, d, width=s // 16 + 1)
        else:
            v = int(2 ** rng.uniform(0, 18))
            plans = penalty(b, v)
        for p, most in zip(plans, (1024, 65536)):
            assert p["item"] >= 1 and (kind != 3 or p["item"] <= 7168)         # (a segment's counts lie in LDS)
            items = b * -(-v // p["item"]) if kind == 3 else b * s * -(-h // p["item"])
            assert 1 <= p["chunks"] <= min(most, items) and p["items"] <= items <= p["chunks"] * p["items"]
    for parts in (1, 3, 1024):
        for p in grad(b=7, s=11, parts=parts):
            assert p["chunks"] == parts and p["items"] * parts * p["item"] >= 7 * 11 * 4


def test_rows_go_in_vectors_where_they_can():
    both = lambda plans: tuple(p["vectors"] for p in plans)
    none = dict(r=0, table=NO, positions=NO)
    for plans in (rope(), rope(flags=4), grad(), store(), load(), penalty(), rope(d=48, **none), store(d=64, groups=8)):
        assert both(plans) == (1, 1)
    # a kernel takes them from any address and to any end, the ring on eight bytes
    for plans in (rope(d=60, **none), rope(d=64, r=20), rope(d=66, r=66, flags=4), rope(x=op(BF16, 769, 257, 65, 1)), rope(x=op(BF16, 768, 256, 64, 1, ptr=AT + 2)),
                  store(d=60), load(d=100), store(cache=op(I8, 2049, 129, 65, 1)), penalty(v=1001)):
        assert both(plans) == (0, 1)
    for plans in (rope(d=65, r=64), rope(d=64, r=6), rope(d=67, r=4, flags=4), rope(d=6, **{**none, "flags": 4}), rope(out=op(F16, 768, 256, 64, 1)),
                  rope(x=op(BF16, 1536, 512, 128, 2)), store(d=7), load(out=op(F16, 7680, 256, 128, 2)), penalty(x=op(F32, 2000, 2)), penalty(bias=op(F32, 0, 2))):
        assert both(plans) == (0, 0)


def test_the_binding_checks_what_the_library_cannot_see():
    x = torch.zeros(2, 4, 64)
    with pytest.raises(ValueError, match="on a GPU"):
        M.norm_rope(x)
    for call in (lambda: M.penalize_logits(torch.zeros(2, 5)), lambda: M.cache_store(x, torch.zeros(2, dtype=torch.int32), x, x),
                 lambda: M.cache_load(x, x, x, None, 3)):
        with pytest.raises(ValueError):
            call()


def test_the_descriptor_has_the_layout_of_the_header():
    assert M._TASK.size == S.MODEL_TASK_BYTES == 8 + 64 + 8 * 48 + 16
    assert set(S.MODEL_IMPL.values()) == set(range(20, 26)) and not set(S.MODEL_OP.values()) & set(S.OP.values())


@pytest.mark.parametrize("pairs", (False, True))
@pytest.mark.parametrize("d,r", ((8, 8), (9, 4), (16, 0), (12, 10)))
def test_the_definition_of_the_gradients_is_that_of_the_function(d, r, pairs):
    gen = torch.Generator().manual_seed(0)
    x = torch.randn(2, 3, 2, d, generator=gen, dtype=torch.float64, requires_grad=True)
    g = torch.randn(d, generator=gen, dtype=torch.float64, requires_grad=True)
    angle = torch.rand(9, r // 2, generator=gen, dtype=torch.float64) * 9
    table = torch.cat((angle.cos(), angle.sin()), 1) if r else None
    p = torch.randint(0, 9, (2, 3), generator=gen) if r else None
    z, _ = ref.norm_rope(x, g, table, p, 1e-3, pairs)
    dz = torch.randn(z.shape, generator=gen, dtype=torch.float64)
    want = torch.autograd.grad(z, (x, g), dz)
    dx, _, dg, _ = ref.norm_rope_grad(dz, x.detach(), g.detach(), table, p, 1e-3, pairs)
    assert torch.allclose(dx, want[0], rtol=1e-12, atol=1e-12) and torch.allclose(dg, want[1], rtol=1e-12, atol=1e-12)


def test_tensors_of_one_call_are_on_one_device():
    class On:
        def __init__(self, device):
            self.device = device

        def get_device(self):
            return self.device

        def numel(self):
            return 1
    task = bytes(S.MODEL_TASK_BYTES)
    assert M._Plan([On(1), On(1)], [task] * 2, [(), ()]).device == 1
    with pytest.raises(ValueError):
        M._Plan([On(0), On(1)], [task] * 2, [(), ()])
