"""Model operators on the GPU, as kernels on a stream and as tasks of the ring, against their definitions
(tests/model_reference.py).

Tolerances.  The cache and the penalties are defined operation by operation in 32 bits: results are equal.  A norm and rotation is
computed in 32 bits and rounded once: half a step of the output's type, and F * 2^-24 of the size its terms have.  F counts
roundings on the longest way: the sum of squares has at most 8 terms in a lane and 6 steps over lanes, the mean, epsilon and the
square root 4 (rsqrtf is good to one step, two half steps), so the root is off by 14 / 2 + 2 < 10; three products and the
rotation's two roundings come on top: F = 16.  Backwards dx has the root three times (30), the second sum (8 + 6 + 2) and eight
products: F = 56.  The gradient of gamma adds what its sums take: rows of a lane, 256 groups of lanes, and the parts' sum."""
import numpy as np
import pytest
import torch

import model_reference as ref
from paper_2604_17861_amd import model as M
from paper_2604_17861_amd import runtime as R
from paper_2604_17861_amd import streams as S

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
CFG = dict(idle_exit_ms=20000, wait_timeout_ms=20000)
ROUTES = ("launch", "ring")
LEAST = {F32: 2.0 ** -149, F16: 2.0 ** -24, BF16: 2.0 ** -133}


_alive = []                        # what descriptors name (a descriptor does not keep it)


@pytest.fixture(autouse=True)
def _let_go():
    yield
    torch.cuda.synchronize()
    _alive.clear()


def up(t):
    """t on the GPU, until the test ends."""
    if t is None:
        return None
    _alive.append(t.cuda())
    return _alive[-1]


def run(route, *tasks):
    """The descriptors' tasks, finished."""
    torch.cuda.synchronize()
    if route == "launch":
        M.launch(*tasks)
        torch.cuda.synchronize()
        return
    with R.Runtime(0, **CFG) as rt:
        M.register(rt)
        rt.submit_model(b"".join(tasks))
        rt.wait()


def check(got, want, size, factor, what=""):
    """Within `factor` roundings of 32 bits of `size`, and one to the type of `got`."""
    half = torch.finfo(got.dtype).eps / 2
    g = got.double().cpu()
    bound = factor * ref.U * size
    bound = bound + half * (want.abs() + bound) + LEAST[got.dtype] / 2
    bad = ~((g - want).abs() <= bound)
    both = torch.isnan(g) & torch.isnan(want)
    bad &= ~both
    assert not bad.any(), "%s: %d of %d off, the first by %g of %g allowed" % (
        what, int(bad.sum()), bad.numel(), float((g - want).abs()[bad][0]), float(bound[bad][0]))


def same(got, want, what=""):
    """Equal, NaN to NaN."""
    g, w = got.cpu(), want
    if g.dtype in (torch.int8, torch.float8_e4m3fn):
        g, w = g.view(torch.int8), w.view(torch.int8)
        bad = g != w
    else:
        bad = ~((g == w) | (torch.isnan(g) & torch.isnan(w)))
    assert not bad.any(), "%s: %d of %d differ, the first: %s, not %s" % (what, int(bad.sum()), bad.numel(), g[bad][0], w[bad][0])


def normal(gen, *shape, dtype=F32, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=gen) * scale + shift).to(dtype)


def laid(t, layout):
    """The same values on the GPU, lying in memory another way, until the test ends."""
    t = _laid(t.cuda(), layout)
    _alive.append(t)
    return t


def _laid(t, layout):
    if layout == "plain":
        return t.clone()
    if layout == "heads":                                    # heads before tokens
        return t.transpose(-3, -2).contiguous().transpose(-3, -2)
    if layout == "wide":                                     # a part of wider rows, off the alignment of vectors
        w = torch.zeros(*t.shape[:-1], t.shape[-1] + 7, dtype=t.dtype, device="cuda")
        w[..., 3:3 + t.shape[-1]] = t
        return w[..., 3:3 + t.shape[-1]]
    if layout == "fused":                                    # some heads of more
        w = torch.zeros(*t.shape[:-2], t.shape[-2] + 3, t.shape[-1], dtype=t.dtype, device="cuda")
        w[..., 1:1 + t.shape[-2], :] = t
        return w[..., 1:1 + t.shape[-2], :]
    assert layout == "strided"                               # every second element
    w = torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype, device="cuda")
    w[..., ::2] = t
    return w[..., ::2]


def rope_inputs(shape, r, dtype, gamma, positions, seed=0):
    gen = torch.Generator().manual_seed(1000 + seed)
    x = normal(gen, *shape, dtype=dtype)
    g = normal(gen, shape[-1], dtype=gamma, scale=0.2, shift=1.0) if gamma is not None else None
    places = shape[-3] + 50
    angle = torch.rand(places, r // 2, generator=gen, dtype=torch.float64) * 100
    table = torch.cat((angle.cos(), angle.sin()), 1).float() if r else None
    p = None
    if positions and r:
        p = torch.randint(0, places, shape[:-2] if positions == "each" else (shape[1],), generator=gen, dtype=torch.int32)
    return gen, x, g, table, p


# shape, R, pairs, dtype, gamma's dtype, layout, positions
ROPE = [
    ((1, 1, 1), 0, False, F32, None, "plain", None),
    ((1, 1, 2), 2, False, BF16, F32, "plain", "each"),
    ((3, 2, 7), 4, True, F16, F16, "plain", "each"),
    ((1, 16, 128), 128, False, BF16, BF16, "plain", "each"),
    ((5, 3, 64), 64, True, F32, F32, "fused", "each"),
    ((67, 5, 80), 32, True, F16, F32, "plain", "each"),
    ((2, 33, 4, 80), 20, False, BF16, BF16, "heads", "each"),       # halves of ten: element by element
    ((2, 33, 4, 128), 128, False, BF16, BF16, "heads", "each"),
    ((3, 40, 2, 128), 64, False, F16, None, "fused", None),         # a part rotated, positions counted
    ((2, 9, 3, 96), 96, True, BF16, F32, "wide", "shared"),
    ((2, 9, 3, 96), 48, False, F32, F32, "wide", "shared"),
    ((4, 3, 64), 64, False, F32, F32, "strided", "each"),
    ((2, 5, 1, 130), 130, False, F16, F16, "plain", "each"),
    ((1, 21, 2, 256), 256, False, F32, F32, "plain", "each"),
    ((11, 2, 512), 512, True, BF16, BF16, "plain", "each"),
    ((3, 2, 511), 510, False, F32, F32, "plain", "each"),
    ((3, 2, 512), 10, True, F16, F32, "plain", "each"),
    ((1000, 12, 64), 64, False, F16, F16, "plain", "each"),         # more rows than one pass of all chunks
    ((130, 3, 24), 0, False, BF16, F32, "plain", None),
    # parts that are no whole number of windows
    ((37, 5, 66), 66, False, BF16, F32, "plain", "each"),
    ((37, 5, 66), 20, True, F16, F32, "fused", "each"),
    ((19, 6, 64), 20, False, F32, BF16, "plain", "each"),
    ((2, 19, 7, 100), 100, False, BF16, BF16, "heads", "each"),
    ((19, 3, 100), 100, True, F16, F16, "wide", "each"),
    ((19, 3, 90), 10, False, F16, F16, "plain", "each"),
    ((19, 4, 90), 82, False, F32, F32, "wide", "each"),
    ((33, 4, 12), 8, False, F32, F32, "plain", "each"),
    ((33, 4, 4), 0, False, BF16, F32, "plain", None),
    ((9, 9, 250), 250, True, BF16, F32, "plain", "each"),
    ((9, 2, 510), 508, False, BF16, F32, "plain", "each"),          # a rest of two: element by element
]


@pytest.mark.parametrize("route", ROUTES)
@pytest.mark.parametrize("case", range(len(ROPE)))
def test_norm_and_rotation(case, route):
    shape, r, pairs, dtype, gamma, layout, positions = ROPE[case]
    gen, x, g, table, p = rope_inputs(shape, r, dtype, gamma, positions, case)
    want, size = ref.norm_rope(x, g, table, p, 1e-6, pairs)
    xg = laid(x, layout)
    out = torch.full(shape, 7.0, dtype=dtype, device="cuda")
    run(route, M.norm_rope_task(xg, up(g), up(table), up(p), out, eps=1e-6, pairs=pairs))
    check(out, want, size, 16)
    assert torch.equal(xg.cpu(), x)
    # in place
    run(route, M.norm_rope_task(xg, up(g), up(table), up(p), xg, eps=1e-6, pairs=pairs))
    assert torch.equal(xg, out)


@pytest.mark.parametrize("route", ROUTES)
@pytest.mark.parametrize("case", range(len(ROPE)))
def test_gradients_of_norm_and_rotation(case, route):
    shape, r, pairs, dtype, gamma, layout, positions = ROPE[case]
    gen, x, g, table, p = rope_inputs(shape, r, dtype, gamma, positions, case)
    dz = normal(gen, *shape, dtype=dtype)
    dx_w, dx_size, dg_w, dg_size = ref.norm_rope_grad(dz, x, g, table, p, 1e-6, pairs)
    rows = x.numel() // shape[-1]
    for parts in {1, min(1024, rows), 1024 if case % 4 == 0 else 7}:
        dx = torch.zeros(shape, dtype=dtype, device="cuda")
        partial = torch.full((shape[-1], parts), 9.0, device="cuda") if g is not None else None
        tasks = [M.norm_rope_grad_task(laid(dz, layout), laid(x, "plain" if layout == "wide" else layout), up(g), up(table), up(p), dx, partial,
                                       eps=1e-6, pairs=pairs)]
        if g is not None:
            dg = torch.zeros(shape[-1], dtype=gamma, device="cuda")
            tasks.append(M.gamma_sum_task(partial, dg, deps=(1,)))
        run(route, *tasks)
        check(dx, dx_w, dx_size, 56, "dx, %d parts" % parts)
        if g is not None:
            check(dg, dg_w, dg_size, 56 + -(-rows // parts) + 256 + 8 + parts / 64, "dgamma, %d parts" % parts)


@pytest.mark.parametrize("pairs", (False, True))
@pytest.mark.parametrize("r", (0, 6, 12, 16))
def test_gradients_against_differences(r, pairs):
    """Central differences of the library's own forward pass in fp32: off by their own truncation and the forward's roundings."""
    gen, x, g, table, p = rope_inputs((5, 2, 16), r, F32, F32, "each", 77)
    dz = normal(gen, 5, 2, 16)
    x, g, table, p, dz = (up(t) for t in (x, g, table, p, dz))
    dx, dg = M.norm_rope_backward(dz, x, g, table, p, pairs=pairs)
    for which, grad in (("x", dx), ("g", dg)):
        way = normal(gen, *grad.shape).cuda()
        h = 2.0 ** -7
        if which == "x":
            up_, down = (M.norm_rope(x + s * h * way, g, table, p, pairs=pairs) for s in (1, -1))
        else:
            up_, down = (M.norm_rope(x, g + s * h * way, table, p, pairs=pairs) for s in (1, -1))
        slope = float(((up_ - down).double() * dz).sum()) / (2 * h)
        want = float((grad.double() * way).sum())
        # 160 products of sizes of up to about 30 each: truncation h^2 / 6 times a third derivative of the row's order (measured against
        # the sum of sizes), and roundings of 16 * 2^-24 / h
        size = float((grad.double() * way).abs().sum()) + float(dz.abs().sum())
        assert abs(slope - want) <= size * (h * h + 16 * ref.U / h)


@pytest.mark.parametrize("tokens,heads", ((3, 1), (64, 4), (300, 8)))
def test_gradients_of_queries_and_keys_together(tokens, heads):
    """Equal sizes, so that whatever is let go of between the two is what the second is given."""
    gen, q, g, table, p = rope_inputs((tokens, heads, 64), 64, BF16, F32, "each", tokens)
    k, dq, dk = (normal(gen, tokens, heads, 64, dtype=BF16) for _ in range(3))
    g2 = normal(gen, 64, shift=1.0)
    torch.cuda.empty_cache()
    got = M.norm_rope_qk_backward(*(t.cuda() for t in (dq, dk, q, k, g, g2, table, p)))
    torch.cuda.synchronize()
    for i, (dz, x, gamma) in enumerate(((dq, q, g), (dk, k, g2))):
        dx, s, dg, gs = ref.norm_rope_grad(dz, x, gamma, table, p, 1e-6, False)
        check(got[i], dx, s, 56, "dx %d" % i)
        check(got[2 + i], dg, gs, 56 + 16 + 256 + 8 + 4, "dgamma %d" % i)


def test_autograd_reaches_every_input_and_expanded_gradients():
    gen, q, gq, table, p = rope_inputs((2, 7, 4, 32), 32, F32, F32, "each", 5)
    k, gk = normal(gen, 2, 7, 2, 32), normal(gen, 32, shift=1.0)
    leaves = [t.cuda().requires_grad_() for t in (q, k, gq, gk)]
    zq, zk = M.norm_rope_qk(*leaves, table.cuda(), p.cuda())
    (zq.sum() + 2.0 * zk.sum()).backward()                   # (gradients that are one number with strides of 0)
    for x, g, leaf, gleaf, w in ((q, gq, leaves[0], leaves[2], 1.0), (k, gk, leaves[1], leaves[3], 2.0)):
        dx, s, dg, gs = ref.norm_rope_grad(torch.full(x.shape, w), x, g, table, p, 1e-6, False)
        check(leaf.grad, dx, s, 56)
        check(gleaf.grad, dg, gs, 400)
    only = gk.cuda().requires_grad_()                        # a gradient of gamma alone, of a tensor used once
    M.norm_rope(k.cuda(), only, table.cuda(), p.cuda()).square().sum().backward()
    assert only.grad is not None and torch.isfinite(only.grad).all()
    with pytest.raises(ValueError):
        M.norm_rope(leaves[0], out=torch.empty_like(leaves[0]))


@pytest.mark.parametrize("route", ROUTES)
def test_positions_outside_the_table_and_values_without_a_norm(route):
    gen, x, g, table, p = rope_inputs((6, 2, 64), 64, F32, F32, "each", 9)
    p[1], p[4] = -1, table.shape[0]
    x[0, 0, 5] = float("inf")
    x[2] = 0.0
    x[3, 1, 3] = float("nan")
    for dtype in (F32, F16):
        xd = x.to(dtype)
        out = torch.zeros(6, 2, 64, dtype=dtype, device="cuda")
        run(route, M.norm_rope_task(up(xd), up(g), up(table), up(p), out, eps=0.0 if dtype == F32 else 1e-6))
        o = out.float().cpu()
        assert torch.isnan(o[1]).all() and torch.isnan(o[4]).all() and torch.isnan(o[3, 1]).all()
        assert torch.isnan(o[0, 0, 5]) and torch.isfinite(o[0, 1]).all() and torch.isfinite(o[3, 0]).all() and torch.isfinite(o[5]).all()
        assert torch.isnan(o[2]).all() if dtype == F32 else (o[2] == 0).all()      # 0 * 1 / sqrt(0); with epsilon 0


@pytest.mark.parametrize("route", ROUTES)
@pytest.mark.parametrize("pairs", (False, True))
@pytest.mark.parametrize("d,r", ((64, 32), (66, 20), (65, 32)))
def test_an_infinity_reaches_its_own_pair_only(d, r, pairs, route):
    gen, x, g, table, p = rope_inputs((4, 2, d), r, F32, F32, "each", 3)
    for t, j in enumerate((0, r - 1, r, d - 1)):
        x[t, 0, j] = float("inf")
    want, _ = ref.norm_rope(x, g, table, p, 1e-6, pairs)
    out = torch.zeros(4, 2, d, device="cuda")
    run(route, M.norm_rope_task(up(x), up(g), up(table), up(p), out, pairs=pairs))
    assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want)) and (out.cpu()[:, 0].nan_to_num() == 0).all()
    # and backwards from dout: elements that are not rotated stay by themselves
    x = normal(gen, 4, 2, d)
    dz = normal(gen, 4, 2, d)
    dz[:, :, d - 1] = float("inf")
    dx = torch.zeros(4, 2, d, device="cuda")
    partial = torch.zeros(d, 3, device="cuda")
    run(route, M.norm_rope_grad_task(up(dz), up(x), up(g), up(table), up(p), dx, partial, pairs=pairs))
    dg = partial.sum(1).cpu()
    assert torch.isfinite(dg[:d - 1]).all() and not torch.isfinite(dg[d - 1])


def cache_of(pages, page, h, d, groups, fmt, layout):
    """A cache with something in it, on the CPU and on the GPU in some layout."""
    gen = torch.Generator().manual_seed(3)
    values = torch.randint(-100, 100, (pages, page, h, d), generator=gen, dtype=torch.int8)
    if fmt != torch.int8:
        values = (values.float() * 4).to(fmt)
    scales = torch.rand(pages, page, h, groups, generator=gen) * 0.1

    def up(t):
        w = t.view(torch.int8) if t.dtype == torch.float8_e4m3fn else t
        w = laid(w, "plain") if layout != "heads" else w.cuda().transpose(1, 2).contiguous().transpose(1, 2)
        if layout == "odd":                                  # slots a byte further apart
            n = torch.zeros(*t.shape[:2], t.shape[2] * t.shape[3] + 1, dtype=w.dtype, device="cuda")
            v = n.as_strided(t.shape, (n.stride(0), n.stride(1), t.shape[3], 1))
            v.copy_(w)
            w = v
        return w.view(t.dtype) if t.dtype == torch.float8_e4m3fn else w
    return values, scales, up(values), up(scales)


# tokens (or [B, S]), H, D, groups, format, page, dtype, layouts of rows and cache
CACHE = [
    ((1,), 1, 1, 1, torch.int8, 1, F32, "plain", "plain"),
    ((5,), 2, 7, 1, torch.float8_e4m3fn, 3, F16, "plain", "plain"),
    ((64,), 8, 128, 1, torch.float8_e4m3fn, 16, BF16, "plain", "plain"),
    ((100,), 4, 128, 4, torch.int8, 16, BF16, "fused", "heads"),
    ((33,), 3, 80, 1, torch.int8, 7, F16, "plain", "plain"),
    ((33,), 3, 80, 5, torch.float8_e4m3fn, 7, F32, "plain", "plain"),
    ((2, 19), 2, 64, 8, torch.int8, 16, F32, "heads", "heads"),
    ((3, 5), 2, 256, 2, torch.float8_e4m3fn, 32, F16, "wide", "odd"),
    ((9,), 2, 256, 1, torch.int8, 4, BF16, "strided", "plain"),
    ((9,), 2, 256, 2, torch.int8, 4, BF16, "strided", "odd"),
    ((9,), 2, 256, 32, torch.float8_e4m3fn, 4, F32, "strided", "odd"),
    ((7,), 1, 511, 1, torch.int8, 5, F32, "plain", "plain"),
    ((7,), 1, 512, 1, torch.float8_e4m3fn, 5, F16, "plain", "plain"),
    ((7,), 1, 512, 2, torch.int8, 5, F16, "wide", "odd"),
    ((1500,), 8, 64, 2, torch.int8, 64, F16, "plain", "plain"),
    ((50,), 5, 100, 1, torch.int8, 16, BF16, "plain", "plain"),
    ((50,), 6, 250, 1, torch.float8_e4m3fn, 16, F32, "wide", "odd"),
    ((50,), 7, 9, 1, torch.int8, 16, F16, "fused", "heads"),
    ((50,), 9, 8, 1, torch.float8_e4m3fn, 16, F16, "plain", "plain"),
]


@pytest.mark.parametrize("route", ROUTES)
@pytest.mark.parametrize("case", range(len(CACHE)))
def test_cache_written_and_read_back(case, route):
    lead, h, d, groups, fmt, page, dtype, layout, cache_layout = CACHE[case]
    gen = torch.Generator().manual_seed(case)
    tokens = int(np.prod(lead))
    pages = -(-tokens // page) + 2
    x = normal(gen, *lead, h, d, dtype=dtype, scale=3.0)
    flat = x.view(-1, h, d)
    flat[0] *= 1e-3
    flat[tokens // 2] = 0.0
    if tokens > 4:
        flat[1, 0, 0], flat[2, h - 1, d - 1] = float("nan"), -float("inf")
        flat[3] = 65504.0 if dtype == F16 else 3e38
    slots = torch.randperm(pages * page, generator=gen)[:tokens].to(torch.int32).reshape(lead)
    if tokens > 6:
        slots.view(-1)[4], slots.view(-1)[5], slots.view(-1)[6] = -1, pages * page, -2147483648
    values, scales, cache, sc = cache_of(pages, page, h, d, groups, fmt, cache_layout)
    want, want_s = ref.store(x, slots, values, scales)
    run(route, M.cache_store_task(laid(x, layout), up(slots), cache, sc))
    same(cache, want, "values")
    same(sc, want_s, "scales")
    # and back: sequences of several lengths, one with a page that there is not
    width = 4
    length = max(1, width * page - 1)
    table = torch.randint(0, pages, (5, width), generator=gen, dtype=torch.int32)
    table[3, 1], table[4, 0] = -1, pages
    lengths = torch.tensor([length, 0, max(1, length // 2), length + 5, length], dtype=torch.int32)
    for lens in (lengths, None):
        out = torch.full((5, length, h, d), 5.0, dtype=dtype, device="cuda")
        o = laid(out, layout)
        run(route, M.cache_load_task(cache, sc, up(table), None if lens is None else up(lens), o))
        same(o, ref.load(want, want_s, table, lens, length, dtype), "read back")


def test_rows_at_ties_and_borders_of_the_formats():
    """x * (qmax / m) on the halves between whole numbers, and every 8-bit float there is."""
    x = torch.zeros(2, 1, 256)
    x[0, 0] = torch.arange(256) / 2 - 63.5
    x[0, 0, 0], x[0, 0, 255] = 127.0, -127.0
    every = torch.arange(256, dtype=torch.uint8).view(torch.int8).view(torch.float8_e4m3fn).float()
    x[1, 0] = torch.where(torch.isnan(every), torch.zeros(()), every)
    slots = torch.tensor([1, 0], dtype=torch.int32)
    for fmt in (torch.int8, torch.float8_e4m3fn):
        for dtype in (F32, BF16, F16):
            values, scales, cache, sc = cache_of(1, 2, 1, 256, 1, fmt, "plain")
            want, want_s = ref.store(x.to(dtype), slots, values, scales)
            M.cache_store(x.to(dtype).cuda(), slots.cuda(), cache, sc)
            same(cache, want)
            same(sc, want_s)
            table = torch.zeros(1, 1, dtype=torch.int32)
            got = M.cache_load(cache, sc, table.cuda(), None, 2, dtype=dtype)
            same(got, ref.load(want, want_s, table, None, 2, dtype))


# B, V, N, dtype, prompts, bias, allowed, layout
PENALTY = [
    (1, 1, 1, F32, True, "one", True, "plain"),
    (1, 31, 5, F16, False, None, True, "plain"),
    (3, 33, 0, BF16, False, "each", True, "plain"),
    (2, 1000, 64, F32, True, None, False, "plain"),
    (4, 4096, 100, BF16, True, "one", True, "plain"),
    (5, 4097, 300, F16, True, "each", True, "plain"),
    (2, 32003, 5000, F32, True, "one", True, "plain"),
    (3, 8200, 9001, BF16, False, None, False, "plain"),
    (3, 5000, 700, F32, True, "each", True, "strided"),
    (3, 5001, 700, F16, True, "each", True, "wide"),
    (300, 777, 20, BF16, True, "one", False, "plain"),
    (2, 12289, None, F32, False, "one", True, "plain"),
]


@pytest.mark.parametrize("route", ROUTES)
@pytest.mark.parametrize("case", range(len(PENALTY)))
def test_penalties(case, route):
    b, v, n, dtype, prompts, bias_kind, masked, layout = PENALTY[case]
    gen = torch.Generator().manual_seed(case)
    x = normal(gen, b, v, dtype=dtype, scale=4.0)
    x[0, 0] = float("nan")
    x[b - 1, v - 1] = float("inf")
    x[b // 2, v // 2] = -float("inf")
    history = params = prompt = bias = allowed = None
    if n is not None:
        history = (v * torch.rand(b, n, generator=gen) ** 4).to(torch.int32)
        if n > 3:
            history[:, 1], history[0, 2], history[0, 3] = -1, v, 2147483647
            history[b - 1, n // 2:] = -2147483648
        params = torch.rand(b, 3, generator=gen) + torch.tensor([0.8, 0.0, -0.3])
        prompt = torch.randint(-1, n + 2, (b,), generator=gen, dtype=torch.int32) if prompts else None
    if bias_kind:
        bias = normal(gen, *((v,) if bias_kind == "one" else (b, v)), dtype=BF16 if bias_kind == "each" else F32)
        bias[..., v // 3] = -float("inf")
        bias[..., v // 4] = torch.finfo(bias.dtype).min
    if masked:
        allowed = torch.randint(-2 ** 31, 2 ** 31, (b, (v + 31) // 32), generator=gen).to(torch.int32)
        allowed[b - 1] = 0                                   # nothing is allowed
    want = ref.penalties(x, history, prompt, params, bias, allowed)
    xg = laid(x, layout)
    out = laid(torch.zeros(b, v, dtype=dtype), layout)
    args = [up(t) for t in (history, prompt, params, bias, allowed)]
    run(route, M.penalty_task(xg, out, *args))
    same(out, want)
    same(xg, x)
    run(route, M.penalty_task(xg, xg, *args))                # in place
    same(xg, want)
    if layout == "plain":                                    # into another type: element by element
        other = torch.zeros(b, v, dtype=F32 if dtype != F32 else F16, device="cuda")
        run(route, M.penalty_task(up(x), other, *args))
        same(other, ref.penalties(x.float(), history, prompt, params, bias, allowed).to(other.dtype))


def test_a_count_of_any_size_and_the_same_token_everywhere():
    x = torch.tensor([[1.0, -2.0, 3.0]])
    history = torch.full((1, 70001), 1, dtype=torch.int32)
    params = torch.tensor([[1.5, 0.25, 0.5]])
    prompt = torch.tensor([1000], dtype=torch.int32)
    got = M.penalize_logits(x.cuda(), history=history.cuda(), prompt_lengths=prompt.cuda(), params=params.cuda())
    same(got, ref.penalties(x, history, prompt, params))


def decode_step(device_kind="cuda"):
    """Inputs of a step: norm and rotation, cache, reading back, scores, penalties."""
    gen = torch.Generator().manual_seed(8)
    b, h, d, page, length = 3, 4, 64, 16, 40
    t = dict(q=normal(gen, b, 1, h, d, dtype=BF16), k=normal(gen, b, 1, h, d, dtype=BF16), v=normal(gen, b, 1, h, d, dtype=BF16),
             g=normal(gen, d, dtype=BF16, shift=1.0, scale=0.1), pages=torch.arange(9, dtype=torch.int32).reshape(3, 3))
    angle = torch.rand(64, d // 2, generator=gen) * 10
    t["table"] = torch.cat((angle.cos(), angle.sin()), 1)
    t["lengths"] = torch.tensor([40, 17, 1], dtype=torch.int32)
    t["positions"] = (t["lengths"] - 1)[:, None].contiguous()
    at = t["lengths"] - 1
    t["slots"] = (t["pages"][torch.arange(3), (at // page).long()] * page + at % page).to(torch.int32)[:, None].contiguous()
    t["history"] = torch.randint(0, 500, (b, 30), generator=gen, dtype=torch.int32)
    t["params"] = torch.tensor([[1.2, 0.3, 0.1]] * b)
    t["logits"] = normal(gen, b, 500, dtype=BF16)
    return t, page, length


def test_a_decode_step_by_tasks_that_wait_for_each_other():
    """norm and rotation -> cache -> read back, and penalties -> softmax, in one stream of tasks of both kinds."""
    t, page, length = decode_step()
    g = {k: v.cuda() for k, v in t.items()}
    values, scales, kc, ks = cache_of(9, page, 4, 64, 1, torch.int8, "plain")
    k2 = torch.empty_like(g["k"])
    back = torch.zeros(3, length, 4, 64, dtype=BF16, device="cuda")
    probs, pen = torch.zeros(3, 500, dtype=BF16, device="cuda"), torch.zeros(3, 500, dtype=BF16, device="cuda")
    soft, pool = S.new_tasks(1)
    S.set_head(soft, 0, S.OP["SOFTMAX_LAST"], (3, 500), 1)
    S.set_tensor(soft, pool, 0, 0, 0, pen.data_ptr(), (500, 1), S.BF16)
    S.set_tensor(soft, pool, 0, 3, 0, probs.data_ptr(), (500, 1), S.BF16)
    soft["dep"][0, 0] = 4
    torch.cuda.synchronize()
    with R.Runtime(0, **CFG) as rt:
        M.register(rt)
        rt.register_table(S.default_table())
        first = rt.submit_model(M.penalty_task(g["logits"], pen, g["history"], None, g["params"])
                                + M.norm_rope_task(g["k"], g["g"], g["table"], g["positions"], k2)
                                + M.cache_store_task(k2, g["slots"], kc, ks, deps=(1,))
                                + M.cache_load_task(kc, ks, g["pages"], g["lengths"], back, deps=(1,)), flush=False)
        second = rt.submit(soft)
        assert (first, second) == (0, 4)
        rt.wait()
        assert (rt.completions(0, 5)["status"] == 0).all()
    z, size = ref.norm_rope(t["k"], t["g"], t["table"], t["positions"], 1e-6, False)
    check(k2, z, size, 16)
    want, want_s = ref.store(k2.cpu(), t["slots"], values, scales)
    same(kc, want)
    same(back, ref.load(want, want_s, t["pages"], t["lengths"], length, BF16))
    p = ref.penalties(t["logits"], t["history"], None, t["params"])
    same(pen, p)
    check(probs, torch.softmax(p.double(), -1), torch.softmax(p.double(), -1), 64)


def test_kernels_and_the_dispatch_filter_wait_for_each_other():
    """Redirected operations feed an operator, its result feeds redirected operations, over and over."""
    from paper_2604_17861_amd.dispatch import GpuosMode
    gen = torch.Generator().manual_seed(12)
    a, b = normal(gen, 40, 4, 64).cuda(), normal(gen, 40, 4, 64).cuda()
    g = normal(gen, 64, shift=1.0).cuda()
    want = a
    for _ in range(6):
        want = torch.relu(M.norm_rope(torch.relu(want + b) * 0.5, g) + b)
    torch.cuda.synchronize()
    mode = GpuosMode(idle_exit_ms=50)
    try:
        for _ in range(3):
            with mode:
                x = a
                for _ in range(6):
                    x = torch.relu(M.norm_rope(torch.relu(x + b) * 0.5, g) + b)
            assert torch.equal(x.cpu(), want.cpu())
        assert mode.stats["redirected"] >= 3 * 6 * 5 and not R.active_filters
    finally:
        mode.close()


def test_only_the_filter_of_the_calling_thread_is_waited_for(monkeypatch):
    """A filter belongs to its thread: its tables are not to be walked from another.  A backward pass runs on a thread of autograd's with the
    modes of the one that called it."""
    import threading
    from paper_2604_17861_amd.dispatch import GpuosMode
    x = torch.randn(40, 4, 64, device="cuda")
    leaf = x.clone().requires_grad_()
    torch.cuda.synchronize()
    mode = GpuosMode(idle_exit_ms=50)
    calls = []
    settle = mode.settle
    monkeypatch.setattr(mode, "settle", lambda ts: (calls.append(threading.get_ident()), settle(ts)))
    try:
        with mode:
            other = threading.Thread(target=lambda: M.norm_rope(x))
            other.start()
            other.join()
            assert not calls
            y = M.norm_rope(leaf)
            assert len(calls) == 1
            y.backward(torch.ones_like(y))
            assert len(calls) == 2
    finally:
        mode.close()
    torch.cuda.synchronize()
    one = x.clone().requires_grad_()
    M.norm_rope(one).backward(torch.ones_like(x))
    assert torch.equal(leaf.grad.cpu(), one.grad.cpu())


def test_a_number_in_a_tensor_is_read_at_every_call():
    x, eps = torch.randn(5, 2, 8, device="cuda"), torch.tensor(1e-6)
    first = M.norm_rope(x, eps=eps)
    assert torch.equal(first, M.norm_rope(x, eps=eps.item()))
    eps.fill_(1.0)
    second = M.norm_rope(x, eps=eps)
    assert torch.equal(second, M.norm_rope(x, eps=1.0)) and not torch.equal(first, second)


def test_outputs_that_autograd_has_saved_or_watches():
    x, w = torch.randn(3, 2, 8, device="cuda"), torch.randn(3, 2, 8, device="cuda", requires_grad=True)
    logits, wl = torch.randn(3, 20, device="cuda"), torch.randn(3, 20, device="cuda", requires_grad=True)
    _, scales, cache, ks = cache_of(2, 4, 2, 8, 1, torch.int8, "heads")
    pages, rows, wr = torch.tensor([[1]], dtype=torch.int32, device="cuda"), torch.randn(1, 3, 2, 8, device="cuda"), torch.randn(1, 3, 2, 8, device="cuda", requires_grad=True)
    calls = [(w, x.clone(), lambda o: M.norm_rope(x, out=o)), (wl, logits.clone(), lambda o: M.penalize_logits(logits, out=o)),
             (wr, rows, lambda o: M.cache_load(cache, ks, pages, None, 3, out=o)),
             (w, x.clone(), lambda o: M.norm_rope_qk(x, x, out=(o, None)))]
    for leaf, out, call in calls:
        product = leaf * out                                 # keeps `out` for the gradient
        call(out)
        with pytest.raises(RuntimeError, match="inplace"):
            product.sum().backward()
        with pytest.raises(ValueError):
            call(leaf)
        with torch.no_grad():
            call(leaf)
        with torch.inference_mode():
            call(torch.empty_like(out))


def test_every_operand_with_strides_of_its_own():
    gen = torch.Generator().manual_seed(13)
    every = lambda t: up(torch.stack((t, t), -1).flatten(-2))[..., ::2]      # every second element of twice as many
    b, s, h, d = 2, 5, 3, 32
    x1 = normal(gen, 1, s, 1, d)
    x = up(x1).expand(b, s, h, d)                            # one row for every sequence and head
    g, angle = normal(gen, d, shift=1.0), torch.rand(20, d // 2, generator=gen)
    table = torch.cat((angle.cos(), angle.sin()), 1)
    p = torch.randint(0, 20, (b, s), generator=gen, dtype=torch.int32)
    dz1 = normal(gen, b, s, h, 1)
    wide = torch.zeros(20, d + 4, device="cuda")
    wide[:, :d] = table.cuda()
    full, dzf = x1.expand(b, s, h, d), dz1.expand(b, s, h, d)
    got = M.norm_rope(x, every(g), wide[:, :d], every(p))
    z, size = ref.norm_rope(full, g, table, p, 1e-6, False)
    check(got, z, size, 16)
    dx, dg = M.norm_rope_backward(up(dz1).expand(b, s, h, d), x, every(g), wide[:, :d], every(p))
    w = ref.norm_rope_grad(dzf, full, g, table, p, 1e-6, False)
    check(dx, w[0], w[1], 56)
    check(dg, w[2], w[3], 56 + 256 + 30)
    shared = torch.arange(s, dtype=torch.int32)              # the same positions for every sequence, and none given
    for q in (every(shared), None):
        z, size = ref.norm_rope(full, g, table, shared, 1e-6, False)
        check(M.norm_rope(x, every(g), wide[:, :d], q), z, size, 16)
    # the cache: slots, scales and lengths apart; pages of a table with gaps
    values, scales, kc, ks = cache_of(4, 4, h, d, 2, torch.int8, "heads")
    slots = torch.randperm(16, generator=gen)[:b * s].to(torch.int32).reshape(b, s)
    M.cache_store(x, every(slots), kc, every(scales)[:])
    want, _ = ref.store(full, slots, values, scales)
    same(kc, want)
    sc = every(scales)
    pages = torch.tensor([[2, 0], [3, 1]], dtype=torch.int32)
    lens = torch.tensor([7, 4], dtype=torch.int32)
    same(M.cache_load(kc, sc, every(pages), every(lens), 8, dtype=F16), ref.load(want, scales, pages, lens, 8, F16))
    logits, hist = normal(gen, 2, 90), torch.randint(0, 90, (2, 40), generator=gen, dtype=torch.int32)
    params, prompts, bias = torch.rand(2, 3, generator=gen) + 0.5, torch.tensor([3, 9], dtype=torch.int32), normal(gen, 2, 90, dtype=F16)
    bits = torch.randint(-2 ** 31, 2 ** 31, (2, 3), generator=gen).to(torch.int32)
    got = M.penalize_logits(every(logits), history=every(hist), prompt_lengths=every(prompts), params=every(params), bias=every(bias), allowed=every(bits))
    same(got, ref.penalties(logits, hist, prompts, params, bias, bits))
    same(M.penalize_logits(up(logits), bias=up(bias[0]), allowed=up(bits[1])), ref.penalties(logits, bias=bias[0], allowed=bits[1]))


def test_what_has_no_gradient_is_refused():
    x = torch.randn(2, 10, device="cuda", requires_grad=True)
    with pytest.raises(ValueError):
        M.penalize_logits(x)
    with torch.no_grad():
        assert torch.equal(M.penalize_logits(x), x)
    t = torch.randn(4, 8, device="cuda", requires_grad=True)
    with pytest.raises(ValueError):
        M.norm_rope(torch.randn(3, 2, 8, device="cuda"), None, t)


def test_many_tasks_of_several_operators_in_one_call():
    """More tasks than a launch holds, operators taking turns, some with nothing to do, dependencies and fences."""
    gen = torch.Generator().manual_seed(1)
    xs = [normal(gen, 3 + i, 2, 64, dtype=BF16) for i in range(21)]
    outs = [torch.zeros(x.shape, dtype=BF16, device="cuda") for x in xs]
    logits = [normal(gen, 2, 100 + i) for i in range(5)]
    pen = [torch.zeros(2, 100 + i, device="cuda") for i in range(5)]
    bias = normal(gen, 200).cuda()
    xg, lg = [x.cuda() for x in xs], [x.cuda() for x in logits]
    tasks = []
    for i in range(21):
        tasks.append(M.norm_rope_task(xg[i], None, None, None, outs[i], deps=(min(i, 3),) if i % 7 == 5 else (), fence=i % 5 == 4))
        if i % 4 == 3:
            j = i // 4
            tasks.append(M.penalty_task(lg[j], pen[j], bias=bias[:100 + j]))
    M.launch(*tasks)
    torch.cuda.synchronize()
    for x, o in zip(xs, outs):
        z, size = ref.norm_rope(x, None, None, None, 1e-6, False)
        check(o, z, size, 16)
    for i in range(5):
        same(pen[i], ref.penalties(logits[i], bias=bias[:100 + i].cpu()))


def test_a_chain_in_one_launch_call_runs_in_order():
    gen = torch.Generator().manual_seed(2)
    x = normal(gen, 40, 4, 96, scale=5.0)
    bufs = [x.cuda()] + [torch.zeros(40, 4, 96, device="cuda") for _ in range(12)]
    tasks = [M.norm_rope_task(bufs[i], None, None, None, bufs[i + 1], eps=0.5, deps=(1,) if i else (), fence=False) for i in range(12)]
    M.launch(*tasks)
    torch.cuda.synchronize()
    for i in range(12):
        z, size = ref.norm_rope(bufs[i].cpu(), None, None, None, 0.5, False)
        check(bufs[i + 1], z, size, 16, "link %d" % i)


def test_empty_tensors_do_nothing():
    e = torch.empty(0, 4, 64, device="cuda")
    g = torch.ones(64, device="cuda", requires_grad=True)
    assert M.norm_rope(e, g.detach()).shape == (0, 4, 64)
    M.norm_rope(e, g).sum().backward()
    assert (g.grad == 0).all()
    cache, sc = torch.zeros(2, 4, 4, 64, dtype=torch.int8, device="cuda"), torch.zeros(2, 4, 4, 1, device="cuda")
    M.cache_store(e, torch.empty(0, dtype=torch.int32, device="cuda"), cache, sc)
    assert M.cache_load(cache, sc, torch.zeros(0, 2, dtype=torch.int32, device="cuda"), None, 3).shape == (0, 3, 4, 64)
    assert M.penalize_logits(torch.empty(0, 10, device="cuda")).shape == (0, 10)
    x = torch.randn(2, 10, device="cuda")
    empty = torch.empty(2, 0, dtype=torch.int32, device="cuda")
    assert torch.equal(M.penalize_logits(x, history=empty, params=torch.ones(2, 3, device="cuda")), x)
    # the shares of no rows at all are zeros
    partial = torch.full((64, 5), 3.0, device="cuda")
    dx = torch.empty(1, 4, 64, device="cuda")
    run("ring", M._pack("NORM_ROPE_GRAD", 0, (1, 0, 4, 64, 0, 0, 5), (M._rows(dx)[1], M._NONE, M._NONE, M._NONE, M._rows(dx)[1], M._rows(dx)[1],
                                                                      M._operand(partial)), 1e-6))
    assert (partial == 0).all()


def test_the_ring_binds_kills_and_brings_back():
    x = torch.randn(8, 2, 64, device="cuda")
    out = torch.zeros_like(x)
    task = M.norm_rope_task(x, None, None, None, out)
    torch.cuda.synchronize()
    with R.Runtime(0, **CFG) as rt:
        assert rt.submit_model(task, check=False)[0] == R.E_BADOP          # not bound
        M.register(rt)
        rt.register_op(40, S.IMPL["RELU"])
        rt.register_op(41, S.IMPL["FAIL"])
        op = S.MODEL_OP["NORM_ROPE"]
        for other in (S.IMPL["RELU"], S.MODEL_IMPL["NORM_ROPE_GRAD"], S.MODEL_IMPL["CACHE_STORE"], S.MODEL_IMPL["CACHE_LOAD"]):
            with pytest.raises(R.GpuosError):
                rt.swap_op(op, other)
        with pytest.raises(R.GpuosError):
            rt.swap_op(40, S.MODEL_IMPL["NORM_ROPE"])
        t0 = rt.submit_model(task)
        rt.wait(t0)
        rt.kill_op(op)
        t1 = rt.submit_model(task)
        assert rt.wait(t1, check=False) == R.E_BADOP
        for other in (S.IMPL["RELU"], S.MODEL_IMPL["CACHE_STORE"]):        # not by way of the stub either
            with pytest.raises(R.GpuosError):
                rt.swap_op(op, other)
        rt.swap_op(op, S.MODEL_IMPL["NORM_ROPE"])
        rt.wait(rt.submit_model(task * 3))
        rt.swap_op(41, S.MODEL_IMPL["NORM_ROPE"])                          # a stub takes a first kind
        with pytest.raises(R.GpuosError):
            rt.swap_op(41, S.IMPL["RELU"])
        # a descriptor of one kind under an operator of the other
        plain, _ = S.new_tasks(1)
        S.set_head(plain, 0, op, (4,), 1)
        assert rt.submit(plain, check=False)[0] != R.OK
        assert rt.submit_model(bytes([40]) + task[1:], check=False)[0] != R.OK
        rt.wait(check=False)
    z, size = ref.norm_rope(x.cpu(), None, None, None, 1e-6, False)
    check(out, z, size, 16)


def test_a_killed_operator_is_not_launched():
    x = torch.zeros(8, 2, 64, device="cuda")
    task = M.norm_rope_task(x, None, None, None, x)
    with pytest.raises(R.GpuosError):
        R.launch_model(task, table={S.MODEL_OP["NORM_ROPE"]: S.IMPL["FAIL"]})
    with pytest.raises(R.GpuosError):
        R.launch_model(task, table={})


@pytest.mark.parametrize("route", ROUTES)
def test_offsets_past_32_bits(route):
    """A cache of 4.6 GB and rows of tensors that far apart: the last pages, and rows on both sides of 2^32."""
    pages, page, h, d = 70000, 64, 8, 128
    cache = torch.empty(pages, page, h, d, dtype=torch.int8, device="cuda")
    scales = torch.empty(pages, page, h, 1, device="cuda")
    gen = torch.Generator().manual_seed(0)
    n = 2 ** 32 // (page * h * d)
    at = torch.tensor([0, n * page - 1, n * page, (pages - 1) * page, pages * page - 1], dtype=torch.int32)
    x = normal(gen, 5, h, d, dtype=BF16)
    run(route, M.cache_store_task(up(x), up(at), cache, scales))
    table = (at // page)[:, None].contiguous()
    out = torch.zeros(5, page, h, d, dtype=BF16, device="cuda")
    # only the stored rows have values: read each through its own page
    run(route, M.cache_load_task(cache, scales, up(table), None, out))
    q, s = ref.quantise(x, 1, torch.int8)
    want = (q.float() * s).to(BF16)
    for i in range(5):
        same(out[i, int(at[i]) % page], want[i])
    del cache, scales, out
    far = torch.empty(2 ** 32 + 4096, dtype=BF16, device="cuda")
    rows = far.as_strided((2, 2, 64), (2 ** 32 - 64, 64, 1))
    y = normal(gen, 2, 2, 64, dtype=BF16)
    rows.copy_(y.cuda())
    run(route, M.norm_rope_task(rows, None, None, None, rows))
    z, size = ref.norm_rope(y, None, None, None, 1e-6, False)
    check(rows, z, size, 16)
