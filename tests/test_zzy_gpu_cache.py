"""Cache operators on the GPU against their definitions (tests/cache_reference.py): what is appended is equal, attention within the bound
that is derived there."""
import pytest
import torch

import cache_reference as ref
from paper_2604_17861_amd import model as M
from test_gpu_model import BF16, F16, F32, _let_go, laid, normal, same, up  # noqa: F401

pytestmark = pytest.mark.gpu
E2M1, I8, E4M3 = torch.uint8, torch.int8, torch.float8_e4m3fn
WIDE = {E2M1: 2, I8: 1, E4M3: 1}                             # elements of a byte


def caches_of(pages, page, h, d, groups, fmt, layout="plain", gen=None):
    """keys' codes and scales, values' codes and scales; with `gen` full of what a program may have put there"""
    out = []
    for _ in range(2):
        for n, dtype in ((d // WIDE[fmt], fmt), (groups, F32)):
            shape = (pages, page, h, n) if layout != "heads" else (pages, h, page, n)
            t = torch.zeros(shape, dtype=torch.uint8 if dtype == fmt else F32)
            if gen is not None:
                if dtype == F32:
                    t = torch.rand(shape, generator=gen) * 0.02 * {E2M1: 25.0, I8: 1.0, E4M3: 0.7}[fmt]
                else:
                    t = torch.randint(0, 256, shape, generator=gen, dtype=torch.uint8)
                    if fmt == E4M3:
                        t = torch.where((t & 0x7f) == 0x7f, torch.zeros_like(t), t)
            t = t.view(fmt) if dtype == fmt else t
            out.append(t if layout != "heads" else t.transpose(1, 2))
    return out


def on_gpu(t):
    """The same strides on the GPU."""
    return up(t) if t.is_contiguous() else up(t.transpose(1, 2).contiguous()).transpose(1, 2)


# ---- appending ------------------------------------------------------------------------------------

APPEND = [
    # b, s, hq, hk, d, r, pairs, groups, page, layout, cache, positions
    (None, 1, 16, 8, 128, 128, False, 1, 16, "fused", "plain", "each"),
    (None, 65, 8, 2, 128, 128, False, 4, 16, "plain", "plain", "each"),
    (3, 7, 3, 5, 64, 64, True, 2, 7, "heads", "heads", "each"),
    (2, 5, 2, 1, 80, 32, False, 10, 1, "wide", "plain", "shared"),
    (2, 5, 2, 1, 80, 24, False, 1, 3, "plain", "heads", None),       # halves of 12: element by element
    (2, 9, 0, 3, 96, 96, True, 1, 16, "strided", "plain", "each"),
    (2, 9, 1, 3, 96, 0, False, 3, 16, "plain", "plain", None),
    (1, 33, 4, 4, 18, 10, True, 1, 5, "plain", "plain", "each"),     # nine bytes a row
    (1, 33, 4, 4, 2, 2, False, 1, 5, "plain", "plain", "each"),
    (2, 17, 7, 3, 256, 128, False, 8, 32, "fused", "plain", "each"),
    (1, 3, 1, 1, 512, 512, False, 64, 4, "plain", "plain", "each"),
    (1, 9, 3, 3, 200, 16, False, 25, 4, "plain", "plain", "each"),
]


@pytest.mark.parametrize("fmt", (E2M1, I8, E4M3))
@pytest.mark.parametrize("dtype", (F32, F16, BF16))
@pytest.mark.parametrize("case", APPEND)
def test_append(case, dtype, fmt):
    b, s, hq, hk, d, r, pairs, groups, page, layout, cl, pos = case
    gen = torch.Generator().manual_seed(sum(map(int, (s, hq, hk, d, r, groups))))
    lead = (s,) if b is None else (b, s)
    n = s * (b or 1)
    q = normal(gen, *lead, hq, d, dtype=dtype) if hq else None
    k, v = normal(gen, *lead, hk, d, dtype=dtype, scale=30.0), normal(gen, *lead, hk, d, dtype=dtype)
    k.flatten(0, -2)[0], v.flatten(0, -2)[-1] = 0.0, -0.0
    if n > 3:
        v.flatten(0, -2)[2, d // 2], k.flatten(0, -2)[3, 0] = float("inf"), float("nan")
    table = None
    if r:
        angle = torch.rand(50, r // 2, generator=gen, dtype=torch.float64) * 100
        table = torch.cat((angle.cos(), angle.sin()), 1).float()
    shape = {"each": lead, "shared": (s,)}.get(pos)
    positions = torch.randint(0, 50, shape, generator=gen, dtype=torch.int32) if shape and r else None
    if positions is not None and n > 8:
        positions.flatten()[1], positions.flatten()[-1] = 50, -1          # not in the table
    pages = n // page + 3
    slots = torch.randperm(pages * page, generator=gen)[:n].to(torch.int32).reshape(lead)
    if n > 4:
        slots.flatten()[4], slots.flatten()[0] = -1, pages * page          # nowhere
    caches = caches_of(pages, page, hk, d, groups, fmt, cl, gen)
    want_q, want = ref.append(q, k, v, slots, caches, table, positions, pairs)
    mine = [on_gpu(c) for c in caches]
    args = [None if t is None else laid(t, layout) for t in (q, k, v)]
    got = M.cache_append_qkv(*args, up(slots), *mine, up(table), up(positions), pairs=pairs)
    assert (got is None) == (q is None)
    if q is not None:
        same(got, want_q, "q")
    for g, w, name in zip(mine, want, ("keys", "scales of keys", "values", "scales of values")):
        same(g, w, name)


def test_append_writes_into_out_and_in_place():
    gen = torch.Generator().manual_seed(5)
    qkv = normal(gen, 40, 12, 64, dtype=BF16)
    table, positions, slots = torch.rand(60, 64, generator=gen), torch.arange(10, 50, dtype=torch.int32), torch.arange(40, dtype=torch.int32)
    caches = caches_of(5, 8, 2, 64, 2, E2M1)
    want_q, want = ref.append(qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], slots, caches, table, positions, False)
    x, mine = up(qkv), [up(c) for c in caches]
    q, version = x[:, :8], [c._version for c in mine]
    out = torch.empty_like(q)
    with pytest.raises(ValueError):
        M.cache_append_qkv(q, x[:, 8:10], x[:, 10:], up(slots), *mine, up(table), up(positions), out=out.float())
    assert M.cache_append_qkv(q, x[:, 8:10], x[:, 10:], up(slots), *mine, up(table), up(positions), out=out) is out
    same(out, want_q)
    assert all(c._version == v + 1 for c, v in zip(mine, version)) and out._version == 1
    for g, w in zip(mine, want):
        same(g, w)
        g.zero_()
    assert M.cache_append_qkv(q, x[:, 8:10], x[:, 10:], up(slots), *mine, up(table), up(positions), out=q) is q      # in place
    same(q, want_q)
    for g, w in zip(mine, want):
        same(g, w)


def test_append_of_nothing_and_of_more_rows_than_a_launch_has_workgroups():
    table = up(torch.rand(10, 128))
    mine = [up(c) for c in caches_of(2, 4, 3, 128, 1, I8)]
    out = M.cache_append_qkv(*(up(torch.zeros(0, 3, 128, dtype=F16)) for _ in range(3)), up(torch.zeros(0, dtype=torch.int32)), *mine, table)
    assert out.shape == (0, 3, 128)
    # 65,536 workgroups of 256 heads of one element pair: some make two passes
    gen = torch.Generator().manual_seed(8)
    n = 9000
    q = normal(gen, n, 4000, 2, dtype=F16)
    slots = torch.arange(n, dtype=torch.int32)
    caches = caches_of(n, 1, 1, 2, 1, E2M1)
    k = normal(gen, n, 1, 2, dtype=F16)
    angle = torch.rand(n, 1, generator=gen, dtype=torch.float64)
    t = torch.cat((angle.cos(), angle.sin()), 1).float()
    mine = [up(c) for c in caches]
    got = M.cache_append_qkv(up(q), up(k), up(k), up(slots), *mine, up(t))
    same(got, ref.rotate(q, t, None, False).to(F16))


# ---- attention ------------------------------------------------------------------------------------

ATTEND = [
    # b, s, hq, hk, d, groups, page, longest, lengths, window, cache
    (1, 1, 16, 8, 128, 1, 16, 301, None, 0, "plain"),
    (4, 1, 8, 8, 128, 4, 16, 130, (130, 1, 64, 65), 0, "plain"),
    (3, 1, 32, 4, 64, 1, 7, 200, (200, 0, 63), 0, "heads"),
    (2, 3, 6, 3, 80, 1, 5, 150, (150, 2), 0, "plain"),
    (2, 5, 4, 1, 96, 3, 32, 97, (97, 40), 33, "heads"),
    (1, 40, 8, 2, 128, 1, 64, 300, (290,), 0, "plain"),
    (1, 40, 4, 2, 256, 8, 64, 129, None, 17, "plain"),
    (2, 1, 5, 1, 256, 1, 1, 100, (77, 100), 0, "plain"),
    (2, 2, 17, 1, 192, 3, 16, 90, (90, 64), 1, "heads"),
    (2, 1, 2, 2, 8, 1, 4, 20, (20, 3), 0, "plain"),
    (3, 1, 12, 4, 128, 1, 16, 1500, (1500, 600, 9), 0, "plain"),      # pieces, a head for each wavefront
    (1, 2, 24, 6, 64, 2, 16, 1100, None, 0, "plain"),
    (2, 1, 4, 1, 128, 2, 64, 1300, (1300, 900), 700, "heads"),        # pieces, the wavefronts share a head
    (1, 1, 4, 4, 40, 1, 3, 700, None, 0, "plain"),
    (1, 1, 1, 1, 128, 1, 128, 40000, None, 0, "plain"),               # more pieces than a wavefront joins
]


def attend_inputs(case, dtype, fmt, seed=0):
    b, s, hq, hk, d, groups, page, longest, lengths, window, cl = case
    gen = torch.Generator().manual_seed(100 + seed + longest + d)
    per = -(-longest // page)
    caches = caches_of(b * per + 2, page, hk, d, groups, fmt, cl, gen)
    q = normal(gen, b, s, hq, d, dtype=dtype, scale=1.5)
    pages = torch.randperm(b * per + 2, generator=gen)[:b * per].to(torch.int32).reshape(b, per)
    return q, caches, pages, None if lengths is None else torch.tensor(lengths, dtype=torch.int32)


def close(got, q, caches, pages, lengths, longest, scale, window, what=""):
    o, size, score = ref.attention(q, caches, pages, lengths, longest, scale, window)
    bound = ref.bound(o, size, score, q.dtype, q.shape[-1], longest)
    g = got.double().cpu()
    assert g.shape == o.shape
    bad = ~(((g - o).abs() <= bound) | (torch.isnan(g) & torch.isnan(o)))
    assert not bad.any(), "%s: %d of %d off, the first by %g of %g allowed" % (what, int(bad.sum()), bad.numel(), float((g - o).abs()[bad][0]), float(bound[bad][0]))
    return o


@pytest.mark.parametrize("fmt", (E2M1, I8, E4M3))
@pytest.mark.parametrize("dtype", (F32, F16, BF16))
@pytest.mark.parametrize("case", ATTEND)
def test_attention(case, dtype, fmt):
    longest, window = case[7], case[9]
    q, caches, pages, lengths = attend_inputs(case, dtype, fmt)
    mine = [on_gpu(c) for c in caches]
    got = M.cache_attention(up(q), *mine, up(pages), up(lengths), longest, window=window)
    o = close(got, q, caches, pages, lengths, longest, q.shape[-1] ** -0.5, window)
    assert bool((got.cpu()[o == 0] == 0).all())              # what sees nothing


@pytest.mark.parametrize("fmt", (E2M1, I8, E4M3))
@pytest.mark.parametrize("d", (16, 24, 32, 48, 56, 72, 88, 104, 120, 136, 152, 184, 200, 216, 248))
def test_rows_that_end_inside_a_piece_of_a_load(d, fmt):
    """A row's bytes modulo 16 take every value there is; what lies beside a head's codes is another's, or a code that is no number."""
    dtype = (BF16, F16, F32)[d // 8 % 3]
    q, caches, pages, lengths = attend_inputs((2, 2, 6, 3, d, 1, 5, 140, (140, 66), 0, "plain"), dtype, fmt, seed=d)
    if fmt == E4M3:
        for c in caches[::2]:
            assert c.dtype == E4M3
            c.view(torch.uint8)[:, :, 1] = 0x7f                  # the head between the others: its own queries' results are none
    mine = [on_gpu(c) for c in caches]
    got = M.cache_attention(up(q), *mine, up(pages), up(lengths), 140)
    o = close(got, q, caches, pages, lengths, 140, d ** -0.5, 0)
    assert bool(torch.isnan(o[:, :, 2:4]).all()) == (fmt == E4M3) and not torch.isnan(o[:, :, :2]).any() and not torch.isnan(o[:, :, 4:]).any()


@pytest.mark.parametrize("fmt", (E2M1, I8, E4M3))
@pytest.mark.parametrize("multi", (1, 2))
def test_attention_of_what_is_not_seen(fmt, multi):
    """Behind the lengths, before a window, in pages that no table names: scales that are no numbers, infinite or huge, codes that are none."""
    case = (3, 4, 6, 3, 64, multi, 16, 100, (100, 37, 2), 20, "plain")
    q, caches, pages, lengths = attend_inputs(case, BF16, fmt)
    want = [c.clone() for c in caches]
    for i in range(3):
        n = int(lengths[i])
        for t in list(range(0, max(0, n - 4 - 20 + 1))) + list(range(n, 7 * 16)):
            for c in (1, 3):
                caches[c][pages[i, t // 16], t % 16] = (float("nan"), float("inf"), 1e30)[t % 3]
            if fmt == E4M3:
                for c in (0, 2):
                    caches[c].view(torch.uint8)[pages[i, t // 16], t % 16] = 0x7f
    got = M.cache_attention(up(q), *[up(c) for c in caches], up(pages), up(lengths), 100, window=20)
    clean = M.cache_attention(up(q), *[up(c) for c in want], up(pages), up(lengths), 100, window=20)
    assert torch.equal(got, clean) and bool(torch.isfinite(got).all())
    close(got, q, caches, pages, lengths, 100, 0.125, 20)


@pytest.mark.parametrize("fmt", (E2M1, E4M3))
def test_attention_of_rows_that_are_no_numbers(fmt):
    case = (4, 2, 4, 2, 128, 1, 16, 90, (90, 90, 90, 90), 0, "plain")
    q, caches, pages, lengths = attend_inputs(case, F16, fmt)
    pages[1, 3] = caches[0].shape[0]                         # a page that is not in the cache
    pages[2, 5] = -1                                         # of the last rows: 80 to 95, seen by both queries
    caches[1][pages[3, 5], 9, 1] = float("nan")              # row 89, seen by the second query only, of one head
    got = M.cache_attention(up(q), *[up(c) for c in caches], up(pages), up(lengths), 90)
    o = close(got, q, caches, pages, lengths, 90, 128 ** -0.5, 0)
    assert bool(torch.isnan(o[1:3]).all()) and not bool(torch.isnan(o[0]).any())
    assert bool(torch.isnan(o[3, 1, 2:]).all()) and not bool(torch.isnan(o[3, 1, :2]).any()) and not bool(torch.isnan(o[3, 0]).any())
    if fmt == E4M3:
        caches[1].copy_(caches[1].nan_to_num(0.01))
        caches[2].view(torch.uint8)[pages[0, 2], 7, 0, 5] = 0xff          # a code of a value: the row is none
        got = M.cache_attention(up(q[:1]), *[up(c) for c in caches], up(pages[:1]), up(lengths[:1]), 90)
        assert bool(torch.isnan(got[0, :, :2]).all()) and not bool(torch.isnan(got[0, :, 2:]).any())


def test_attention_takes_rows_of_any_strides_and_one_token_a_sequence():
    case = (3, 1, 6, 2, 64, 1, 16, 50, (50, 20, 33), 0, "plain")
    q, caches, pages, lengths = attend_inputs(case, F16, E2M1)
    mine = [up(c) for c in caches]
    want = M.cache_attention(up(q), *mine, up(pages), up(lengths), 50, scale=0.2)
    close(want, q, caches, pages, lengths, 50, 0.2, 0)
    for layout in ("heads", "wide", "fused", "strided"):
        assert torch.equal(M.cache_attention(laid(q, layout), *mine, up(pages), up(lengths), 50, scale=0.2), want), layout
        into = laid(torch.zeros_like(q), layout)
        assert M.cache_attention(up(q), *mine, up(pages), up(lengths), 50, scale=0.2, out=into) is into
        assert torch.equal(into, want), layout
    assert torch.equal(M.cache_attention(up(q[:, 0]), *mine, up(pages), up(lengths), 50, scale=0.2), want[:, 0])
    wide = torch.full((3, 9), 10 ** 6, dtype=torch.int32)    # a table wider than what is read, a slice of it
    wide[:, 2:6] = pages
    assert torch.equal(M.cache_attention(up(q), *mine, up(wide)[:, 2:], up(torch.stack((lengths, lengths), 1))[:, 1], 50, scale=0.2), want)
    assert M.cache_attention(up(q[:0]), *mine, up(pages[:0]), up(lengths[:0]), 50).shape == (0, 1, 6, 64)
    assert bool((M.cache_attention(up(q), *mine, up(pages), None, 0) == 0).all())


@pytest.mark.parametrize("fmt,d", ((E2M1, 64), (E2M1, 72), (I8, 128), (E4M3, 40)))
def test_codes_at_any_address(fmt, d):
    """Rows of a cache one byte off any alignment, wider than they are, and scales of every third float."""
    case = (2, 1, 6, 3, d, 1, 5, 200, (200, 77), 0, "plain")
    q, caches, pages, lengths = attend_inputs(case, F16, fmt)
    mine = []
    for c in caches:
        n = c.shape[-1]
        if c.dtype == F32:
            wide = torch.zeros(*c.shape[:-1], 3 * n, device="cuda")[..., 1::3]
        else:
            wide = torch.zeros(*c.shape[:-1], n + 9, dtype=torch.uint8, device="cuda").view(c.dtype)[..., 1:1 + n]
        mine.append(wide)
        wide.view(torch.uint8 if c.dtype != F32 else F32).copy_(c.view(torch.uint8 if c.dtype != F32 else F32).cuda())
    got = M.cache_attention(up(q), *mine, up(pages), up(lengths), 200)
    assert torch.equal(got, M.cache_attention(up(q), *[up(c) for c in caches], up(pages), up(lengths), 200))
    gen = torch.Generator().manual_seed(1)
    k, v, slots = normal(gen, 30, 3, d, dtype=F16), normal(gen, 30, 3, d, dtype=F16), torch.randperm(60, generator=gen)[:30].to(torch.int32)
    _, want = ref.append(None, k, v, slots, caches, None, None, False)
    M.cache_append_qkv(None, up(k), up(v), up(slots), *mine)
    for g, w in zip(mine, want):
        same(g.contiguous(), w)
    rows = mine[0].view(torch.uint8) if fmt != E2M1 else mine[0]
    base = rows.as_strided((*rows.shape[:-1], rows.shape[-1] + 9), rows.stride(), rows.storage_offset() - 1)
    assert bool((base[..., 0] == 0).all()) and bool((base[..., rows.shape[-1] + 1:] == 0).all())      # what lies between the rows


def test_attention_of_a_cache_past_32_bits():
    """Rows 5 GB into codes and into scales."""
    pages, page, h, d = 82000, 64, 8, 128
    cache = torch.empty(pages, page, h, d, dtype=torch.uint8, device="cuda")[..., :d // 2]
    scales = torch.empty(pages, page, h, 32, device="cuda")[..., :1]
    assert cache.stride(0) * pages > 2 ** 32 and scales.stride(0) * pages * 4 > 2 ** 32
    gen = torch.Generator().manual_seed(3)
    small = caches_of(5, page, h, d, 1, E2M1, "plain", gen)
    table = torch.tensor([[81999, 3, 81998, 40000, 81990]], dtype=torch.int32)
    for i, at in enumerate(table[0].tolist()):
        cache[at] = small[0][i].cuda()
        scales[at] = small[1][i].cuda()
    q = normal(gen, 1, 1, 16, d, dtype=BF16)
    got = M.cache_attention(up(q), cache, scales, cache, scales, up(table), None, 300)
    close(got, q, (small[0], small[1], small[0], small[1]), torch.arange(5, dtype=torch.int32)[None], None, 300, d ** -0.5, 0)
    del cache, scales
    torch.cuda.empty_cache()


# ---- together --------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", (E2M1, I8, E4M3))
def test_a_prompt_in_pieces_and_tokens_behind_it(fmt):
    """What a program does: a prompt appended in pieces, each attended to, then single tokens of two sequences; against the definitions' caches."""
    gen = torch.Generator().manual_seed(11)
    b, hq, hk, d, page, dtype = 2, 8, 2, 64, 16, BF16
    mine = [up(c) for c in caches_of(12, page, hk, d, 2, fmt)]
    caches = [c.cpu() for c in mine]
    pages = torch.randperm(12, generator=gen)[:10].to(torch.int32).reshape(b, 5)
    angle = torch.rand(80, d // 2, generator=gen, dtype=torch.float64) * 6
    table = torch.cat((angle.cos(), angle.sin()), 1).float()
    done = [0, 0]
    for s in (37, 20, 1, 1, 1):
        qkv = normal(gen, b, s, hq + 2 * hk, d, dtype=dtype)
        at = torch.stack([torch.arange(n, n + s) for n in done])
        slots = (pages.long().gather(1, at // page) * page + at % page).to(torch.int32)
        done = [n + s for n in done]
        lengths = torch.tensor(done, dtype=torch.int32)
        want_q, caches = ref.append(qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:], slots, caches, table, at.to(torch.int32), False)
        x = up(qkv)
        q = M.cache_append_qkv(x[:, :, :hq], x[:, :, hq:hq + hk], x[:, :, hq + hk:], up(slots), *mine, up(table), up(at.to(torch.int32)))
        out = M.cache_attention(q, *mine, up(pages), up(lengths), 80)
        same(q, want_q)
        close(out, want_q, caches, pages, lengths, 80, d ** -0.5, 0, "%d tokens" % s)
    if fmt != E2M1:                                          # the other operators of such a cache read and write the same
        k, v = M.cache_load_kv(*mine, up(pages), up(lengths), 60, dtype=F32)
        for g, c in ((k, 0), (v, 2)):
            full = ref.values(*caches[c:c + 2])[pages.long()].flatten(1, 2)[:, :60]
            assert torch.equal(g.cpu(), full.float())
