"""The cache's part of a decoding step or a prompt, as cases that can be timed and checked: queries and keys rotated by
position and keys and values quantised into a paged cache of 4 or 8 bits on the way, and attention that reads such a
cache as it is held.

`run` computes a case in plain torch operations in 32 bits, or, where `own` is set, by the library's calls
(`paper_2604_17861_amd.model`).  `exact` computes it in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
FORMATS = {"e2m1": torch.uint8, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
BITS = {"e2m1": 4, "int8": 8, "e4m3": 8}
QMAX = {"e2m1": 6.0, "int8": 127.0, "e4m3": 448.0}
RMS = {"e2m1": 2.93, "int8": 73.0, "e4m3": 100.0}       # of the values that `prepare` fills a cache with
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)         # by the lower three bits; the fourth is the sign
TINY = 2.0 ** -100                                      # the least maximum of a group that a scale is made of


# ---- cases ---------------------------------------------------------------------------------------

def listed():
    return [
        # the new token of one request, views of one projection's result: latency is what counts
        {"name": "append_token", "kind": "append", "b": 1, "s": 1, "hq": 16, "hk": 8, "d": 128, "r": 128, "pairs": False,
         "group": 128, "format": "e2m1", "page": 16, "dtype": "bf16", "layout": "fused", "cache": "pshd"},
        # the new tokens of a batch of requests, a scale for 32 elements each
        {"name": "append_batch", "kind": "append", "b": 64, "s": 1, "hq": 32, "hk": 8, "d": 128, "r": 128, "pairs": False,
         "group": 32, "format": "e2m1", "page": 16, "dtype": "bf16", "layout": "fused", "cache": "pshd"},
        # small and odd: heads before tokens, a part of each head rotated, neighbours as pairs, pages of 7
        {"name": "append_odd", "kind": "append", "b": 3, "s": 197, "hq": 12, "hk": 12, "d": 80, "r": 32, "pairs": True,
         "group": 80, "format": "int8", "page": 7, "dtype": "f32", "layout": "bhsd", "cache": "phsd"},
        # prompts into an 8-bit cache
        {"name": "append_prompts_8bit", "kind": "append", "b": 4, "s": 2048, "hq": 16, "hk": 16, "d": 128, "r": 128,
         "pairs": False, "group": 128, "format": "e4m3", "page": 64, "dtype": "f16", "layout": "bshd", "cache": "pshd"},
        # a long prompt into the 4-bit cache
        {"name": "append_prompt", "kind": "append", "b": 1, "s": 16384, "hq": 32, "hk": 8, "d": 128, "r": 128, "pairs": False,
         "group": 32, "format": "e2m1", "page": 64, "dtype": "bf16", "layout": "fused", "cache": "pshd"},
        # one request with a short history: latency
        {"name": "attend_request", "kind": "attend", "b": 1, "s": 1, "l": 301, "hq": 16, "hk": 8, "d": 128, "group": 128,
         "format": "e2m1", "page": 16, "window": 0, "dtype": "bf16", "cache": "pshd"},
        # one request with a long document behind it
        {"name": "attend_document", "kind": "attend", "b": 1, "s": 1, "l": 131072, "hq": 32, "hk": 8, "d": 128, "group": 32,
         "format": "e2m1", "page": 64, "window": 0, "dtype": "bf16", "cache": "pshd"},
        # a batch of requests of different lengths
        {"name": "attend_batch", "kind": "attend", "b": 64, "s": 1, "l": 4096, "hq": 32, "hk": 8, "d": 128, "group": 128,
         "format": "e2m1", "page": 16, "window": 0, "dtype": "bf16", "cache": "pshd"},
        # the same from an 8-bit cache whose pages have heads before slots
        {"name": "attend_batch_8bit", "kind": "attend", "b": 32, "s": 1, "l": 4096, "hq": 16, "hk": 8, "d": 128, "group": 128,
         "format": "int8", "page": 64, "window": 0, "dtype": "f16", "cache": "phsd"},
        # a head of keys for each of queries, heads of 80, a few drafted tokens, a window, pages of 7, fp32
        {"name": "attend_odd", "kind": "attend", "b": 5, "s": 3, "l": 777, "hq": 12, "hk": 12, "d": 80, "group": 80,
         "format": "e4m3", "page": 7, "window": 200, "dtype": "f32", "cache": "phsd"},
        # drafted tokens checked in a batch, narrow heads, eight queries a key
        {"name": "attend_drafts", "kind": "attend", "b": 16, "s": 4, "l": 8192, "hq": 32, "hk": 4, "d": 64, "group": 64,
         "format": "e2m1", "page": 32, "window": 0, "dtype": "bf16", "cache": "pshd"},
        # a piece of a prompt over itself and what is in the cache before it
        {"name": "attend_prompt", "kind": "attend", "b": 1, "s": 1024, "l": 4096, "hq": 32, "hk": 8, "d": 128, "group": 128,
         "format": "e2m1", "page": 64, "window": 0, "dtype": "bf16", "cache": "pshd"},
    ]


def draw(rng):
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    kind = rng.choice(["append", "attend"])
    c = {"kind": kind, "dtype": rng.choice(["f32", "f16", "bf16", "bf16"]), "format": rng.choice(["e2m1", "e2m1", "int8", "e4m3"]),
         "page": rng.choice([1, 16, 32, 64, rng.randint(2, 200)]), "cache": rng.choice(["pshd", "phsd"])}
    hk = rng.choice([1, 2, 4, 8, 12, 16])
    hq = hk * rng.choice([1, 2, 4, 5, 8])
    if kind == "append":
        d = rng.choice([64, 80, 96, 128, 128, 192, 256, 2 * rng.randint(8, 128)])
        tokens = logint(1, (16 << 20) // ((hq + 2 * hk) * d))
        b = min(tokens, logint(1, 64))
        c.update(b=b, s=max(1, tokens // b), r=rng.choice([d, d, 2 * max(1, d // 8), 2 * rng.randint(1, d // 2)]),
                 pairs=rng.random() < 0.4, layout=rng.choice(["fused", "bshd", "bhsd"]))
        least = 16
    else:
        d = rng.choice([64, 80, 96, 128, 128, 192, 256, 8 * rng.randint(2, 32)])
        tokens = logint(1, (64 << 20) // (hk * d))
        b = min(tokens, logint(1, 64))
        l = max(1, tokens // b)
        # one token a sequence, a few, or a piece of a prompt
        s = min(l, rng.choice([1, 1, 1, rng.randint(2, 8), logint(9, 600)]), max(1, (8 << 30) // (b * l * hq * d)))
        c.update(b=b, s=s, l=l, window=rng.choice([0, 0, logint(1, 2 * l)]))
        least = 32
    c.update(hq=hq, hk=hk, d=d, group=rng.choice([d] + [g for g in (16, 32, 64, 128) if g >= least and d % g == 0]))
    return c


# ---- inputs ----------------------------------------------------------------------------------------

def _width(case):
    return case["d"] * BITS[case["format"]] // 8


def _cache(case, pages):
    """A cache's bytes and scales, [pages, page, heads, ...] however they lie in memory."""
    h, page = case["hk"], case["page"]

    def make(n, dtype):
        if case["cache"] == "pshd":
            return torch.zeros(pages, page, h, n, dtype=dtype, device="cuda")
        return torch.zeros(pages, h, page, n, dtype=dtype, device="cuda").transpose(1, 2)
    return make(_width(case), FORMATS[case["format"]]), make(case["d"] // case["group"], torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 6007 + 17)
    dt = DTYPES[case["dtype"]]
    b, s, hq, hk, d, page = (case[k] for k in ("b", "s", "hq", "hk", "d", "page"))

    def normal(*shape, scale=1.0, dtype=dt):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, scale, generator=gen).to(dtype)

    def ints(lo, hi, *shape, dtype=torch.int32):
        return torch.randint(lo, hi, shape, dtype=dtype, device="cuda", generator=gen)

    state = {"case": dict(case)}
    if case["kind"] == "append":
        r = case["r"]
        if case["layout"] == "fused":
            qkv = normal(b, s, hq + 2 * hk, d)
            q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:]
        elif case["layout"] == "bshd":
            q, k, v = normal(b, s, hq, d), normal(b, s, hk, d), normal(b, s, hk, d)
        else:
            q, k, v = (normal(b, h, s, d).transpose(1, 2) for h in (hq, hk, hk))
        # positions: requests at different places of their sequences; angles made in 64 bits
        freq = 10000.0 ** (-torch.arange(r // 2, dtype=torch.float64, device="cuda") * 2 / r)
        angle = torch.arange(s + 4096, dtype=torch.float64, device="cuda")[:, None] * freq
        positions = ints(0, 4096, b, 1) + torch.arange(s, dtype=torch.int32, device="cuda")
        # every sequence goes into pages of its own, in any order, from some place of the first on; a sixteenth of the tokens of a batch are
        # padding (slot -1)
        per = -(-s // page) + 1
        ids = torch.randperm(b * per + 2, device="cuda", generator=gen)[:b * per].to(torch.int32).reshape(b, per)
        at = ints(0, page, b, 1) + torch.arange(s, dtype=torch.int32, device="cuda")
        slots = ids.gather(1, (at // page).long()) * page + at % page
        if b * s > 1:
            slots = torch.where(ints(0, 16, b, s) == 0, torch.full_like(slots, -1), slots)
        state.update(q=q, k=k, v=v, table=torch.cat((angle.cos(), angle.sin()), 1).float(), positions=positions, slots=slots.contiguous())
        for name in "kv":
            cache, scales = _cache(case, b * per + 2)
            state.update({name + "_cache": cache, name + "_scales": scales})
        return state
    l = case["l"]
    per = -(-l // page)
    # scores spread as those of trained heads do: a few of a thousand rows have most of the weight
    state["q"] = normal(b, s, hq, d, scale=2.0)
    state["pages"] = torch.randperm(b * per + 3, device="cuda", generator=gen)[:b * per].to(torch.int32).reshape(b, per)
    state["lengths"] = ints(max(s, l // 2), l + 1, b) if b > 1 else torch.full((1,), l, dtype=torch.int32, device="cuda")
    for name in "kv":
        cache, scales = _cache(case, b * per + 3)
        if case["format"] == "e2m1":
            cache.copy_(ints(0, 256, *cache.shape, dtype=torch.uint8))
        elif case["format"] == "int8":
            cache.copy_(ints(-127, 128, *cache.shape, dtype=torch.int8))
        else:
            cache.copy_(normal(*cache.shape, scale=100.0, dtype=torch.float16).clamp_(-448, 448).to(torch.float8_e4m3fn))
        scales.uniform_(0.5 / RMS[case["format"]], 1.5 / RMS[case["format"]], generator=gen)
        state.update({name + "_cache": cache, name + "_scales": scales})
    return state


# ---- one pass --------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    caches = tuple(state[k] for k in ("k_cache", "k_scales", "v_cache", "v_scales"))
    if own:
        from paper_2604_17861_amd import model as M
        if case["kind"] == "append":
            q = M.cache_append_qkv(state["q"], state["k"], state["v"], state["slots"], *caches, state["table"], state["positions"],
                                   pairs=case["pairs"])
            return (q, *caches)
        return M.cache_attention(state["q"], *caches, state["pages"], state["lengths"], case["l"], window=case["window"])
    if case["kind"] == "append":
        slots = state["slots"]
        valid = slots >= 0
        page, place = slots[valid].long() // case["page"], slots[valid].long() % case["page"]
        q, k = _turn(state["q"], state), _turn(state["k"], state)
        for rows, cache, scales in ((k, *caches[:2]), (state["v"].float(), *caches[2:])):
            codes, scale = _quantise(rows[valid], case)
            cache.view(torch.uint8)[page, place] = codes.view(torch.uint8)
            scales[page, place] = scale
        return (q.to(state["q"].dtype), *caches)
    return _attend(state, case).to(state["q"].dtype)


def _turn(x, state):
    """The rotation of [b, s, h, d]; every product and every sum is rounded to 32 bits by itself."""
    case = state["case"]
    r, n = case["r"], case["r"] // 2
    x = x.float()
    angles = state["table"][state["positions"].long()][:, :, None]
    c, s = angles[..., :n], angles[..., n:]
    if case["pairs"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        z = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = x[..., :n], x[..., n:r]
        z = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((z, x[..., r:]), -1)


def _quantise(x, case):
    """The codes and the scale of each group; every rounding is one of 32 bits, the last one is to the nearest code, to the even one of two."""
    n, h, d = x.shape
    x = x.reshape(n, h, d // case["group"], case["group"])
    qmax = torch.full((), QMAX[case["format"]], device=x.device)
    top = x.abs().amax(-1, keepdim=True).clamp_min(TINY)
    y = (x * (qmax / top)).reshape(n, h, d)
    if case["format"] == "int8":
        codes = y.round().to(torch.int8)
    elif case["format"] == "e4m3":
        codes = y.clamp(-448, 448).to(torch.float8_e4m3fn)
    else:
        m = y.abs()
        code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
                + 8 * torch.signbit(y).to(torch.uint8)).to(torch.uint8)
        codes = code[..., 0::2] + 16 * code[..., 1::2]
    return codes, (top / qmax)[..., 0]


def _read(state, name):
    """Every sequence's rows, [b, h, l, d] in 32 bits."""
    case = state["case"]
    l, page = case["l"], case["page"]
    at = torch.arange(l, device="cuda")
    pages = state["pages"].long()[:, at // page]
    # (indexed as bytes: an 8-bit float is one of these)
    codes = state[name + "_cache"].view(torch.uint8)[pages, at % page]
    scale = state[name + "_scales"][pages, at % page]
    if case["format"] == "e2m1":
        value = torch.tensor(E2M1 + tuple(-v for v in E2M1), device="cuda")
        x = torch.stack((value[(codes & 15).int()], value[(codes >> 4).int()]), -1).flatten(-2)
    else:
        x = codes.view(FORMATS[case["format"]]).float()
    return (x.reshape(*scale.shape, case["group"]) * scale[..., None]).flatten(-2).transpose(1, 2).contiguous()


def _attend(state, case):
    b, s, hq, hk, d, l = (case[k] for k in ("b", "s", "hq", "hk", "d", "l"))
    k, v = _read(state, "k"), _read(state, "v")
    # the queries that share a head of keys are rows of one product
    q = state["q"].float().reshape(b, s, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, hq // hk * s, d) * (1 / math.sqrt(d))
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).reshape(b, hk, hq // hk, s, l)
    at = torch.arange(l, device="cuda")
    here = state["lengths"].long()[:, None] - s + torch.arange(s, device="cuda")
    seen = at <= here[..., None]
    if case["window"]:
        seen &= at > here[..., None] - case["window"]
    seen = seen[:, None, None]
    x = torch.where(seen, x, torch.full((), -math.inf, device="cuda"))
    top = x.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(x - top), torch.zeros((), device="cuda"))
    o = torch.matmul(p.reshape(b, hk, hq // hk * s, l), v).reshape(b, hk, hq // hk, s, d)
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, o / total, torch.zeros((), device="cuda"))
    return o.permute(0, 3, 1, 2, 4).reshape(b, s, hq, d)


def _seen(case):
    """Rows of the cache that a sequence's queries see together, and pairs of a query and a row, on average."""
    s, l, w = case["s"], case["l"], case["window"]
    n = l if case["b"] == 1 else (max(s, l // 2) + l) / 2
    rows = min(n, s - 1 + w) if w else n
    first = n - s + 1                                   # what the first query has behind it, itself included
    pairs = s * (first + n) / 2
    if w:
        short = min(s, max(0.0, w - first))             # queries that the window cuts nothing from
        pairs = short * first + short * (short - 1) / 2 + (s - short) * min(w, n)
    return rows, pairs


def work(case):
    e, group = SIZE[case["dtype"]], case["group"]
    per = _width(case) + 4 * (case["d"] // group)       # bytes of a head's row in the cache
    if case["kind"] == "append":
        tokens = case["b"] * case["s"]
        stored = tokens * (15 / 16 if tokens > 1 else 1.0)
        n = tokens * (case["hq"] + 2 * case["hk"]) * case["d"]
        angles = min(tokens, case["s"] + 4096) * case["r"] * 4
        return {"bytes": n * e + tokens * case["hq"] * case["d"] * e + stored * 2 * case["hk"] * per + angles + 8 * tokens, "flops": 5 * n}
    rows, pairs = _seen(case)
    n = case["b"] * case["s"] * case["hq"] * case["d"]
    return {"bytes": 2 * n * e + case["b"] * rows * 2 * case["hk"] * per, "flops": 4 * case["b"] * pairs * case["hq"] * case["d"]}


# ---- the same in 64 bits, written from the definitions ----------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    d, page, fmt = case["d"], case["page"], case["format"]
    if case["kind"] == "append":
        r, n = case["r"], case["r"] // 2
        first = torch.arange(n, device="cuda") * (2 if case["pairs"] else 1)
        second = first + (1 if case["pairs"] else n)
        turn = st["table"].double()[st["positions"].long()].unsqueeze(2)
        cos, sin = turn[..., :n], turn[..., n:]

        def turned(x, rounded):
            x = x.double().contiguous()
            z = x.clone()
            z[..., first] = rounded(rounded(x[..., first] * cos) - rounded(x[..., second] * sin))
            z[..., second] = rounded(rounded(x[..., second] * cos) + rounded(x[..., first] * sin))
            return z
        slots = st["slots"].flatten()
        rows = (slots >= 0).nonzero()[:, 0]
        where = slots[rows].long()
        result = [turned(st["q"], lambda z: z)]
        # the definition of what is stored has roundings to 32 bits: the rotation's products and sums, the scale, its inverse, the product with it
        keys = turned(st["k"], lambda z: z.float().double())
        for name, x in (("k", keys), ("v", st["v"].double())):
            x = x.flatten(0, 1)[rows].unflatten(-1, (-1, case["group"]))
            top = x.abs().amax(-1, keepdim=True).clamp(min=TINY)
            y = (x * (QMAX[fmt] / top).float().double()).float().double().flatten(-2)
            cache, scales = st[name + "_cache"], st[name + "_scales"].double()
            if fmt == "int8":
                full = cache.clone()
                full[where // page, where % page] = torch.round(y).to(torch.int8)
            elif fmt == "e4m3":                          # to the nearest of the 3-bit fractions, subnormal below 2^-6
                full = cache.float().double()
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                full[where // page, where % page] = (torch.round(y / step) * step).clamp(-448, 448)
            else:                                        # to the nearest 1-bit fraction, subnormal below 1
                m = y.abs()
                step = torch.exp2(torch.floor(torch.log2(m.clamp(min=1.0))) - 1)
                m = torch.round(m / step) * step
                code = torch.zeros_like(m, dtype=torch.long)
                for i, value in enumerate(E2M1):
                    code[m == value] = i
                code += 8 * torch.signbit(y).long()
                full = cache.clone()
                full[where // page, where % page] = (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8)
            scales[where // page, where % page] = (top / QMAX[fmt]).float().double().squeeze(-1)
            result += [full, scales]
        return tuple(result)
    s, hk, per_k = case["s"], case["hk"], case["hq"] // case["hk"]
    out = torch.zeros(case["b"], s, case["hq"], d, dtype=torch.float64, device="cuda")
    for b, length in enumerate(st["lengths"].tolist()):
        kv = []
        for name in "kv":
            ids = st["pages"][b].long()
            codes, scale = st[name + "_cache"].view(torch.uint8)[ids].flatten(0, 1)[:length], st[name + "_scales"][ids].flatten(0, 1)[:length].double()
            if fmt == "e2m1":
                nibbles = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
                e, f = (nibbles >> 1) & 3, (nibbles & 1).double()
                x = torch.where(e > 0, (1 + f / 2) * torch.exp2(e.double() - 1), f / 2) * (1 - 2 * (nibbles >> 3)).double()
            elif fmt == "int8":
                x = codes.view(torch.int8).double()
            else:
                x = codes.view(torch.float8_e4m3fn).float().double()
            kv.append(x * scale.repeat_interleave(case["group"], -1))
        at = torch.arange(length, device="cuda")
        here = length - s + torch.arange(s, device="cuda")[:, None]
        hidden = at > here
        if case["window"]:
            hidden |= at <= here - case["window"]
        for h in range(hk):
            q = st["q"][b, :, h * per_k:(h + 1) * per_k].double().transpose(0, 1)
            x = (q @ kv[0][:, h].T.contiguous()) / math.sqrt(d)
            p = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
            out[b, :, h * per_k:(h + 1) * per_k] = (p @ kv[1][:, h].contiguous()).transpose(0, 1)
    return out
