"""The operators of a decoding or training step that stand round its matrix products, as cases that can be timed and
checked: queries and keys normalised by head and rotated by position (and the gradients of that), key and value rows
quantised into a paged 8-bit cache and sequences read back from it, penalties, bias and grammar mask on rows of logits.

`run` computes a case in plain torch operations in 32 bits, or, where `own` is set, by the library's calls
(`paper_2604_17861_amd.model`).  `exact` computes it in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "int8": torch.int8,
          "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
QMAX = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100                  # the least maximum of a group that a scale is made of


# ---- cases ---------------------------------------------------------------------------------------

def listed():
    return [
        # one token of one request: queries and keys of a layer, latency is what counts
        {"name": "rope_token", "kind": "rope", "b": 1, "s": 1, "hq": 16, "hk": 8, "d": 128, "r": 128, "pairs": False,
         "dtype": "bf16", "layout": "fused"},
        # a batch of decoding requests, queries and keys views of one projection's result
        {"name": "rope_batch", "kind": "rope", "b": 64, "s": 1, "hq": 32, "hk": 8, "d": 128, "r": 128, "pairs": False,
         "dtype": "bf16", "layout": "fused"},
        # prompts: long sequences
        {"name": "rope_prompt", "kind": "rope", "b": 2, "s": 4096, "hq": 32, "hk": 8, "d": 128, "r": 128, "pairs": False,
         "dtype": "bf16", "layout": "fused"},
        # training, small and odd: heads before tokens, a part of each head rotated, neighbours as pairs
        {"name": "rope_grad_odd", "kind": "rope_grad", "b": 3, "s": 197, "hq": 12, "hk": 12, "d": 80, "r": 32, "pairs": True,
         "dtype": "f32", "layout": "bhsd"},
        # training: a micro-batch of sequences
        {"name": "rope_grad_train", "kind": "rope_grad", "b": 4, "s": 2048, "hq": 16, "hk": 16, "d": 128, "r": 128,
         "pairs": False, "dtype": "bf16", "layout": "bshd"},
        # the new tokens of a decoding batch, written into the cache
        {"name": "store_tokens", "kind": "store", "t": 64, "h": 8, "d": 128, "group": 128, "format": "e4m3", "page": 16,
         "dtype": "bf16", "layout": "pshd"},
        # a prompt's keys and values, a scale for 32 elements each
        {"name": "store_prompt", "kind": "store", "t": 16384, "h": 8, "d": 128, "group": 32, "format": "int8", "page": 64,
         "dtype": "bf16", "layout": "pshd"},
        # one request's sequence, read back for attention
        {"name": "load_request", "kind": "load", "b": 1, "l": 1000, "h": 8, "d": 128, "group": 128, "format": "e4m3",
         "page": 16, "dtype": "bf16", "layout": "pshd"},
        # a batch of sequences of different lengths; heads before slots in a page
        {"name": "load_batch", "kind": "load", "b": 32, "l": 4096, "h": 8, "d": 128, "group": 128, "format": "int8",
         "page": 64, "dtype": "f16", "layout": "phsd"},
        # one request's logits over a vocabulary that is no multiple of anything
        {"name": "penalty_request", "kind": "penalty", "b": 1, "v": 32003, "n": 200, "dtype": "f32", "bias": False,
         "mask": False},
        # a batch with grammar masks and biases
        {"name": "penalty_batch", "kind": "penalty", "b": 64, "v": 100352, "n": 2048, "dtype": "bf16", "bias": True,
         "mask": True},
        # long contexts
        {"name": "penalty_long", "kind": "penalty", "b": 8, "v": 65537, "n": 32768, "dtype": "f16", "bias": False,
         "mask": False},
    ]


def draw(rng):
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rope", "rope_grad", "store", "load", "penalty"])
    c = {"kind": kind, "dtype": rng.choice(["f32", "f16", "bf16"])}
    if kind in ("rope", "rope_grad"):
        d = rng.choice([64, 80, 96, 128, 128, 192, 256, 2 * rng.randint(8, 128)])
        hk = rng.choice([1, 2, 4, 8, 12, 16])
        hq = hk * rng.choice([1, 1, 2, 4])
        tokens = logint(1, max(1, (20 << 20) // ((hq + hk) * d)))
        b = min(tokens, logint(1, 64))
        c.update(b=b, s=max(1, tokens // b), hq=hq, hk=hk, d=d, r=rng.choice([d, d, 2 * max(1, d // 8), 2 * rng.randint(1, d // 2)]),
                 pairs=rng.random() < 0.4, layout=rng.choice(["fused", "bshd", "bhsd"]))
    elif kind in ("store", "load"):
        d = rng.choice([64, 80, 128, 128, 256, rng.randint(16, 256)])
        h = rng.choice([1, 2, 4, 8, 12, 16])
        groups = [d] + [g for g in (16, 32, 64, 128) if d % g == 0]
        tokens = logint(1, max(1, (32 << 20) // (h * d)))
        c.update(h=h, d=d, group=rng.choice(groups), format=rng.choice(["int8", "e4m3"]), page=rng.choice([1, 16, 32, 64, rng.randint(2, 200)]),
                 layout=rng.choice(["pshd", "phsd"]))
        if kind == "store":
            c.update(t=tokens)
        else:
            b = min(tokens, logint(1, 64))
            c.update(b=b, l=max(1, tokens // b))
    else:
        v = logint(1000, 200000)
        b = logint(1, max(1, min(256, (6 << 20) // v)))
        c.update(v=v, b=b, n=logint(1, max(2, min(32768, (1 << 20) // b))), bias=rng.random() < 0.5, mask=rng.random() < 0.5)
    return c


# ---- inputs ----------------------------------------------------------------------------------------

def _pages_needed(case):
    per = -(-(case["t"] if case["kind"] == "store" else case["l"]) // case["page"])
    return per * (1 if case["kind"] == "store" else case["b"]) + 3


def _cache(case, pages):
    """A cache's 8-bit values and scales, [pages, page, heads, ...] however they lie in memory."""
    h, d, g, page = case["h"], case["d"], case["group"], case["page"]

    def make(n, dtype):
        if case["layout"] == "pshd":
            return torch.zeros(pages, page, h, n, dtype=dtype, device="cuda")
        return torch.zeros(pages, h, page, n, dtype=dtype, device="cuda").transpose(1, 2)
    return make(d, DTYPES[case["format"]]), make(d // g, torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 31)
    kind, dt = case["kind"], DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, shift=0.0, dtype=dt):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(shift, scale, generator=gen).to(dtype)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi, shape, dtype=torch.int32, device="cuda", generator=gen)

    state = {"case": dict(case)}
    if kind in ("rope", "rope_grad"):
        b, s, hq, hk, d, r = (case[k] for k in ("b", "s", "hq", "hk", "d", "r"))

        def heads(h):
            return normal(b, h, s, d).transpose(1, 2) if case["layout"] == "bhsd" else normal(b, s, h, d)
        if case["layout"] == "fused":
            qkv = normal(b, s, hq + 2 * hk, d)
            q, k = qkv[:, :, :hq], qkv[:, :, hq:hq + hk]
        else:
            q, k = heads(hq), heads(hk)
        # positions: requests at different places of their sequences; angles made in 64 bits
        places = s + 4096
        freq = 10000.0 ** (-torch.arange(r // 2, dtype=torch.float64, device="cuda") * 2 / r)
        angle = torch.arange(places, dtype=torch.float64, device="cuda")[:, None] * freq
        table = torch.cat((angle.cos(), angle.sin()), 1).float()
        positions = ints(0, 4096, b, 1) + torch.arange(s, dtype=torch.int32, device="cuda")
        state.update(q=q, k=k, gq=normal(d, scale=0.1, shift=1.0), gk=normal(d, scale=0.1, shift=1.0), table=table,
                     positions=positions)
        if kind == "rope_grad":
            state.update(dq=heads(hq), dk=heads(hk))
    elif kind == "store":
        t, h, d, page = case["t"], case["h"], case["d"], case["page"]
        pages = _pages_needed(case)
        # a sixteenth of the rows are padding (slot -1); the others go to slots of pages in any order
        order = torch.randperm(pages * page, device="cuda", generator=gen)[:t].to(torch.int32)
        if t > 256:                                     # (a prompt fills its pages in order)
            ids = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
            at = torch.arange(t, dtype=torch.int32, device="cuda")
            order = ids[(at // page).long()] * page + at % page
        slots = torch.where(ints(0, 16, t) == 0, torch.full_like(order, -1), order).contiguous()
        for name in ("k", "v"):
            cache, scales = _cache(case, pages)
            state.update({name: normal(t, h, d), name + "_cache": cache, name + "_scales": scales})
        state.update(slots=slots)
    elif kind == "load":
        b, l, h, d, page = case["b"], case["l"], case["h"], case["d"], case["page"]
        pages, per = _pages_needed(case), -(-l // page)
        table = torch.randperm(pages, device="cuda", generator=gen)[:b * per].to(torch.int32).reshape(b, per)
        lengths = ints(l // 2, l + 1, b) if b > 1 else torch.full((1,), l, dtype=torch.int32, device="cuda")
        for name in ("k", "v"):
            cache, scales = _cache(case, pages)
            if case["format"] == "int8":
                cache.copy_(torch.randint(-127, 128, cache.shape, dtype=torch.int8, device="cuda", generator=gen))
            else:
                cache.copy_(normal(*cache.shape, scale=100.0, dtype=torch.float16).clamp_(-448, 448).to(torch.float8_e4m3fn))
            scales.uniform_(0.5 / QMAX[case["format"]], 4.0 / QMAX[case["format"]], generator=gen)
            state.update({name + "_cache": cache, name + "_scales": scales})
        state.update(pages=table, lengths=lengths)
    else:
        b, v, n = case["b"], case["v"], case["n"]
        x = normal(b, v, scale=3.0)
        # tokens as text has them: a few very often; some rows shorter (padded with -1); a part of each is the prompt
        u = torch.rand(b, n, device="cuda", generator=gen)
        history = (v * u.pow(3)).to(torch.int32).clamp_(0, v - 1)
        lengths = ints(n // 2, n + 1, b, 1)
        history = torch.where(torch.arange(n, device="cuda") < lengths, history, torch.full_like(history, -1))
        prompt = (lengths[:, 0].float() * torch.rand(b, device="cuda", generator=gen)).to(torch.int32)
        params = torch.rand(b, 3, device="cuda", generator=gen) * torch.tensor([0.5, 0.5, 1.0], device="cuda")
        params[:, 0] += 1.0
        state.update(x=x, history=history, prompt=prompt, params=params.contiguous(), bias=None, allowed=None)
        if case["bias"]:
            bias = torch.where(torch.rand(v, device="cuda", generator=gen) < 0.01, normal(v, scale=4.0, dtype=torch.float32),
                               torch.zeros(v, device="cuda"))
            state.update(bias=bias)
        if case["mask"]:                                # a grammar allows a few per cent of the tokens, or all of them
            words = -(-v // 32)
            bits = torch.rand(b, words * 32, device="cuda", generator=gen) < torch.rand(b, 1, device="cuda", generator=gen)
            bits = bits.reshape(b, words, 32).long() << torch.arange(32, device="cuda")
            state.update(allowed=bits.sum(-1).to(torch.int32).contiguous())
    return state


# ---- one pass --------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        from paper_2604_17861_amd import model as M
        if kind == "rope":
            return M.norm_rope_qk(state["q"], state["k"], state["gq"], state["gk"], state["table"], state["positions"],
                                  eps=EPS, pairs=case["pairs"])
        if kind == "rope_grad":
            return M.norm_rope_qk_backward(state["dq"], state["dk"], state["q"], state["k"], state["gq"], state["gk"],
                                           state["table"], state["positions"], eps=EPS, pairs=case["pairs"])
        if kind == "store":
            M.cache_store_kv(state["k"], state["v"], state["slots"], state["k_cache"], state["k_scales"],
                             state["v_cache"], state["v_scales"])
            return state["k_cache"], state["k_scales"], state["v_cache"], state["v_scales"]
        if kind == "load":
            return M.cache_load_kv(state["k_cache"], state["k_scales"], state["v_cache"], state["v_scales"], state["pages"],
                                   state["lengths"], case["l"], dtype=DTYPES[case["dtype"]])
        return M.penalize_logits(state["x"], history=state["history"], prompt_lengths=state["prompt"],
                                 params=state["params"], bias=state["bias"], allowed=state["allowed"])
    if kind == "rope":
        return tuple(_rope(state[x], state["g" + x], state, case, torch.float32).to(state[x].dtype) for x in "qk")
    if kind == "rope_grad":
        (dq, dgq), (dk, dgk) = (_rope_grad(state["d" + x], state[x], state["g" + x], state, case, torch.float32) for x in "qk")
        return (dq.to(state["q"].dtype), dk.to(state["k"].dtype), dgq.to(state["gq"].dtype), dgk.to(state["gk"].dtype))
    if kind == "store":
        slots = state["slots"].long()
        valid = slots >= 0
        at = slots[valid]
        for name in ("k", "v"):
            q, scale = _quantise(state[name][valid], case)
            state[name + "_cache"].view(torch.int8)[at // case["page"], at % case["page"]] = q.view(torch.int8)
            state[name + "_scales"][at // case["page"], at % case["page"]] = scale
        return state["k_cache"], state["k_scales"], state["v_cache"], state["v_scales"]
    if kind == "load":
        return tuple(_read_back(state, name, case, torch.float32).to(DTYPES[case["dtype"]]) for name in ("k", "v"))
    return _penalties(state, case, torch.float32).to(state["x"].dtype)


def _turn(y, state, case, wide, back=False):
    """The rotation of [b, s, h, d], or its transpose."""
    r, n = case["r"], case["r"] // 2
    angles = state["table"].to(wide)[state["positions"].long()][:, :, None]
    c, s = angles[..., :n], angles[..., n:]
    if back:
        s = -s
    if case["pairs"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        z = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = y[..., :n], y[..., n:r]
        z = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((z, y[..., r:]), -1)


def _rope(x, gamma, state, case, wide):
    x, gamma = x.to(wide), gamma.to(wide)
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma
    return _turn(y, state, case, wide)


def _rope_grad(dz, x, gamma, state, case, wide):
    dz, x, gamma = dz.to(wide), x.to(wide), gamma.to(wide)
    dy = _turn(dz, state, case, wide, back=True)
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    u = dy * gamma
    dx = r * u - x * r ** 3 * (u * x).mean(-1, keepdim=True)
    return dx, (dy * x * r).sum((0, 1, 2))


def _quantise(x, case):
    """The 8-bit values and the scale of each group; every rounding is one of 32 bits."""
    n, h, d = x.shape
    x = x.float().reshape(n, h, d // case["group"], case["group"])
    qmax = torch.full((), QMAX[case["format"]], device=x.device)
    top = x.abs().amax(-1, keepdim=True).clamp_min(TINY)
    y = (x * (qmax / top)).reshape(n, h, d)
    q = y.round().to(torch.int8) if case["format"] == "int8" else y.clamp(-448, 448).to(torch.float8_e4m3fn)
    return q, (top / qmax)[..., 0]


def _read_back(state, name, case, wide):
    b, l, page = case["b"], case["l"], case["page"]
    at = torch.arange(l, device="cuda")
    pages = state["pages"].long()[:, at // page]
    # (indexed as bytes: an 8-bit float is one of these)
    q = state[name + "_cache"].view(torch.int8)[pages, at % page].view(DTYPES[case["format"]]).to(wide)
    scale = state[name + "_scales"][pages, at % page].to(wide)
    x = (q.reshape(*scale.shape, case["group"]) * scale[..., None]).reshape(b, l, case["h"], case["d"])
    inside = (at < state["lengths"][:, None])[:, :, None, None]
    return torch.where(inside, x, torch.zeros((), dtype=wide, device="cuda"))


def _penalties(state, case, wide):
    x, history = state["x"].to(wide), state["history"].long()
    b, v, n = case["b"], case["v"], case["n"]
    ids = torch.where(history >= 0, history, torch.full_like(history, v))
    ones = torch.ones_like(ids)
    behind = (torch.arange(n, device="cuda") >= state["prompt"][:, None]).long()
    seen = torch.zeros(b, v + 1, dtype=torch.long, device="cuda").scatter_add_(1, ids, ones)[:, :v]
    count = torch.zeros(b, v + 1, dtype=torch.long, device="cuda").scatter_add_(1, ids, behind)[:, :v]
    rep, freq, pres = (state["params"][:, k:k + 1].to(wide) for k in range(3))
    x = torch.where(seen > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - count.to(wide) * freq - (count > 0).to(wide) * pres
    if state["bias"] is not None:
        x = x + state["bias"].to(wide)
    if state["allowed"] is not None:
        bits = (state["allowed"][:, :, None] >> torch.arange(32, dtype=torch.int32, device="cuda")) & 1
        x = torch.where(bits.reshape(b, -1)[:, :v] != 0, x, torch.full((), -math.inf, dtype=wide, device="cuda"))
    return x


def work(case):
    kind = case["kind"]
    if kind in ("rope", "rope_grad"):
        tokens = case["b"] * case["s"]
        n = tokens * (case["hq"] + case["hk"]) * case["d"]
        passes = 2 if kind == "rope" else 3
        small = tokens * 4 + min(tokens, case["s"] + 4096) * case["r"] * 4
        return {"bytes": n * SIZE[case["dtype"]] * passes + small, "flops": n * (8 if kind == "rope" else 16)}
    if kind == "store":
        n = 2 * case["t"] * case["h"] * case["d"] * 15 / 16         # (a sixteenth is padding)
        return {"bytes": n * (SIZE[case["dtype"]] + 1 + 4 / case["group"]) + 4 * case["t"], "flops": 4 * n}
    if kind == "load":
        n = 2 * case["b"] * case["l"] * case["h"] * case["d"]
        part = 0.75 if case["b"] > 1 else 1.0                       # sequences are half as long as the longest at least
        return {"bytes": n * SIZE[case["dtype"]] + n * part * (1 + 4 / case["group"]), "flops": 2 * n * part}
    n = case["b"] * case["v"]
    small = 4 * case["b"] * case["n"] + (4 * case["v"] if case["bias"] else 0) + (n / 8 if case["mask"] else 0)
    return {"bytes": 2 * n * SIZE[case["dtype"]] + small, "flops": 4 * n}


# ---- the same in 64 bits, written from the definitions ----------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rope", "rope_grad"):
        d, r, n = case["d"], case["r"], case["r"] // 2
        first = torch.arange(n, device="cuda") * (2 if case["pairs"] else 1)
        second = first + (1 if case["pairs"] else n)
        turn = st["table"].double()[st["positions"].long()].unsqueeze(2)
        cos, sin = turn[..., :n], turn[..., n:]
        outs, gains = [], []
        for name in "qk":
            x, g = st[name].double().contiguous(), st["g" + name].double()
            inv = (x.square().sum(-1, keepdim=True) / d + EPS).rsqrt()
            if kind == "rope":
                y = x * inv * g
                z = y.clone()
                z[..., first] = y[..., first] * cos - y[..., second] * sin
                z[..., second] = y[..., second] * cos + y[..., first] * sin
                outs.append(z)
                continue
            dz = st["d" + name].double().contiguous()
            dy = dz.clone()
            dy[..., first] = dz[..., first] * cos + dz[..., second] * sin
            dy[..., second] = dz[..., second] * cos - dz[..., first] * sin
            n_hat = x * inv                              # y = n_hat * gamma
            gains.append((dy * n_hat).flatten(0, 2).sum(0))
            dn = dy * g
            outs.append(inv * (dn - n_hat * (dn * n_hat).sum(-1, keepdim=True) / d))
        return tuple(outs + gains)
    if kind == "store":
        result = []
        slots, page = st["slots"].tolist(), case["page"]
        rows = torch.tensor([i for i, s in enumerate(slots) if s >= 0], dtype=torch.long, device="cuda")
        where = torch.tensor([s for s in slots if s >= 0], dtype=torch.long, device="cuda")
        for name in ("k", "v"):
            x = st[name].double()[rows].unflatten(-1, (-1, case["group"]))
            top = x.abs().amax(-1, keepdim=True).clamp(min=TINY)
            # the definition has three roundings to 32 bits: the scale, its inverse, the product with it
            inverse = (QMAX[case["format"]] / top).float().double()
            y = (x * inverse).float().double().flatten(-2)
            values, scales = st[name + "_cache"], st[name + "_scales"].double()
            full = values.double() if case["format"] == "int8" else values.float().double()
            if case["format"] == "int8":
                y = torch.round(y)
            else:                                        # to the nearest of the 3-bit fractions, subnormal below 2^-6
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                y = (torch.round(y / step) * step).clamp(-448, 448)
            full[where // page, where % page] = y
            scales[where // page, where % page] = (top / QMAX[case["format"]]).float().double().squeeze(-1)
            result += [full.to(torch.int8) if case["format"] == "int8" else full, scales]
        return tuple(result)
    if kind == "load":
        result = []
        for name in ("k", "v"):
            q, scale = st[name + "_cache"], st[name + "_scales"].double()
            q = q.double() if case["format"] == "int8" else q.float().double()
            out = torch.zeros(case["b"], case["l"], case["h"], case["d"], dtype=torch.float64, device="cuda")
            for b, length in enumerate(st["lengths"].tolist()):
                pages = st["pages"][b].long()
                seq = q[pages].flatten(0, 1)[:length]
                out[b, :length] = seq * scale[pages].flatten(0, 1)[:length].repeat_interleave(case["group"], -1)
            result.append(out)
        return tuple(result)
    x = st["x"].double()
    for b in range(case["b"]):
        ids = st["history"][b]
        prompt = int(st["prompt"][b])
        rep, freq, pres = st["params"][b].double().tolist()
        total = torch.bincount(ids[ids >= 0].long(), minlength=case["v"]).double()
        tail = ids[prompt:]
        count = torch.bincount(tail[tail >= 0].long(), minlength=case["v"]).double()
        row = x[b]
        row = torch.where(total > 0, torch.where(row > 0, row / rep, row * rep), row)
        x[b] = row - count * freq - (count > 0).double() * pres
    if st["bias"] is not None:
        x += st["bias"].double()
    if st["allowed"] is not None:
        v = torch.arange(case["v"], device="cuda")
        x[(st["allowed"][:, v // 32] >> (v % 32).to(torch.int32)) & 1 == 0] = -math.inf
    return x
