"""The cache operators by their definitions, on the CPU: what is appended in 32 bits, operation by operation; attention in 64 bits,
beside the sizes that its rounding errors scale with."""
import math

import torch

import model_reference as ref

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
QMAX = {torch.uint8: 6.0, torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def rotate(x, table, positions, pairs):
    """Every product and sum rounded to 32 bits by itself; NaN where the position is not in the table."""
    x = x.float()
    if table is None or table.shape[1] == 0:
        return x
    r, lead = table.shape[1], x.shape[:-2]
    if positions is None:
        positions = torch.arange(lead[-1]).expand(lead)
    p = positions.expand(lead).long()
    inside = (p >= 0) & (p < table.shape[0])
    rows = torch.where(inside[..., None], table[torch.where(inside, p, 0)], float("nan"))[..., None, :]
    c, s = rows[..., :r // 2], rows[..., r // 2:]
    a, b = ref._halves(x, r, pairs)
    z = ref._join(a * c - b * s, b * c + a * s, x[..., r:], pairs)
    return torch.where(inside[..., None, None], z, float("nan"))


def encode(y):
    """Codes of e2m1 in bytes of their own: the nearest, the even one of two."""
    m = y.abs().double()
    value = E2M1.double()
    off = (m[..., None] - value).abs()
    low = off.min(-1).indices                                # (of two as near the first; the even one is taken below)
    up = (low + 1).clamp(max=7)
    tie = (off.gather(-1, low[..., None]) == off.gather(-1, up[..., None]))[..., 0] & (up != low)
    code = torch.where(tie & (low % 2 == 1), up, low)
    return (code + 8 * torch.signbit(y).long()).to(torch.uint8)


def quantise(x, groups, fmt):
    """(codes as they lie in the cache, scales) of rows [..., D]"""
    if fmt != torch.uint8:
        return ref.quantise(x, groups, fmt)
    qmax = torch.tensor(6.0)
    x = x.float().unflatten(-1, (groups, -1))
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    m = x.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -100)
    code = encode(torch.where(bad, torch.zeros(()), x * (qmax / m)).flatten(-2))
    return code[..., 0::2] + 16 * code[..., 1::2], torch.where(bad, float("nan"), m / qmax)[..., 0]


def append(q, k, v, slots, caches, table, positions, pairs):
    """(q', what the four tensors of caches hold behind the call)"""
    out = [c.clone() for c in caches]
    for x, cache, scales in ((rotate(k, table, positions, pairs), out[0], out[1]), (v.float(), out[2], out[3])):
        page = cache.shape[1]
        codes, sc = quantise(x, scales.shape[-1], cache.dtype)
        for at, row, s in zip(slots.flatten().tolist(), codes.view(torch.uint8).flatten(0, -3), sc.flatten(0, -3)):
            if 0 <= at < cache.shape[0] * page:
                cache.view(torch.uint8)[at // page, at % page] = row
                scales[at // page, at % page] = s
    return None if q is None else rotate(q, table, positions, pairs).to(q.dtype), out


def values(cache, scales):
    """What codes and scales stand for, in 64 bits: [pages, page, H, D]"""
    if cache.dtype == torch.uint8:
        nibbles = torch.stack((cache & 15, cache >> 4), -1).flatten(-2).long()
        x = E2M1.double()[nibbles & 7] * (1 - 2 * (nibbles >> 3)).double()
    else:
        x = cache.float().double()
    return x * scales.double().repeat_interleave(x.shape[-1] // scales.shape[-1], -1)


def attention(q, caches, pages, lengths, longest, scale, window=0):
    """(o, the sum of the sizes of its terms, the largest size of a score's terms) of q [B, S, Hq, D], each [B, S, Hq, D] or [B, S, Hq, 1]"""
    k_all, v_all = values(*caches[:2]), values(*caches[2:])
    b, s, hq, d = q.shape
    hk, page = k_all.shape[2], k_all.shape[1]
    out, size, score = (torch.zeros(b, s, hq, n, dtype=torch.float64) for n in (d, d, 1))
    for i in range(b):
        n = longest if lengths is None else max(0, min(longest, int(lengths[i])))
        for j in range(s):
            last = n - s + j
            first = max(0, last - window + 1) if window else 0
            if last < first:
                continue
            at = torch.arange(first, last + 1)
            entry = pages[i].long()[at // page]
            there = (entry >= 0) & (entry < k_all.shape[0])
            k, v = (torch.where(there[:, None, None], t[torch.where(there, entry, 0), at % page], float("nan")) for t in (k_all, v_all))
            for h in range(hq):
                terms = q[i, j, h].double() * k[:, h // (hq // hk)] * scale
                p = torch.softmax(terms.sum(-1), 0)
                out[i, j, h] = (p[:, None] * v[:, h // (hq // hk)]).sum(0)
                size[i, j, h] = (p[:, None] * v[:, h // (hq // hk)].abs()).sum(0)
                score[i, j, h] = terms.abs().sum(-1).max()
    return out, size, score


def bound(o, size, score, dtype, d, n):
    """How far a result may be off, in half steps u of 32 bits.  Roundings of a sum of N terms in 32 bits, each of half a step of what has been
    summed at most, are taken as independent: 6 sqrt(N) of the size of the terms (sums of a matrix instruction's 32 products have fewer).
    A score: all products are exact, a query of 16 / 32 bits is two / three parts at most, so N = 3 * 32 for each 32 elements begun; six roundings more (the group's
    scale, alpha, powers of two, the maximum taken off, the exponential).  It enters p as a power, in the weights and in their total:
    twice.  A weight: the value's scale, and bf16 parts that hold it to 2^-16 (two, for results of 16 bits) or 2^-23 (three).  The sums of
    n weights, of their products with codes (N = 3 n), of pieces; a division."""
    u = 2.0 ** -24
    steps = 6 * math.sqrt(96 * -(-d // 32)) + 6
    parts = 2.0 ** -23 if dtype == torch.float32 else 2.0 ** -16
    err = size * (2 * steps * u * score + parts + (6 * math.sqrt(3 * n) + 8) * u) + o.abs() * (6 * math.sqrt(n) + 8) * u
    half = torch.finfo(dtype).eps / 2
    least = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}[dtype]
    return err + half * (o.abs() + err) + least / 2
