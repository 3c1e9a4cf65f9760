"""The model operators by their definitions, on the CPU: norm and rotation with their gradients in 64 bits beside the sizes that
their rounding errors scale with; the cache and the penalties in 32 bits, operation by operation, as they are defined."""
import torch

U = 2.0 ** -24                     # half a step of fp32, relative


def _halves(t, r, pairs):
    return (t[..., 0:r:2], t[..., 1:r:2]) if pairs else (t[..., :r // 2], t[..., r // 2:r])


def _join(a, b, rest, pairs):
    turned = torch.stack((a, b), -1).flatten(-2) if pairs else torch.cat((a, b), -1)
    return torch.cat((turned, rest), -1)


def _angles(x, table, positions):
    """cosines and sines of every token, [..., 1, R / 2]; NaN where the position is not in the table"""
    lead = x.shape[:-2]
    if positions is None:
        positions = torch.arange(lead[-1]).expand(lead)
    p = positions.expand(lead).long()
    inside = (p >= 0) & (p < table.shape[0])
    rows = table.double()[torch.where(inside, p, 0)]
    rows = torch.where(inside[..., None], rows, float("nan"))[..., None, :]
    n = table.shape[1] // 2
    return rows[..., :n], rows[..., n:]


def norm_rope(x, gamma, table, positions, eps, pairs):
    """(z, scale): the result and the size of the terms that its errors scale with"""
    x = x.double()
    g = gamma.double() if gamma is not None else torch.ones(x.shape[-1], dtype=torch.float64)
    y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * g
    if table is None or table.shape[1] == 0:
        return y, y.abs()
    r = table.shape[1]
    c, s = _angles(x, table, positions)
    a, b = _halves(y, r, pairs)
    rest = y[..., r:] + 0 * c[..., :1]                       # (NaN with the rest of its row)
    z = _join(a * c - b * s, b * c + a * s, rest, pairs)
    size = _join((a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs(), rest.abs(), pairs)
    return z, size


def norm_rope_grad(dz, x, gamma, table, positions, eps, pairs):
    """(dx, its errors' scale, dgamma, the sum of its terms' sizes)"""
    dz, x = dz.double(), x.double()
    d = x.shape[-1]
    g = gamma.double() if gamma is not None else torch.ones(d, dtype=torch.float64)
    if table is None or table.shape[1] == 0:
        dy, dy_size = dz, dz.abs()
    else:
        r = table.shape[1]
        c, s = _angles(x, table, positions)
        a, b = _halves(dz, r, pairs)
        rest = dz[..., r:] + 0 * c[..., :1]
        dy = _join(a * c + b * s, b * c - a * s, rest, pairs)
        dy_size = _join((a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs(), rest.abs(), pairs)
    inv = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    u, u_size = dy * g, dy_size * g.abs()
    dx = inv * (u - x * inv ** 2 * (u * x).mean(-1, keepdim=True))
    dx_size = inv * (u_size + x.abs() * inv ** 2 * (u_size * x.abs()).mean(-1, keepdim=True))
    lead = tuple(range(x.dim() - 1))
    return dx, dx_size, (dy * x * inv).sum(lead), (dy_size * x.abs() * inv).sum(lead)


def quantise(x, groups, fmt):
    """(8-bit values, scales) of rows [..., D]"""
    qmax = torch.tensor(127.0 if fmt == torch.int8 else 448.0)
    x = x.float().unflatten(-1, (groups, -1))
    m = x.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    m = m.clamp(min=2.0 ** -100)
    y = torch.where(bad, torch.zeros(()), x * (qmax / m)).flatten(-2)
    q = y.round().to(torch.int8) if fmt == torch.int8 else y.clamp(-448, 448).to(torch.float8_e4m3fn)
    return q, torch.where(bad, float("nan"), m / qmax)[..., 0]


def store(x, slots, cache, scales):
    """what cache and scales hold after the rows with a slot in them are stored (copies)"""
    cache, scales = cache.clone(), scales.clone()
    page = cache.shape[1]
    q, sc = quantise(x, scales.shape[-1], cache.dtype)
    raw = cache.view(torch.int8)
    for at, row, s in zip(slots.flatten().tolist(), q.view(torch.int8).flatten(0, -3), sc.flatten(0, -3)):
        if 0 <= at < cache.shape[0] * page:
            raw[at // page, at % page] = row
            scales[at // page, at % page] = s
    return cache, scales


def load(cache, scales, pages, lengths, length, dtype):
    b = pages.shape[0]
    out = torch.zeros(b, length, *cache.shape[2:])
    values = cache.float() if cache.dtype != torch.int8 else cache.to(torch.float32)
    wide = values * scales.repeat_interleave(cache.shape[3] // scales.shape[3], -1)
    for i in range(b):
        n = length if lengths is None else max(0, min(length, int(lengths[i])))
        for j in range(n):
            page = int(pages[i, j // cache.shape[1]])
            out[i, j] = wide[page, j % cache.shape[1]] if 0 <= page < cache.shape[0] else float("nan")
    return out.to(dtype)


def penalties(x, history=None, prompts=None, params=None, bias=None, allowed=None):
    dtype, (b, v) = x.dtype, x.shape
    x = x.float().clone()
    for i in range(b):
        if history is not None:
            ids = history[i].long()
            inside = (ids >= 0) & (ids < v)
            first = int(prompts[i]) if prompts is not None else 0
            behind = inside & (torch.arange(len(ids)) >= first)
            seen = torch.bincount(ids[inside], minlength=v)
            count = torch.bincount(ids[behind], minlength=v)
            rep, freq, pres = params[i]
            y = torch.where(x[i] > 0, x[i] / rep, x[i] * rep)
            y = y - count.float() * freq - torch.where(count > 0, pres, torch.zeros(()))
            x[i] = torch.where(seen > 0, y, x[i])
        if bias is not None:
            x[i] = x[i] + (bias if bias.dim() == 1 else bias[i]).float()
        if allowed is not None:
            words = allowed if allowed.dim() == 1 else allowed[i]
            at = torch.arange(v)
            x[i] = torch.where((words[at // 32] >> (at % 32).to(torch.int32)) & 1 != 0, x[i], -float("inf"))
    return x.to(dtype)
