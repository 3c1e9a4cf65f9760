"""Cache operators on PyTorch tensors (public as functions of `model`): appending rotated keys and values to a paged cache of 4 or 8
bits, and attention that reads it as it is held.  include/gpuos.h says what they compute and take; everything here is checking
of shapes and marshalling.  They are not differentiable: what requires a gradient is refused where gradients are recorded."""
import struct
import sys

import torch
from torch.autograd import forward_ad
from torch.fx import _symbolic_trace

from . import runtime as R
from . import streams as S

APPEND, ATTENTION = 1, 2
OPERANDS = 11
# struct gpuos_cache_task: op, flags, size[12], operand[11] as {ptr, stride[4], dtype, pad}, alpha, pad
_TASK = struct.Struct("<II12q" + "Q4qB7x" * OPERANDS + "f4x")
assert _TASK.size == S.CACHE_TASK_BYTES
_CACHES = {torch.int8: 4, torch.float8_e4m3fn: 5, torch.uint8: 6}


def _caches_operand(c):
    return (c.data_ptr(), *c.stride(), _CACHES[c.dtype])


def _pack(op, flags, sizes, operands, alpha=0.0):
    fill = [x for o in operands for x in o] + [x for _ in range(OPERANDS - len(operands)) for x in M._NONE]
    return _TASK.pack(op, flags, *sizes, *(0,) * (12 - len(sizes)), *fill, alpha)


def _check_caches(dev, hk, d, k_cache, k_scales, v_cache, v_scales):
    M._check(k_cache, "k_cache", _CACHES, (4,), None, dev)
    wide = 2 if k_cache.dtype == torch.uint8 else 1
    M._need(d % wide == 0, "heads of a 4-bit cache have an even number of elements, not %d", d)
    M._check(v_cache, "v_cache", (k_cache.dtype,), (4,), k_cache.shape, dev)
    M._need(tuple(k_cache.shape[2:]) == (hk, d // wide), "caches are [pages, page, %d, %d], not %s", hk, d // wide, list(k_cache.shape))
    M._check(k_scales, "k_scales", M._F32, (4,), None, dev)
    M._check(v_scales, "v_scales", M._F32, (4,), k_scales.shape, dev)
    M._need(k_scales.shape[:3] == k_cache.shape[:3] and k_scales.shape[3] >= 1 and d % k_scales.shape[3] == 0,
            "scales are [pages, page, heads, groups] of the caches %s, not %s", list(k_cache.shape), list(k_scales.shape))


B = None                           # the module _binding, with the first call


def _load():
    """As runtime.lib: what is not built raises with the first call, not with the import."""
    global B
    try:
        from . import _binding
    except ImportError as e:
        raise FileNotFoundError("_binding.so is not built for this PyTorch; run `python -m paper_2604_17861_amd.build`") from e
    B = _binding
    return B


class _Plan:
    """A call's descriptor by everything about it but addresses: checked and packed once, then only the addresses are put in.  places: which operand each
    of the call's tensors is; written: which of them the caller gave and the call writes."""
    __slots__ = ("task", "places", "written", "device", "workspace", "empty")

    def __init__(self, task, places, written, device, empty):
        self.task, self.places, self.written, self.device, self.empty = task, bytes(places), bytes(written), device, empty
        self.workspace = R.cache_workspace(task)


_launch = None


def _run(plan, operands):
    """As model._run."""
    global _launch
    if plan.empty:
        return
    if forward_ad._current_level >= 0:
        M._no_tangent(operands)
    if M._modes() or _symbolic_trace._is_fx_tracing_flag or M._jit_tracing():
        M._under_modes(operands)
    if _launch is None:
        _launch = R.cache_launch_address()
    rc = B.launch(_launch, plan.task, plan.places, operands, plan.written, plan.device, plan.workspace, M._stream_of(plan.device))
    if rc:
        raise R.GpuosError(rc, "gpuos_launch_cache")


def append_task(q, k, v, slots, k_cache, k_scales, v_cache, v_scales, table=None, positions=None, out=None, *, pairs=False):
    """GPUOS_CACHE_APPEND as a descriptor (for runtime.launch_cache; it holds addresses, the caller keeps the tensors)."""
    M._check(k, "k", M._FLOAT, (3, 4))
    dev, sh = k.device, k.shape
    M._check(v, "v", (k.dtype,), None, sh, dev)
    hq = 0
    if q is not None:
        M._check(q, "q", (k.dtype,), (k.dim(),), None, dev)
        hq = q.shape[-2]
        M._need(q.shape[:-2] == sh[:-2] and q.shape[-1] == sh[-1], "q is %s with heads of its own, not %s", list(sh), list(q.shape))
        M._check(out, "out", (k.dtype,), None, q.shape, dev)
    else:
        M._need(out is None, "out without q")
    if table is not None:
        M._check(table, "table", M._F32, (2,), None, dev)
        if positions is not None:
            M._check(positions, "positions", M._INT, (1, 2), None, dev)
            ps = tuple(positions.shape)
            M._need(ps == tuple(sh[:-2]) or (k.dim() == 4 and ps == (sh[1],)), "positions are %s for k %s", list(sh[:-2]), list(sh))
    else:
        M._need(positions is None, "positions without a table")
    M._check(slots, "slots", M._INT, None, sh[:-2], dev)
    _check_caches(dev, sh[-2], sh[-1], k_cache, k_scales, v_cache, v_scales)
    (b, s, hk, d), ko = M._rows(k)
    rot, places = (table.shape[1], table.shape[0]) if table is not None else (0, 0)
    return _pack(APPEND, M.FLAG_PAIRS if pairs else 0, (b, s, hq, hk, d, rot, places, k_cache.shape[0], k_cache.shape[1], k_scales.shape[3]),
                 (M._NONE if q is None else M._rows(q)[1], ko, M._rows(v)[1], M._operand(table), M._NONE if positions is None else M._tokens(positions),
                  M._tokens(slots), M._NONE if q is None else M._rows(out)[1], _caches_operand(k_cache), M._operand(k_scales),
                  _caches_operand(v_cache), M._operand(v_scales)))


def attention_task(q, k_cache, k_scales, v_cache, v_scales, pages, lengths, longest, out, *, scale=None, window=0):
    """GPUOS_CACHE_ATTENTION as a descriptor (for runtime.launch_cache; it holds addresses, the caller keeps the tensors).  Its workspace has
    runtime.cache_workspace bytes, with out = q and D > 128 at least 4 B S Hq (D + 2)."""
    longest, window = int(longest), int(window)
    M._check(q, "q", M._FLOAT, (3, 4))
    dev = q.device
    M._check(k_cache, "k_cache", _CACHES, (4,), None, dev)
    qo, oo, sh = q, out, q.shape
    M._check(out, "out", (q.dtype,), None, sh, dev)
    if q.dim() == 3:                                        # one token a sequence
        qo, oo, sh = q.unsqueeze(1), out.unsqueeze(1), (sh[0], 1, *sh[1:])
    b, s, hq, d = sh
    hk = k_cache.shape[2]
    M._need(hk >= 1 and hq % hk == 0, "%d heads of queries are no multiple of %d of keys", hq, hk)
    _check_caches(dev, hk, d, k_cache, k_scales, v_cache, v_scales)
    M._check(pages, "pages", M._INT, (2,), None, dev)
    M._need(pages.shape[0] == b, "pages has a row for each of %d sequences", b)
    M._need(0 <= longest <= pages.shape[1] * k_cache.shape[1], "%d pages of %d do not hold %d rows", pages.shape[1], k_cache.shape[1], longest)
    M._need(window >= 0, "a window is 0 (none) or more")
    M._need(d % 8 == 0 and d <= 256, "heads have a multiple of eight elements, at most 256, not %d", d)
    group = d // k_scales.shape[3]
    M._need(group == d or (group >= 32 and group & (group - 1) == 0), "a scale is for the whole head or for a power of two of elements from 32 on, not %d", group)
    if lengths is not None:
        M._check(lengths, "lengths", M._INT, None, (b,), dev)
    scale = float(scale) if scale is not None else d ** -0.5 if d else 1.0
    return _pack(ATTENTION, 0, (b, s, hq, hk, d, k_cache.shape[0], k_cache.shape[1], k_scales.shape[3], pages.shape[1], longest, min(window, 2 ** 31 - 1)),
                 (M._operand(qo), _caches_operand(k_cache), M._operand(k_scales), _caches_operand(v_cache), M._operand(v_scales), M._operand(pages),
                  M._operand(lengths), M._operand(oo)), scale)


def _untraced(f):
    """f, kept from torch.compile, under which its checks see other values than are there.  (Only where that is loaded: it takes 0.8 s.)"""
    return torch.compiler.disable(f) if "torch._dynamo" in sys.modules else f


def cache_append_qkv(q, k, v, slots, k_cache, k_scales, v_cache, v_scales, table=None, positions=None, *, pairs=False, out=None):
    """Rotate q and k [T, H, D] or [B, S, H, D] by the angles of table [places, R] (cosines | sines, float32; None: not at all) at the tokens'
    positions (None: 0, 1, ... in every sequence; pairs: neighbours are rotated together, else the halves), and quantise k
    and v into slots (page index * page + place; negative: nowhere) of the caches [pages, page, H, D] (int8, float8_e4m3fn) or
    [pages, page, H, D / 2] (uint8: two e2m1 a byte, the earlier one in the lower half) and their scales [pages, page, H, groups]
    (float32), in one launch.  Returns q' (out may be q; None without q).  Slots are distinct.  Not differentiable: what
    requires a gradient is refused where gradients are recorded."""
    given = (q, k, v, table, positions, slots, out, k_cache, k_scales, v_cache, v_scales)      # in the descriptor's order
    key = (B or _load()).key(given) + (b"append pairs" if pairs else b"append")
    plan = M._plans.get(key)
    if plan is None:
        if q is not None and out is None:
            M._check(q, "q", M._FLOAT, (3, 4))
        M._no_gradient("cache_append_qkv", *given)
    made = q is not None and out is None
    operands = (q, k, v, table, positions, slots, B.like(q), k_cache, k_scales, v_cache, v_scales) if made else given
    if plan is None:
        task = _untraced(append_task)(q, k, v, slots, k_cache, k_scales, v_cache, v_scales, table, positions, operands[6], pairs=bool(pairs))
        plan = M._keep(key, _Plan(task, range(11), ([] if made or q is None else [6]) + [7, 8, 9, 10], k.get_device(),
                                  k.numel() == 0 and (q is None or q.numel() == 0)))
    _run(plan, operands)
    return operands[6]


def cache_attention(q, k_cache, k_scales, v_cache, v_scales, pages, lengths, longest, *, scale=None, window=0, out=None):
    """Attention of q [B, Hq, D] (a token of every sequence) or [B, S, Hq, D] over the first lengths[b] rows (None: all `longest`, which is the
    most there may be) of sequence b, through pages [B, width], in caches and scales as cache_append_qkv fills them, Hq a
    multiple of their H, D a multiple of 8 up to 256, a scale for D or 32 elements and more.  The S queries are the last of those rows: each sees the
    rows up to its own, with window > 0 the last `window` of these.  scale: of the scores (None: 1 / sqrt(D)).  A query that
    sees nothing gets zeros.  out may be q.  Not differentiable: what requires a gradient is refused where gradients are recorded."""
    longest, window = int(longest), int(window)
    given = (q, k_cache, k_scales, v_cache, v_scales, pages, lengths, out)      # in the descriptor's order
    key = (B or _load()).key(given), longest, window, scale if scale is None else float(scale)
    plan = M._plans.get(key)
    if plan is None:
        M._check(q, "q", M._FLOAT, (3, 4))
        M._no_gradient("cache_attention", *given)
    made = out is None
    operands = (q, k_cache, k_scales, v_cache, v_scales, pages, lengths, B.like(q)) if made else given
    if plan is None:
        task = _untraced(attention_task)(*operands[:7], longest, operands[7], scale=scale, window=window)
        plan = M._keep(key, _Plan(task, range(8), [] if made else [7], q.get_device(), q.numel() == 0))
    _run(plan, operands)
    return operands[7]


# Behind the functions, because model takes them from here, whichever of the two is imported first.
from . import model as M  # noqa: E402
