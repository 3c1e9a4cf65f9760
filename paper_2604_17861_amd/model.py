"""Model operators on PyTorch tensors: the memory-bound steps that stand round a model's matrix products.

    q, k = norm_rope_qk(q, k, gamma_q, gamma_k, table, positions)      # norm of every head and rotation, differentiable
    cache_store_kv(k, v, slots, k_cache, k_scales, v_cache, v_scales)  # into a paged cache of 8-bit values (this and on: no gradients)
    k, v = cache_load_kv(k_cache, k_scales, v_cache, v_scales, pages, lengths, longest, dtype=q.dtype)
    x = penalize_logits(x, history=tokens, params=params, allowed=bits)

The functions launch the library's kernels on PyTorch's current stream of the tensors' device (gpuos_launch_model): they
wait for nothing, and may be captured into a graph.  The `*_task` functions make the descriptors that the functions
launch; `b"".join` of some goes to `Runtime.submit_model`, which runs them as tasks of the ring (bind the operators with
`register` first), or to `runtime.launch_model`; they hold addresses, the caller keeps the tensors.  include/gpuos.h says what every operator computes and takes.

PyTorch sees no operators here.  norm_rope and norm_rope_qk are autograd functions; everything else is refused where a gradient would be
lost, and so are second derivatives, forward mode and traces (make_fx, torch.export, torch.jit.trace).  torch.compile breaks its graph at a
call.  What a descriptor writes, autograd does not hear of.

Shapes: rows of heads are [T, H, D] or [B, S, H, D] of any strides, with one position, slot or length for each token or
sequence.  int32 is the only integer type.  Everything here is checking of shapes and marshalling.
"""
import struct
from array import array
from itertools import chain, repeat

import torch
from torch.autograd import forward_ad
from torch.fx import _symbolic_trace
from torch.utils._python_dispatch import _get_current_dispatch_mode_stack

from . import runtime as R
from . import streams as S

_FLOAT = {torch.float32: S.F32, torch.float16: S.F16, torch.bfloat16: S.BF16}
_DT = dict(_FLOAT)
_DT.update({torch.int32: S.I32, torch.int8: 4, torch.float8_e4m3fn: 5})
_CACHE = (torch.int8, torch.float8_e4m3fn)
FLAG_PAIRS = 4
PARTS_MAX = 1024
# struct gpuos_model_task: header, size[8], operand[8] as {ptr, stride[4], dtype, pad}, alpha, dep[3], pad
_TASK = struct.Struct("<HBBI8q" + "Q4qB7x" * 8 + "f3H6x")
assert _TASK.size == S.MODEL_TASK_BYTES
_NONE = (0, 0, 0, 0, 0, 0)
_PAD = ((0, 0, 0, 0), (0, 0, 0), (0, 0), (0,), ())


def register(rt):
    """Bind the model operators of `streams.MODEL_OP` on a Runtime."""
    for name, impl in S.MODEL_IMPL.items():
        rt.register_op(S.MODEL_OP[name], impl)


def launch(*tasks, device=None):
    """Descriptors as kernels on the current stream of `device` (None: the current device).  Under a dispatch filter its tasks on
    these tensors have to be complete (GpuosMode.settle)."""
    stream = torch.cuda.current_stream(device)
    R.launch_model(tasks[0] if len(tasks) == 1 else b"".join(tasks), stream.device_index, stream.cuda_stream)


# A call's descriptors by everything about it but addresses: checked and packed once, then only the addresses are put in.  (Checking and
# packing one of five operands takes 6.5 us, looking it up 2.)
_plans = {}
_WORDS = S.MODEL_TASK_BYTES // 8
_POINTER = 9                       # word of the first operand's address; the others' every six words


def _sig(t):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device(), t.is_neg())


class _Plan:
    """The descriptors of one or more tasks, without those that have nothing to do (an empty tensor has no address).
    rows: what tells which those are; operands: of every task, in the descriptor's order (None: left out); places: where each of them is in what
    _run is given (None: all tasks' operands, one after the other)."""
    __slots__ = ("words", "n", "device", "at")

    def __init__(self, rows, tasks, operands, places=None):
        tasks = [t for x, t in zip(rows, tasks) if x.numel() != 0]
        self.words = array("Q", b"".join(tasks))
        self.n, self.device = len(tasks), rows[0].get_device()
        _need(all(x.get_device() == self.device for x in rows), "the tensors of one call are on one device")
        if places is None:
            count = iter(range(8 * len(operands)))
            places = [[next(count) for _ in mine] for mine in operands]
        self.at = []                                        # (word, which of what _run is given)
        first = 0
        for x, mine, at in zip(rows, operands, places):
            if x.numel() != 0:
                for o in range(8):
                    self.words[first + _POINTER + 6 * o] = 0
                self.at += [(first + _POINTER + 6 * o, at[o]) for o, t in enumerate(mine) if t is not None]
                first += _WORDS


def _keep(key, plan):
    if len(_plans) >= 4096:
        _plans.clear()
    _plans[key] = plan
    return plan


def _run(plan, operands, written=()):
    """Launch with these addresses: the operands of all tasks, one after the other (or as the plan's `places` say).  written: tensors of the caller's among
    them that the call writes; what autograd has saved of those is no longer what it was."""
    if plan.n:
        if forward_ad._current_level >= 0:
            _no_tangent(operands)
        if _modes() or _symbolic_trace._is_fx_tracing_flag or _jit_tracing():
            _under_modes(operands)
        words = plan.words[:]
        for word, k in plan.at:
            words[word] = at = operands[k].data_ptr()
            if not at:
                _need(operands[k].numel() == 0, "a tensor without memory (of a trace, say)")
        R.launch_model_at(words.buffer_info()[0], plan.n, plan.device, _stream_of(plan.device))
        if written:
            try:
                torch._C._increment_version(written)        # (torch.autograd.graph.increment_version, 0.4 us less)
            except RuntimeError:                            # tensors of inference mode have no versions
                torch._C._increment_version([o for o in written if not o.is_inference()])


def _no_tangent(operands):
    """Inside forward_ad.dual_level: a tangent has no way through a kernel."""
    _need(all(t is None or forward_ad.unpack_dual(t).tangent is None for t in operands), "model operators have no forward-mode derivative")


_modes, _jit_tracing, _included = torch._C._len_torch_dispatch_stack, torch._C._is_tracing, torch._C._dispatch_tls_is_dispatch_key_included


def _under_modes(operands):
    """Tasks of this thread's dispatch filter may still be working on these.  A trace (the modes that have a key are those of make_fx and
    torch.export) would hold the results' allocation, and no kernel."""
    trace = _jit_tracing() or _included(torch._C.DispatchKey.PreDispatch)
    for f in _get_current_dispatch_mode_stack():
        if f in R.active_filters:
            f.settle(operands)
        trace = trace or getattr(f, "_mode_key", None) is not None
    _need(not trace, "model operators cannot be traced: PyTorch does not see their kernels")


# the handle of a device's current stream: torch.cuda.current_stream(device).cuda_stream, which makes two objects for it (1.1 us)
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


# ---- descriptors -----------------------------------------------------------------------------------

def _operand(t):
    """{ptr, stride[4], dtype} of a tensor of at most four dims, or of none."""
    if t is None:
        return _NONE
    st = t.stride()
    return (t.data_ptr(), *st, *_PAD[len(st)], _DT[t.dtype])


def _rows(t):
    """Rows of heads as [B, S, H, D]: sizes, and {ptr, stride[4], dtype}."""
    sh, st = t.shape, t.stride()
    if len(sh) == 4:
        return sh, (t.data_ptr(), *st, _DT[t.dtype])
    return (1, *sh), (t.data_ptr(), 0, *st, _DT[t.dtype])


def _tokens(t):
    """A number for each token, [B, S] like the rows it belongs to."""
    st = t.stride()
    if len(st) == 1:                                        # (one sequence; or the same numbers for every one)
        return (t.data_ptr(), 0, st[0], 0, 0, _DT[t.dtype])
    return (t.data_ptr(), *st, 0, 0, _DT[t.dtype])


def _pack(name, flags, sizes, operands, alpha=0.0, deps=()):
    n, fill = len(operands), []
    for o in operands:
        fill += o
    return _TASK.pack(S.MODEL_OP[name], n, 0, flags, *sizes, *(0,) * (8 - len(sizes)), *fill, *_NONE * (8 - n), alpha, *deps,
                      *(0,) * (3 - len(deps)))


def _need(ok, what, *args):
    if not ok:
        raise ValueError(what % args if args else what)


def _check(x, what, dtypes=None, dims=None, shape=None, device=None, dense=False):
    if not isinstance(x, torch.Tensor) or (device is None and x.device.type != "cuda") or (device is not None and x.device != device):
        raise ValueError("%s is a tensor on %s" % (what, device if device is not None else "a GPU"))
    if dtypes is not None and x.dtype not in dtypes:
        raise ValueError("%s is one of %s, not %s" % (what, ", ".join(str(d) for d in dtypes), x.dtype))
    if dims is not None and x.dim() not in dims:
        raise ValueError("%s has %s dims, not %d" % (what, " or ".join(map(str, dims)), x.dim()))
    if shape is not None and tuple(x.shape) != tuple(shape):
        raise ValueError("%s is %s, not %s" % (what, list(shape), list(x.shape)))
    if x.is_neg() or x.is_conj():
        raise ValueError("%s is a lazily negated view" % what)


_INT = (torch.int32,)
_F32 = (torch.float32,)


def _check_rope(x, gamma, table, positions, out):
    _check(x, "x", _FLOAT, (3, 4))
    dev, sh = x.device, x.shape
    _check(out, "out", _FLOAT, None, sh, dev)
    if gamma is not None:
        _check(gamma, "gamma", _FLOAT, None, sh[-1:], dev)
    if table is not None:
        _check(table, "table", _F32, (2,), None, dev)
        if positions is not None:
            _check(positions, "positions", _INT, (1, 2), None, dev)
            ps = tuple(positions.shape)
            _need(ps == tuple(sh[:-2]) or (len(sh) == 4 and ps == (sh[1],)), "positions are %s for x %s", list(sh[:-2]), list(sh))
    else:
        _need(positions is None, "positions without a table")


def _rope_operands(x, gamma, table, positions, out):
    sizes, xo = _rows(x)
    rot, places = (table.shape[1], table.shape[0]) if table is not None else (0, 0)
    return ((*sizes, rot, places), (xo, _operand(gamma), _operand(table), _NONE if positions is None else _tokens(positions),
                                    _rows(out)[1]))


def norm_rope_task(x, gamma, table, positions, out, *, eps=1e-6, pairs=False, deps=(), fence=False):
    """NORM_ROPE: every head of x normalised, its first table.shape[1] elements rotated, into out."""
    _check_rope(x, gamma, table, positions, out)
    sizes, ops = _rope_operands(x, gamma, table, positions, out)
    return _pack("NORM_ROPE", (FLAG_PAIRS if pairs else 0) | fence, sizes, ops, eps, deps)


def norm_rope_grad_task(dout, x, gamma, table, positions, dx, partial, *, eps=1e-6, pairs=False, deps=(), fence=False):
    """NORM_ROPE_GRAD: the gradient of x into dx, shares of gamma's gradient into the columns of partial [D, parts] (or None)."""
    _check_rope(x, gamma, table, positions, dx)
    _check(dout, "dout", _FLOAT, None, x.shape, x.device)
    if partial is not None:
        _check(partial, "partial", _F32, (2,), None, x.device)
        _need(partial.shape[0] == x.shape[-1], "partial has a row for each of %d elements", x.shape[-1])
    sizes, ops = _rope_operands(x, gamma, table, positions, dx)
    return _pack("NORM_ROPE_GRAD", (FLAG_PAIRS if pairs else 0) | fence, (*sizes, partial.shape[1] if partial is not None else 0),
                 (*ops, _rows(dout)[1], _operand(partial)), eps, deps)


def gamma_sum_task(partial, out, *, deps=(), fence=False):
    """GAMMA_SUM: the sums of partial's rows into out [D]."""
    _check(partial, "partial", _F32, (2,))
    _check(out, "out", _FLOAT, None, partial.shape[:1], partial.device)
    return _pack("GAMMA_SUM", int(fence), tuple(partial.shape), (_operand(partial), _operand(out)), 0.0, deps)


def _check_cache(x, what, cache, scales):
    _check(x, what, _FLOAT, (3, 4))
    dev = x.device
    _check(cache, "cache", _CACHE, (4,), None, dev)
    _check(scales, "scales", _F32, (4,), None, dev)
    _need(cache.shape[2:] == x.shape[-2:], "cache is [pages, page, %d, %d], not %s", *x.shape[-2:], list(cache.shape))
    _need(scales.shape[:3] == cache.shape[:3] and scales.shape[3] >= 1 and x.shape[-1] % scales.shape[3] == 0,
          "scales are [pages, page, heads, groups] of the cache %s, not %s", list(cache.shape), list(scales.shape))


def cache_store_task(x, slots, cache, scales, *, deps=(), fence=False):
    """CACHE_STORE: rows of x quantised into the slots of a cache [pages, page, H, D] and its scales [pages, page, H, groups]."""
    _check_cache(x, "x", cache, scales)
    _check(slots, "slots", _INT, None, x.shape[:-2], x.device)
    sizes, xo = _rows(x)
    return _pack("CACHE_STORE", int(fence), (*sizes, cache.shape[0], cache.shape[1], scales.shape[3]),
                 (xo, _tokens(slots), _operand(cache), _operand(scales)), 0.0, deps)


def cache_load_task(cache, scales, pages, lengths, out, *, deps=(), fence=False):
    """CACHE_LOAD: sequences of a cache by their page tables [B, width] into out [B, L, H, D]."""
    _check_cache(out, "out", cache, scales)
    _need(out.dim() == 4, "out is [B, L, H, D]")
    _check(pages, "pages", _INT, (2,), None, out.device)
    _need(pages.shape[0] == out.shape[0], "pages has a row for each of %d sequences", out.shape[0])
    _need(out.shape[1] <= pages.shape[1] * cache.shape[1], "%d pages of %d do not hold %d rows", pages.shape[1], cache.shape[1], out.shape[1])
    if lengths is not None:
        _check(lengths, "lengths", _INT, None, out.shape[:1], out.device)
    return _pack("CACHE_LOAD", int(fence), (*out.shape, cache.shape[0], cache.shape[1], scales.shape[3], pages.shape[1]),
                 (_operand(cache), _operand(scales), _operand(pages), _operand(lengths), _rows(out)[1]), 0.0, deps)


def penalty_task(x, out, history=None, prompt_lengths=None, params=None, bias=None, allowed=None, *, deps=(), fence=False):
    """LOGIT_PENALTY on x [B, V] into out.  history [B, N]; params [B, 3]: repetition, frequency, presence; bias [V] or
    [B, V]; allowed [(V + 31) // 32] or [B, that]: bits."""
    _check(x, "x", _FLOAT, (2,))
    b, v = x.shape
    dev = x.device
    _check(out, "out", _FLOAT, None, x.shape, dev)
    _need((history is None) == (params is None), "history and params go together")
    n = 0
    if history is not None:
        _check(history, "history", _INT, (2,), None, dev)
        _need(history.shape[0] == b, "history has a row for each of %d", b)
        _check(params, "params", _F32, None, (b, 3), dev)
        n = history.shape[1]
        if n == 0:                                          # (nothing is counted: as without one)
            history = params = prompt_lengths = None
    if prompt_lengths is not None:
        _need(history is not None, "prompt_lengths without a history")
        _check(prompt_lengths, "prompt_lengths", _INT, None, (b,), dev)

    def row(t, width, what, dtypes):
        if t is None:
            return _NONE
        _check(t, what, dtypes, (1, 2), (width,) if t.dim() == 1 else (b, width), dev)
        return (t.data_ptr(), 0, t.stride(0), 0, 0, _DT[t.dtype]) if t.dim() == 1 else _operand(t)
    return _pack("LOGIT_PENALTY", int(fence), (b, v, n),
                 (_operand(x), _operand(out), _operand(history), _operand(prompt_lengths), _operand(params), row(bias, v, "bias", _FLOAT),
                  row(allowed, (v + 31) // 32, "allowed", _INT)), 0.0, deps)


# ---- norm and rotation -----------------------------------------------------------------------------

def _parts(x, tensors=1):
    """Shares of gamma's gradient, a workgroup each: one for 32 rows, which is a workgroup's pass over rows of 128 elements of 16 bits (of 64 it
    takes twice as many rows, and half of the shares of a short call are empty; of 512 a quarter), at most PARTS_MAX, and of all tensors of
    a launch no more than the card's 256 units take at once by their registers (five of 16 bits each, four of 32).  Two of 8,192 x 16 heads
    of 128 bf16 with 1,024 / 768 / 640 / 512 shares each: 52, 46, 47, 48 us; 8,192 x 32 of fp32 153, 165, 155, 152; one alone 26 to 29."""
    rows = x.numel() // x.shape[-1]
    return min(PARTS_MAX, 256 * (4 if x.dtype == torch.float32 else 5) // tensors, max(1, rows // 32))


def _empty_like(x):
    return torch.empty_like(x, memory_format=torch.contiguous_format)


class _NormRope(torch.autograd.Function):
    """Any number of tensors with their gammas, rotated by one table: x0, gamma0, x1, gamma1, ..."""

    @staticmethod
    def forward(ctx, table, positions, eps, pairs, *xs):
        ctx.save_for_backward(table, positions, *xs)
        ctx.eps, ctx.pairs = eps, pairs
        return _norm_rope(xs[0::2], xs[1::2], table, positions, eps, pairs, [None] * (len(xs) // 2))

    @staticmethod
    def backward(ctx, *douts):
        table, positions, *xs = ctx.saved_tensors
        douts = [d.resolve_neg() for d in douts]            # (of a conjugate's imaginary part)
        if torch.is_grad_enabled():                         # (create_graph)
            return (None, None, None, None, *_NormRopeGrad.apply(table, positions, ctx.eps, ctx.pairs, len(douts), *douts, *xs))
        dxs, dgs = _norm_rope_backward(douts, xs[0::2], xs[1::2], table, positions, ctx.eps, ctx.pairs)
        return (None, None, None, None, *(g for pair in zip(dxs, dgs) for g in pair))


class _NormRopeGrad(torch.autograd.Function):
    """The gradients as results that know what they come from, so that whoever differentiates them again is told.  (once_differentiable marks
    them only where dout requires a gradient, and by a node that leads to none of their sources: a second derivative on the way to another
    is then left out in silence.)"""

    @staticmethod
    def forward(ctx, table, positions, eps, pairs, n, *tensors):
        xs = tensors[n:]
        dxs, dgs = _norm_rope_backward(tensors[:n], xs[0::2], xs[1::2], table, positions, eps, pairs)
        return tuple(g for pair in zip(dxs, dgs) for g in pair)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the gradients of norm_rope are not differentiable themselves")


def _norm_rope(xs, gammas, table, positions, eps, pairs, outs):
    eps, pairs = float(eps), bool(pairs)                    # (a key holds values, not objects)
    key = ("norm_rope", eps, pairs, *map(_sig, (table, positions, *xs, *gammas, *outs)))
    plan = _plans.get(key)
    if plan is None:
        _need(len(outs) == len(xs), "out has %d entries (None: made here)", len(xs))
    given, outs = [o for o in outs if o is not None], [_empty_like(x) if o is None else o for x, o in zip(xs, outs)]
    operands = list(zip(xs, gammas, repeat(table), repeat(positions), outs))
    if plan is None:
        plan = _keep(key, _Plan(xs, [norm_rope_task(*o, eps=eps, pairs=pairs) for o in operands], operands))
    _run(plan, list(chain.from_iterable(operands)), given)
    return tuple(outs)


def _norm_rope_backward(douts, xs, gammas, table, positions, eps, pairs):
    eps, pairs = float(eps), bool(pairs)
    key = ("backward", eps, pairs, *map(_sig, (table, positions, *xs, *gammas, *douts)))
    plan = _plans.get(key)
    dxs, dgs, grads, sums = [], [], [], []
    for dout, x, gamma in zip(douts, xs, gammas):
        dx, dg, partial = _empty_like(x), None, None
        if gamma is not None:
            if x.numel() == 0:
                dg = torch.zeros_like(gamma)
            else:
                dg, partial = _empty_like(gamma), x.new_empty((x.shape[-1], _parts(x, len(xs))), dtype=torch.float32)
                sums.append((partial, dg))
        grads.append((x, gamma, table, positions, dx, dout, partial))
        dxs.append(dx)
        dgs.append(dg)
    if plan is None:                                        # (a sum is another operator than what it adds up, so a launch behind it)
        tasks = [norm_rope_grad_task(o[5], *o[:5], o[6], eps=eps, pairs=pairs) for o in grads] + [gamma_sum_task(*o) for o in sums]
        plan = _keep(key, _Plan([o[0] for o in grads + sums], tasks, grads + sums))
    _run(plan, list(chain.from_iterable(grads + sums)))
    return dxs, dgs


def _differentiable(xs, outs):
    if not torch.is_grad_enabled():
        return False
    for t in xs:
        if t is not None and t.requires_grad:
            break
    else:
        return False
    _need(all(o is None for o in outs), "out does not go with gradients")
    if forward_ad._current_level >= 0:                      # (the function itself is given them without their tangents)
        _no_tangent(xs)
    return True


def _no_gradient(what, *xs):
    if torch.is_grad_enabled():
        for t in xs:
            if t is not None and t.requires_grad:
                raise ValueError("%s has no gradient here" % what)


def norm_rope(x, gamma=None, table=None, positions=None, *, eps=1e-6, pairs=False, out=None):
    """Root-mean-square norm of every head of x [T, H, D] or [B, S, H, D] over D, times gamma [D], and the rotation of its
    first R elements by the angles of table [places, R] (cosines | sines, float32) at the tokens' positions (None: 0, 1, ...
    in every sequence); pairs: neighbours are rotated together, else the halves.  Differentiable in x and gamma."""
    _no_gradient("table", table)
    if _differentiable((x, gamma), (out,)):
        return _NormRope.apply(table, positions, eps, pairs, x, gamma)[0]
    _no_gradient("out", out)
    return _norm_rope((x,), (gamma,), table, positions, eps, pairs, (out,))[0]


def norm_rope_qk(q, k, gamma_q=None, gamma_k=None, table=None, positions=None, *, eps=1e-6, pairs=False, out=(None, None)):
    """norm_rope of queries and keys in one launch: (q', k')."""
    _no_gradient("table", table)
    if _differentiable((q, k, gamma_q, gamma_k), out):
        return _NormRope.apply(table, positions, eps, pairs, q, gamma_q, k, gamma_k)
    _no_gradient("out", *out)
    return _norm_rope((q, k), (gamma_q, gamma_k), table, positions, eps, pairs, out)


def norm_rope_backward(dout, x, gamma=None, table=None, positions=None, *, eps=1e-6, pairs=False):
    """Gradients of norm_rope for x and gamma (None without one).  Not differentiable themselves."""
    _no_gradient("norm_rope_backward", dout, x, gamma, table)
    (dx,), (dg,) = _norm_rope_backward((dout,), (x,), (gamma,), table, positions, eps, pairs)
    return dx, dg


def norm_rope_qk_backward(dq, dk, q, k, gamma_q=None, gamma_k=None, table=None, positions=None, *, eps=1e-6, pairs=False):
    """Gradients of norm_rope_qk for q, k, gamma_q and gamma_k, in two launches.  Not differentiable themselves."""
    _no_gradient("norm_rope_qk_backward", dq, dk, q, k, gamma_q, gamma_k, table)
    (gq, gk), (ggq, ggk) = _norm_rope_backward((dq, dk), (q, k), (gamma_q, gamma_k), table, positions, eps, pairs)
    return gq, gk, ggq, ggk


# ---- the cache -------------------------------------------------------------------------------------

def _store(xs, slots, caches, scales):
    _no_gradient("cache_store", *xs, *scales)
    given = (slots, *xs, *caches, *scales)
    key = ("store", *map(_sig, given))
    plan, n = _plans.get(key), len(xs)
    if plan is None:
        operands = list(zip(xs, repeat(slots), caches, scales))
        plan = _keep(key, _Plan(xs, [cache_store_task(*o) for o in operands], operands, [(1 + i, 0, 1 + n + i, 1 + 2 * n + i) for i in range(n)]))
    _run(plan, given, given[1 + n:])


def cache_store(x, slots, cache, scales):
    """Quantise rows of x [T, H, D] (or [B, S, H, D]) into slots (page index * page + place; negative: nowhere) of cache
    [pages, page, H, D] (int8 or float8_e4m3fn) and scales [pages, page, H, groups] (float32).  Slots are distinct.  Not
    differentiable: rows or scales that require a gradient are refused where gradients are recorded."""
    _store((x,), slots, (cache,), (scales,))


def cache_store_kv(k, v, slots, k_cache, k_scales, v_cache, v_scales):
    """cache_store of keys and values in one launch."""
    _store((k, v), slots, (k_cache, v_cache), (k_scales, v_scales))


def _load(caches, scales, pages, lengths, length, dtype, outs):
    length = int(length)
    _no_gradient("cache_load", *scales, *outs)
    given = (pages, lengths, *caches, *scales)
    key = ("load", length, dtype, *map(_sig, (*given, *outs)))
    plan, n = _plans.get(key), len(caches)
    if plan is None:
        _need(len(outs) == n, "out has %d entries (None: made here)", n)
        for c in caches:
            _check(c, "cache", _CACHE, (4,))
        _check(pages, "pages", _INT, (2,), None, caches[0].device)
        for c, o in zip(caches, outs):
            if o is not None:
                _check(o, "out", _FLOAT if dtype is None else (dtype,), None, (pages.shape[0], length, *c.shape[2:]), c.device)
    written, rows, dtype = [o for o in outs if o is not None], pages.shape[0], dtype or torch.float32
    outs = [c.new_empty((rows, length, *c.shape[2:]), dtype=dtype) if o is None else o for c, o in zip(caches, outs)]
    if plan is None:
        operands = list(zip(caches, scales, repeat(pages), repeat(lengths), outs))
        plan = _keep(key, _Plan(outs, [cache_load_task(*o) for o in operands], operands, [(2 + i, 2 + n + i, 0, 1, 2 + 2 * n + i) for i in range(n)]))
    _run(plan, (*given, *outs), written)
    return tuple(outs)


def cache_load(cache, scales, pages, lengths, length, *, dtype=None, out=None):
    """The first lengths[b] rows (None: all `length`) of every sequence b, through pages [B, width], as [B, length, H, D] of dtype
    (None: out's, without one float32); zeros behind them.  Not differentiable: scales that require a gradient are refused where gradients are recorded."""
    return _load((cache,), (scales,), pages, lengths, length, dtype, (out,))[0]


def cache_load_kv(k_cache, k_scales, v_cache, v_scales, pages, lengths, length, *, dtype=None, out=(None, None)):
    """cache_load of keys and values in one launch: (k, v)."""
    return _load((k_cache, v_cache), (k_scales, v_scales), pages, lengths, length, dtype, out)


# ---- logits ----------------------------------------------------------------------------------------

def penalize_logits(x, *, history=None, prompt_lengths=None, params=None, bias=None, allowed=None, out=None):
    """Penalties of the tokens in history [B, N] (entries that are no token count for nothing; the first prompt_lengths[b] for the
    repetition penalty only) by params [B, 3] = repetition, frequency, presence; bias; -inf where a bit of allowed is
    not set.  out may be x.  Not differentiable: logits that require a gradient are refused where gradients are recorded."""
    _no_gradient("penalize_logits", x, params, bias, out)
    key = ("penalty", *map(_sig, (x, history, prompt_lengths, params, bias, allowed, out)))
    plan = _plans.get(key)
    if plan is None:
        _check(x, "x", _FLOAT, (2,))
    given, out = () if out is None else (out,), _empty_like(x) if out is None else out
    operands = (x, out, history, prompt_lengths, params, bias, allowed)
    if plan is None:
        task = penalty_task(*operands)
        if history is not None and history.shape[1] == 0:   # (nothing is counted: as without one)
            operands = (x, out, None, None, None, bias, allowed)
        plan = _keep(key, _Plan((x,), (task,), (operands,)))
    _run(plan, operands, given)
    return out
