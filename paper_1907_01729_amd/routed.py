"""Routed layers: the router with its balance loss, the experts' products, dropout and the combination of expert
rows.  Marshalling and autograd wrappers of the C ABI; every step runs in the HIP library.

With C = -logits and uniform masses, ``lam * beta`` of ``sinkhorn_forward`` is the per-expert offset under which
tokens spread evenly over the experts; it goes into ``sinkhorn_route`` as ``bias``:

    out = sk.sinkhorn_forward(mu, nu, -logits, lam, n_iter)        # mu [1, T], nu [1, E]
    r = sk.sinkhorn_route(logits, k, bias=lam * out["beta"][0])
    h = sk.sinkhorn_expert_product(x, w, r.offsets, r.tokens, r.slots)
    y = sk.sinkhorn_expert_combine(h, r.weights, r.slots, r.offsets, residual=x, p=0.1, seed=seed)
    loss = loss + 0.01 * r.balance
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from ._binding import SinkhornError, SkCombine, SkExperts, SkRouter, _dev, _int32, _scratch, load_library

_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_HALF = {torch.bfloat16: 1, torch.float16: 2}
_U64 = (1 << 64) - 1


class Routing(NamedTuple):
    """What sinkhorn_route gives: see include/sinkhorn.h for each."""
    weights: torch.Tensor  # [T, k] float32, differentiable
    experts: torch.Tensor  # [T, k] int32, -1: none
    counts: torch.Tensor   # [E] int32
    offsets: torch.Tensor  # [E + 1] int32
    tokens: torch.Tensor   # [T k] int32, -1: row of no expert
    slots: torch.Tensor    # [T, k] int32, -1: none
    balance: torch.Tensor  # [] float32, differentiable
    z_loss: torch.Tensor   # [] float32, differentiable


# ---- checks and calls ----

def _typed(t, name, allowed=_DTYPE):
    """A contiguous GPU tensor of one of the element types the operators take."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype not in allowed:
        raise TypeError(f"{name} must be one of {[str(a) for a in allowed]}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _match(t, name, ref, shape=None, dtype=None):
    """A contiguous GPU tensor on ref's device, of the dtype and shape given."""
    if dtype is not None:
        _dev(t, name, dtype)
    if t.device != ref.device:
        raise ValueError(f"{name} must be on {ref.device}, got {t.device}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


# The current stream's handle.  The public property builds a Stream object for it, which takes twenty times as long.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _call(fn, dev, *args):
    """fn(*args, stream): on dev's current stream, whichever device is current."""
    index = dev.index
    if torch.cuda.current_device() == index:
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status != 0:
        raise SinkhornError(status, fn.__name__)


def _forward_mode():
    """Within a level of forward-mode differentiation.  Asked instead of every input's tangent, which takes a third of
    a microsecond each."""
    return getattr(forward_ad, "_current_level", 0) >= 0


def _recorded(*inputs):
    """Whether a call goes through autograd: where a gradient of an input is wanted, and in forward mode, where autograd
    refuses an input with a tangent (the operators have no such derivative, and a result without one would pass for
    zero), and within torch.jit.trace, which keeps an autograd function, but of a call past it the allocations alone.  A
    call that goes past it saves ten microseconds."""
    if _forward_mode() or torch._C._is_tracing():
        return True
    if torch.is_grad_enabled():
        for t in inputs:
            if t is not None and t.requires_grad:
                return True
    return False


def _first_order(fn):
    """A backward pass that has no derivative itself: who asks for one gets an error, in forward mode too.  Only where a
    graph is built for it, since the wrapper takes ten microseconds of a backward pass."""
    refuses = once_differentiable(fn)

    @functools.wraps(fn)
    def backward(ctx, *grads):
        if _forward_mode() and any(g is not None and forward_ad.unpack_dual(g).tangent is not None for g in grads):
            raise NotImplementedError("routed layers: the gradients have no derivative in forward mode AD")
        return refuses(ctx, *grads) if torch.is_grad_enabled() else fn(ctx, *grads)
    return backward


def _on_stream(fn):
    """Gives fn a keyword argument stream: the call, its outputs and its workspace on that stream."""
    @functools.wraps(fn)
    def call(*args, stream=None, **kwargs):
        if stream is None:
            return fn(*args, **kwargs)
        with torch.cuda.stream(stream):
            return fn(*args, **kwargs)
    return call


# A call's sizes as the library takes them, and the bytes of workspace they need: functions of the sizes alone.
@functools.lru_cache(maxsize=1024)
def _router(T, E, k, dtype, renormalize):
    r = SkRouter(*_int32(T, E, k), dtype, renormalize)
    return ctypes.byref(r), int(load_library().sinkhorn_route_workspace_bytes(ctypes.byref(r)))


@functools.lru_cache(maxsize=1024)
def _experts(T, k, E, K, N, dtype):
    p = SkExperts(*_int32(T, k, E, K, N), dtype)
    lib, ref = load_library(), ctypes.byref(p)
    return ref, int(lib.sinkhorn_experts_workspace_bytes(ref)), int(lib.sinkhorn_experts_weight_workspace_bytes(ref))


@functools.lru_cache(maxsize=1024)
def _combine(T, D, k, dtype):
    return ctypes.byref(SkCombine(*_int32(T, D, k), dtype))


def _workspace(workspace, need, dev):
    """As _scratch, and nothing where nothing is needed or given."""
    return _scratch(workspace, need, dev) if need or workspace is not None else None


def _ptr(t):
    return None if t is None else t.data_ptr()


def _counter(p, seed, offset):
    if not 0.0 <= p < 1.0:
        raise ValueError(f"p must be in [0, 1), got {p}")
    return float(p), int(seed) & _U64, int(offset) & _U64


# ---- router ----

@_on_stream
def sinkhorn_route_forward(logits, k, bias=None, mask=None, renormalize=True, workspace=None):
    """logits [T, E] float32, bfloat16 or float16; bias [E] float32; mask [T] bool (False: no token).
    Returns (Routing, state); state goes to sinkhorn_route_backward.  stream=: as in sinkhorn_forward."""
    return _route_forward(logits, k, bias, mask, renormalize, True, workspace)


def _route_forward(logits, k, bias, mask, renormalize, with_state, workspace=None):
    _typed(logits, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits must be [T, E], got {list(logits.shape)}")
    T, E = logits.shape
    k = int(k)
    if bias is not None:
        _match(bias, "bias", logits, (E,), torch.float32)
    if mask is not None:
        _match(mask, "mask", logits, (T,), torch.bool)
    r, need = _router(T, E, k, _DTYPE[logits.dtype], int(bool(renormalize)))
    dev, n = logits.device, max(k, 0)
    whole, real = {"device": dev, "dtype": torch.int32}, {"device": dev, "dtype": torch.float32}
    weights, experts, slots = torch.empty((T, n), **real), torch.empty((T, n), **whole), torch.empty((T, n), **whole)
    tokens, counts, offsets = (torch.empty((T * n,), **whole), torch.empty((E,), **whole),
                               torch.empty((E + 1,), **whole))
    balance, z = torch.empty((), **real), torch.empty((), **real)
    state = torch.empty((2 * T + 1,), **real) if with_state else None
    scratch = _workspace(workspace, need, dev)
    _call(load_library().sinkhorn_route_forward, dev, r, logits.data_ptr(), _ptr(bias), _ptr(mask),
          weights.data_ptr(), experts.data_ptr(), counts.data_ptr(), offsets.data_ptr(), tokens.data_ptr(),
          slots.data_ptr(), balance.data_ptr(), z.data_ptr(), _ptr(state), _ptr(scratch), need)
    return Routing(weights, experts, counts, offsets, tokens, slots, balance, z), state


@_on_stream
def sinkhorn_route_backward(logits, k, weights, experts, counts, state, grad_weights=None, grad_balance=None,
                            grad_z=None, renormalize=True):
    """Gradient of the logits from those of weights, balance and z_loss (each may be None)."""
    _typed(logits, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits must be [T, E], got {list(logits.shape)}")
    T, E = logits.shape
    for t, n, shape, typ in ((weights, "weights", (T, k), torch.float32), (experts, "experts", (T, k), torch.int32),
                             (counts, "counts", (E,), torch.int32), (state, "state", (2 * T + 1,), torch.float32)):
        _match(t, n, logits, shape, typ)
    for t, n, shape in ((grad_weights, "grad_weights", (T, k)), (grad_balance, "grad_balance", ()),
                        (grad_z, "grad_z", ())):
        if t is not None:
            _match(t, n, logits, shape, torch.float32)
    return _route_backward(logits, int(k), weights, experts, counts, state, grad_weights, grad_balance, grad_z,
                           renormalize)


def _route_backward(logits, k, weights, experts, counts, state, grad_weights, grad_balance, grad_z, renormalize):
    T, E = logits.shape
    r, _ = _router(T, E, k, _DTYPE[logits.dtype], int(bool(renormalize)))
    grad = torch.empty_like(logits)
    _call(load_library().sinkhorn_route_backward, logits.device, r, logits.data_ptr(), weights.data_ptr(),
          experts.data_ptr(), counts.data_ptr(), state.data_ptr(), _ptr(grad_weights), _ptr(grad_balance),
          _ptr(grad_z), grad.data_ptr())
    return grad


def _contiguous(g):
    return None if g is None else g.contiguous()


def _saved(ctx):
    """The saved tensors, dense: hooks on them may give the same values back with other strides."""
    return map(_contiguous, ctx.saved_tensors)


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, bias, mask, renormalize):
        r, state = _route_forward(logits, k, bias, mask, renormalize, True)
        ctx.save_for_backward(logits, r.weights, r.experts, r.counts, state)
        ctx.k, ctx.renormalize = int(k), renormalize
        ctx.mark_non_differentiable(r.experts, r.counts, r.offsets, r.tokens, r.slots)
        ctx.set_materialize_grads(False)  # no zeros for outputs without a gradient
        return tuple(r)

    @staticmethod
    @_first_order
    def backward(ctx, g_weights, _e, _c, _o, _t, _s, g_balance, g_z):
        logits, weights, experts, counts, state = _saved(ctx)
        return _route_backward(logits, ctx.k, weights, experts, counts, state, _contiguous(g_weights),
                               _contiguous(g_balance), _contiguous(g_z), ctx.renormalize), None, None, None, None


def sinkhorn_route(logits, k, bias=None, mask=None, renormalize=True) -> Routing:
    """The k experts of each token (first by logits + bias), their weights, the counts, the balance and z losses and
    the rows of each expert; weights, balance and z_loss are differentiable with respect to the logits.  The bias
    only chooses, and is a constant."""
    logits = logits.contiguous()
    bias = None if bias is None else bias.detach().contiguous()
    mask = None if mask is None else mask.contiguous()
    if _recorded(logits):
        return Routing(*_Route.apply(logits, k, bias, mask, renormalize))
    return _route_forward(logits, k, bias, mask, renormalize, False)[0]


# ---- experts' products ----

def _rows_of(rows, T, name):
    """Pairs of a token, where `rows` rows belong to T tokens."""
    if T == 0:
        if rows:
            raise ValueError(f"{name}: {rows} rows of no token")
        return 1
    if rows % T or not rows:
        raise ValueError(f"{name}: {rows} rows are not a whole number for each of {T} tokens")
    return rows // T


def _rows_in_order(rows):
    """(T, k) for rows that are not gathered, where only T k counts: a token has up to 16 rows, so there are more of
    them than the library takes tokens."""
    for k in range(1, 17):
        if rows <= k << 24 and rows % k == 0:
            return rows // k, k
    return rows, 1  # the library refuses it


def _half_rows(t, name, cols, ref):
    _typed(t, name, _HALF)
    if t.dim() != 2 or t.shape[1] != cols:
        raise ValueError(f"{name} must have {cols} columns, got {list(t.shape)}")
    if t.dtype != ref.dtype:
        raise TypeError(f"{name} must be {ref.dtype}, got {t.dtype}")
    _match(t, name, ref)


def _weight(w):
    _typed(w, "weight", _HALF)
    if w.dim() != 3:
        raise ValueError(f"weight must be [E, N, K], got {list(w.shape)}")
    return w.shape


@_on_stream
def sinkhorn_experts_forward(x, weight, offsets, tokens=None):
    """Rows of each expert times its matrix: y [R, N].  x [T, K] gathered through tokens [R], or, without tokens,
    x [R, K] in the rows' order; weight [E, N, K]; offsets [E + 1]."""
    return _run_experts(x, weight, offsets, tokens, _experts_sizes(x, weight, offsets, tokens))


def _experts_sizes(x, weight, offsets, tokens):
    E, N, K = _weight(weight)
    _half_rows(x, "x", K, weight)
    _match(offsets, "offsets", x, (E + 1,), torch.int32)
    if tokens is None:
        T, k = _rows_in_order(x.shape[0])
    else:
        _match(tokens, "tokens", x, None, torch.int32)
        T = x.shape[0]
        k = _rows_of(tokens.numel(), T, "tokens")
    return *map(int, (T, k, E, K, N)), _HALF[x.dtype]  # torch.jit.trace gives out sizes as tensors


def _run_experts(x, weight, offsets, tokens, sizes):
    T, k, _, _, N, _ = sizes
    y = torch.empty((T * k, N), device=x.device, dtype=x.dtype)
    _call(load_library().sinkhorn_experts_forward, x.device, _experts(*sizes)[0], x.data_ptr(), weight.data_ptr(),
          offsets.data_ptr(), _ptr(tokens), y.data_ptr())
    return y


@_on_stream
def sinkhorn_experts_backward_input(grad_y, weight, offsets, slots=None, workspace=None):
    """Gradient of x: [T, K] with slots [T, k], else that of the rows, [R, K]."""
    E, N, K = _weight(weight)
    _half_rows(grad_y, "grad_y", N, weight)
    _match(offsets, "offsets", grad_y, (E + 1,), torch.int32)
    rows = grad_y.shape[0]
    if slots is None:
        T, k = _rows_in_order(rows)
    else:
        _match(slots, "slots", grad_y, None, torch.int32)
        if slots.dim() != 2 or slots.numel() != rows:
            raise ValueError(f"slots must be [T, k] with T k = {rows}, got {list(slots.shape)}")
        T = slots.shape[0]
        k = _rows_of(rows, T, "slots")
    return _run_experts_input(grad_y, weight, offsets, slots, (T, k, E, K, N, _HALF[grad_y.dtype]), workspace)


def _run_experts_input(grad_y, weight, offsets, slots, sizes, workspace=None):
    p, need, _ = _experts(*sizes)
    rows = grad_y.shape[0] if slots is None else sizes[0]
    gx = torch.empty((rows, sizes[3]), device=grad_y.device, dtype=grad_y.dtype)
    scratch = None if slots is None else _workspace(workspace, need, grad_y.device)
    _call(load_library().sinkhorn_experts_backward_input, grad_y.device, p, grad_y.data_ptr(), weight.data_ptr(),
          offsets.data_ptr(), _ptr(slots), gx.data_ptr(), _ptr(scratch), need)
    return gx


@_on_stream
def sinkhorn_experts_backward_weight(grad_y, x, offsets, tokens=None, workspace=None):
    """Gradient of the weight, [E, N, K]."""
    _typed(grad_y, "grad_y", _HALF)
    if grad_y.dim() != 2 or x.dim() != 2:
        raise ValueError("grad_y must be [R, N] and x [T, K] or [R, K]")
    (rows, N), (T, K) = grad_y.shape, x.shape
    _half_rows(x, "x", K, grad_y)
    _match(offsets, "offsets", x, None, torch.int32)
    E = offsets.numel() - 1
    if tokens is not None:
        _match(tokens, "tokens", x, (rows,), torch.int32)
        k = _rows_of(rows, T, "tokens")
    elif T != rows:
        raise ValueError(f"without tokens x must have {rows} rows as grad_y, got {T}")
    else:
        T, k = _rows_in_order(rows)
    return _run_experts_weight(grad_y, x, offsets, tokens, (T, k, E, K, N, _HALF[x.dtype]), workspace)


def _run_experts_weight(grad_y, x, offsets, tokens, sizes, workspace=None):
    _, _, E, K, N, _ = sizes
    p, _, need = _experts(*sizes)
    gw = torch.empty((E, N, K), device=x.device, dtype=x.dtype)
    scratch = _workspace(workspace, need, x.device)
    _call(load_library().sinkhorn_experts_backward_weight, x.device, p, grad_y.data_ptr(), x.data_ptr(),
          offsets.data_ptr(), _ptr(tokens), gw.data_ptr(), _ptr(scratch), need)
    return gw


class _ExpertProduct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, offsets, tokens, slots, sizes):
        ctx.save_for_backward(x, weight, offsets, tokens, slots)
        ctx.sizes = sizes
        return _run_experts(x, weight, offsets, tokens, sizes)

    @staticmethod
    @_first_order
    def backward(ctx, gy):
        x, weight, offsets, tokens, slots = _saved(ctx)
        gy, need_x, need_w = gy.contiguous(), *ctx.needs_input_grad[:2]
        gx = _run_experts_input(gy, weight, offsets, slots, ctx.sizes) if need_x else None
        gw = _run_experts_weight(gy, x, offsets, tokens, ctx.sizes) if need_w else None
        return gx, gw, None, None, None, None


def sinkhorn_expert_product(x, weight, offsets, tokens=None, slots=None):
    """Each expert's rows times its matrix, [R, N]; differentiable with respect to x and weight [E, N, K].

    With tokens [R] and slots [T, k] of a Routing, x is [T, K] and its rows are gathered; without both, x is [R, K],
    in the rows' order.  Rows from offsets[E] on are zero.  bfloat16 or float16, sums in 32 bits."""
    if (tokens is None) != (slots is None):
        raise ValueError("tokens and slots go together")
    x, weight = x.contiguous(), weight.contiguous()
    sizes = _experts_sizes(x, weight, offsets, tokens)
    if slots is not None:
        T, k = sizes[:2]
        _match(slots, "slots", x, (T, k) if T else (0, *slots.shape[1:2]), torch.int32)
    if _recorded(x, weight):
        return _ExpertProduct.apply(x, weight, offsets, tokens, slots, sizes)
    return _run_experts(x, weight, offsets, tokens, sizes)


# ---- dropout ----

def _run_dropout(x, residual, counter):
    y = torch.empty_like(x)
    _call(load_library().sinkhorn_dropout, x.device, x.numel(), _DTYPE[x.dtype], x.data_ptr(), _ptr(residual),
          y.data_ptr(), *counter)
    return y


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, counter):
        ctx.counter = counter
        return _run_dropout(x, residual, counter)

    @staticmethod
    @_first_order
    def backward(ctx, gy):
        gx = _run_dropout(gy.contiguous(), None, ctx.counter) if ctx.needs_input_grad[0] else None
        return gx, gy if ctx.needs_input_grad[1] else None, None


@_on_stream
def sinkhorn_dropout(x, p, seed, offset=0, residual=None):
    """residual + dropout(x), differentiable with respect to x and residual.  An element is dropped with probability
    p (to 16 bits) by a generator keyed with seed (64 bits) and counted by offset (64 bits) and the element's number
    in x, so the mask is never stored: the same seed and offset drop the same elements.  A dropped element adds
    nothing, whatever it holds."""
    x = x.contiguous()
    _typed(x, "x")
    if residual is not None:
        residual = residual.contiguous()
        _match(residual, "residual", x, x.shape, x.dtype)
    counter = _counter(p, seed, offset)
    if _recorded(x, residual):
        return _Dropout.apply(x, residual, counter)
    return _run_dropout(x, residual, counter)


# ---- combination of expert rows ----

def _combine_sizes(z, weights, slots):
    _typed(z, "z")
    _match(slots, "slots", z, None, torch.int32)
    if z.dim() != 2 or slots.dim() != 2 or z.shape[0] != slots.numel():
        raise ValueError(f"z must be [T k, D] and slots [T, k], got {list(z.shape)} {list(slots.shape)}")
    _match(weights, "weights", z, slots.shape, torch.float32)
    T, k = slots.shape
    return tuple(map(int, (T, z.shape[1], max(k, 1) if T == 0 else k)))


@_on_stream
def sinkhorn_combine_forward(z, weights, slots, residual=None, p=0.0, seed=0, offset=0):
    """y [T, D] = residual + dropout(sum_s weights[t, s] z[slots[t, s]])."""
    T, D, k = _combine_sizes(z, weights, slots)
    if residual is not None:
        _match(residual, "residual", z, (T, D), z.dtype)
    return _run_combine(z, weights, slots, residual, T, D, k, _counter(p, seed, offset))


def _run_combine(z, weights, slots, residual, T, D, k, counter):
    y = torch.empty((T, D), device=z.device, dtype=z.dtype)
    _call(load_library().sinkhorn_combine_forward, z.device, _combine(T, D, k, _DTYPE[z.dtype]), z.data_ptr(),
          weights.data_ptr(), slots.data_ptr(), _ptr(residual), y.data_ptr(), *counter)
    return y


@_on_stream
def sinkhorn_combine_backward(z, weights, slots, offsets, grad_y, p=0.0, seed=0, offset=0):
    """(grad_z [T k, D], grad_weights [T, k]); offsets as from the router (its last entry: the rows in use).  Rows that
    no slot names have no gradient."""
    T, D, k = _combine_sizes(z, weights, slots)
    _match(grad_y, "grad_y", z, (T, D), z.dtype)
    _used(offsets, z)
    return _run_combine_backward(z, weights, slots, offsets, grad_y, T, D, k, _counter(p, seed, offset))


def _used(offsets, z):
    _match(offsets, "offsets", z, None, torch.int32)
    if offsets.numel() < 1:
        raise ValueError("offsets must be [E + 1]")


def _run_combine_backward(z, weights, slots, offsets, grad_y, T, D, k, counter):
    gz, gw = torch.empty_like(z), torch.empty_like(weights)
    _call(load_library().sinkhorn_combine_backward, z.device, _combine(T, D, k, _DTYPE[z.dtype]), z.data_ptr(),
          weights.data_ptr(), slots.data_ptr(), offsets.data_ptr() + 4 * (offsets.numel() - 1), grad_y.data_ptr(),
          gz.data_ptr(), gw.data_ptr(), *counter)
    return gz, gw


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, z, weights, slots, offsets, residual, sizes, counter):
        ctx.save_for_backward(z, weights, slots, offsets)
        ctx.call = (*sizes, counter)
        return _run_combine(z, weights, slots, residual, *sizes, counter)

    @staticmethod
    @_first_order
    def backward(ctx, gy):
        z, weights, slots, offsets = _saved(ctx)
        gz = gw = None
        if ctx.needs_input_grad[0] or ctx.needs_input_grad[1]:
            gz, gw = _run_combine_backward(z, weights, slots, offsets, gy.contiguous(), *ctx.call)
        return gz, gw, None, None, gy if ctx.needs_input_grad[4] else None, None, None


def sinkhorn_expert_combine(z, weights, slots, offsets, residual=None, p=0.0, seed=0, offset=0):
    """residual + dropout(weighted sum of each token's expert rows), [T, D]; differentiable with respect to z
    [T k, D], weights [T, k] and residual.  slots and offsets are a Routing's, where a slot set to -1 leaves its pair
    out (a limit on an expert's rows); p, seed and offset as in sinkhorn_dropout, over the elements of the result."""
    z, weights = z.contiguous(), weights.contiguous()
    T, D, k = sizes = _combine_sizes(z, weights, slots)
    if residual is not None:
        residual = residual.contiguous()
        _match(residual, "residual", z, (T, D), z.dtype)
    counter = _counter(p, seed, offset)
    if _recorded(z, weights, residual):
        _used(offsets, z)
        return _Combine.apply(z, weights, slots, offsets, residual, sizes, counter)
    return _run_combine(z, weights, slots, residual, T, D, k, counter)
