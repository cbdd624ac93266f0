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
from typing import NamedTuple

import torch

from ._binding import (SinkhornError, SkCombine, SkExperts, SkRouter, _dev, _on, _ptr, _stream, load_library)

_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
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


def _typed(t, name, allowed=tuple(_DTYPE)):
    """A contiguous GPU tensor of one of the element types the operators take."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype not in allowed:
        raise TypeError(f"{name} must be one of {[str(a) for a in allowed]}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _shape(t, shape, name):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _like(t, ref, name):
    if t.device != ref.device:
        raise ValueError(f"{name} must be on {ref.device}, got {t.device}")



def _call(fn, dev, stream, *args):
    """fn(*args, stream) on dev, whichever device is current."""
    if torch.cuda.current_device() == dev.index:
        st = fn(*args, _stream(dev, stream))
    else:
        with torch.cuda.device(dev):
            st = fn(*args, _stream(dev, stream))
    if st != 0:
        raise SinkhornError(st, fn.__name__)


def _counter(p, seed, offset):
    if not 0.0 <= p < 1.0:
        raise ValueError(f"p must be in [0, 1), got {p}")
    return ctypes.c_double(p), ctypes.c_uint64(int(seed) & _U64), ctypes.c_uint64(int(offset) & _U64)


# ---- router ----

def sinkhorn_route_forward(logits, k, bias=None, mask=None, renormalize=True, stream=None, workspace=None):
    """logits [T, E] float32, bfloat16 or float16; bias [E] float32; mask [T] bool (False: no token).
    Returns (Routing, state); state goes to sinkhorn_route_backward."""
    lib = load_library()
    _typed(logits, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits must be [T, E], got {list(logits.shape)}")
    T, E = logits.shape
    if bias is not None:
        _dev(bias, "bias"), _shape(bias, (E,), "bias"), _like(bias, logits, "bias")
    if mask is not None:
        _dev(mask, "mask", torch.bool), _shape(mask, (T,), "mask"), _like(mask, logits, "mask")
    r = SkRouter(T, E, int(k), _DTYPE[logits.dtype], int(bool(renormalize)))
    dev = logits.device
    need = int(lib.sinkhorn_route_workspace_bytes(ctypes.byref(r)))
    with _on(stream):
        n = T * max(int(k), 0)
        whole = torch.empty((3 * n + 2 * E + 1,), device=dev, dtype=torch.int32)
        real = torch.empty((n + 2 * T + 3,), device=dev, dtype=torch.float32)
        if need and (workspace is None or workspace.numel() < need):
            workspace = torch.empty((need,), device=dev, dtype=torch.uint8)
    experts, slots, tokens, counts, offsets = whole.split((n, n, n, E, E + 1))
    weights, state, balance, z = real.split((n, 2 * T + 1, 1, 1))
    _call(lib.sinkhorn_route_forward, dev, stream, ctypes.byref(r), _ptr(logits), _ptr(bias), _ptr(mask),
          _ptr(weights), _ptr(experts), _ptr(counts), _ptr(offsets), _ptr(tokens), _ptr(slots), _ptr(balance),
          _ptr(z), _ptr(state), _ptr(workspace) if need else None, ctypes.c_size_t(need))
    return Routing(weights.view(T, k), experts.view(T, k), counts, offsets, tokens, slots.view(T, k),
                   balance.view(()), z.view(())), state


def sinkhorn_route_backward(logits, k, weights, experts, counts, state, grad_weights=None, grad_balance=None,
                            grad_z=None, renormalize=True, stream=None):
    """Gradient of the logits from those of weights, balance and z_loss (each may be None)."""
    lib = load_library()
    _typed(logits, "logits")
    T, E = logits.shape
    for t, n, shape, typ in ((weights, "weights", (T, k), torch.float32), (experts, "experts", (T, k), torch.int32),
                             (counts, "counts", (E,), torch.int32), (state, "state", (2 * T + 1,), torch.float32),
                             (grad_weights, "grad_weights", (T, k), torch.float32),
                             (grad_balance, "grad_balance", (), torch.float32),
                             (grad_z, "grad_z", (), torch.float32)):
        if t is not None or n in ("weights", "experts", "counts", "state"):
            _dev(t, n, typ), _shape(t, shape, n), _like(t, logits, n)
    r = SkRouter(T, E, int(k), _DTYPE[logits.dtype], int(bool(renormalize)))
    with _on(stream):
        grad = torch.empty_like(logits)
    _call(lib.sinkhorn_route_backward, logits.device, stream, ctypes.byref(r), _ptr(logits), _ptr(weights),
          _ptr(experts), _ptr(counts), _ptr(state), _ptr(grad_weights), _ptr(grad_balance), _ptr(grad_z), _ptr(grad))
    return grad


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, bias, mask, renormalize):
        r, state = sinkhorn_route_forward(logits, k, bias, mask, renormalize)
        ctx.save_for_backward(logits, r.weights, r.experts, r.counts, state)
        ctx.k, ctx.renormalize = k, renormalize
        ctx.mark_non_differentiable(r.experts, r.counts, r.offsets, r.tokens, r.slots)
        ctx.set_materialize_grads(False)
        return tuple(r)

    @staticmethod
    def backward(ctx, g_weights, _e, _c, _o, _t, _s, g_balance, g_z):
        logits, weights, experts, counts, state = ctx.saved_tensors
        c = lambda g: None if g is None else g.contiguous()  # noqa: E731
        return sinkhorn_route_backward(logits, ctx.k, weights, experts, counts, state, c(g_weights), c(g_balance),
                                       c(g_z), ctx.renormalize), None, None, None, None


def sinkhorn_route(logits, k, bias=None, mask=None, renormalize=True) -> Routing:
    """The k experts of each token (first by logits + bias), their weights, the counts, the balance and z losses and
    the rows of each expert; weights, balance and z_loss are differentiable with respect to the logits.  The bias
    only chooses, and is a constant."""
    logits = logits.contiguous()
    bias = None if bias is None else bias.detach().contiguous()
    mask = None if mask is None else mask.contiguous()
    if torch.is_grad_enabled() and logits.requires_grad:
        return Routing(*_Route.apply(logits, k, bias, mask, renormalize))
    return sinkhorn_route_forward(logits, k, bias, mask, renormalize)[0]


# ---- experts' products ----

_HALF = (torch.bfloat16, torch.float16)


def _experts(rows, x_shape, w_shape, offsets, index, dtype, name):
    """The SkExperts of a call: rows = T k; index: slots [T, k], tokens [T k] or None."""
    E, N, K = w_shape
    T, k = (rows, 1) if x_shape is None else (x_shape[0], rows // max(x_shape[0], 1))
    if T * k != rows or (rows and k < 1):
        raise ValueError(f"{name}: {rows} rows are not a whole number for each of {T} tokens")
    return SkExperts(T, max(k, 1), E, K, N, _DTYPE[dtype])


def _product_args(w, offsets, *index):
    _typed(w, "weight", _HALF)
    if w.dim() != 3:
        raise ValueError(f"weight must be [E, N, K], got {list(w.shape)}")
    _dev(offsets, "offsets", torch.int32), _shape(offsets, (w.shape[0] + 1,), "offsets")
    _like(offsets, w, "offsets")
    for t, n in index:
        if t is not None:
            _dev(t, n, torch.int32), _like(t, w, n)


def _rows_2d(t, cols, ref, name):
    _typed(t, name, _HALF)
    if t.dim() != 2 or t.shape[1] != cols:
        raise ValueError(f"{name} must have {cols} columns, got {list(t.shape)}")
    if t.dtype != ref.dtype:
        raise TypeError(f"{name} must be {ref.dtype} as the weight, got {t.dtype}")
    _like(t, ref, name)


def sinkhorn_experts_forward(x, weight, offsets, tokens=None, stream=None):
    """Rows of each expert times its matrix: y [R, N].  x [T, K] gathered through tokens [R], or, without tokens,
    x [R, K] in the rows' order; weight [E, N, K]; offsets [E + 1]."""
    lib = load_library()
    _product_args(weight, offsets, (tokens, "tokens"))
    E, N, K = weight.shape
    _rows_2d(x, K, weight, "x")
    rows = x.shape[0] if tokens is None else tokens.numel()
    p = _experts(rows, None if tokens is None else x.shape, weight.shape, offsets, tokens, x.dtype, "tokens")
    with _on(stream):
        y = torch.empty((rows, N), device=x.device, dtype=x.dtype)
    _call(lib.sinkhorn_experts_forward, x.device, stream, ctypes.byref(p), _ptr(x), _ptr(weight), _ptr(offsets),
          _ptr(tokens), _ptr(y))
    return y


def sinkhorn_experts_backward_input(grad_y, weight, offsets, slots=None, stream=None, workspace=None):
    """Gradient of x: [T, K] with slots [T, k], else that of the rows, [R, K]."""
    lib = load_library()
    _product_args(weight, offsets, (slots, "slots"))
    E, N, K = weight.shape
    _rows_2d(grad_y, N, weight, "grad_y")
    rows = grad_y.shape[0]
    if slots is not None and (slots.dim() != 2 or slots.numel() != rows):
        raise ValueError(f"slots must be [T, k] with T k = {rows}, got {list(slots.shape)}")
    p = _experts(rows, None if slots is None else slots.shape, weight.shape, offsets, slots, grad_y.dtype, "slots")
    need = int(lib.sinkhorn_experts_workspace_bytes(ctypes.byref(p))) if slots is not None else 0
    with _on(stream):
        gx = torch.empty((p.T, K), device=grad_y.device, dtype=grad_y.dtype)
        if need and (workspace is None or workspace.numel() < need):
            workspace = torch.empty((need,), device=grad_y.device, dtype=torch.uint8)
    _call(lib.sinkhorn_experts_backward_input, grad_y.device, stream, ctypes.byref(p), _ptr(grad_y), _ptr(weight),
          _ptr(offsets), _ptr(slots), _ptr(gx), _ptr(workspace) if need else None, ctypes.c_size_t(need))
    return gx


def sinkhorn_experts_backward_weight(grad_y, x, offsets, tokens=None, stream=None):
    """Gradient of the weight, [E, N, K]."""
    lib = load_library()
    _typed(grad_y, "grad_y", _HALF), _typed(x, "x", _HALF)
    if grad_y.dim() != 2 or x.dim() != 2:
        raise ValueError("grad_y must be [R, N] and x [T, K] or [R, K]")
    N, K = grad_y.shape[1], x.shape[1]
    _dev(offsets, "offsets", torch.int32), _like(offsets, x, "offsets")
    _rows_2d(grad_y, N, x, "grad_y")
    rows = grad_y.shape[0]
    E = offsets.numel() - 1
    if tokens is not None:
        _dev(tokens, "tokens", torch.int32), _shape(tokens, (rows,), "tokens"), _like(tokens, x, "tokens")
    elif x.shape[0] != rows:
        raise ValueError(f"without tokens x must have {rows} rows as grad_y, got {x.shape[0]}")
    p = _experts(rows, None if tokens is None else x.shape, (E, N, K), offsets, tokens, x.dtype, "tokens")
    with _on(stream):
        gw = torch.empty((E, N, K), device=x.device, dtype=x.dtype)
    _call(lib.sinkhorn_experts_backward_weight, x.device, stream, ctypes.byref(p), _ptr(grad_y), _ptr(x),
          _ptr(offsets), _ptr(tokens), _ptr(gw))
    return gw


class _ExpertProduct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, offsets, tokens, slots):
        ctx.save_for_backward(x, weight, offsets, tokens, slots)
        return sinkhorn_experts_forward(x, weight, offsets, tokens)

    @staticmethod
    def backward(ctx, gy):
        x, weight, offsets, tokens, slots = ctx.saved_tensors
        gy = gy.contiguous()
        gx = sinkhorn_experts_backward_input(gy, weight, offsets, slots) if ctx.needs_input_grad[0] else None
        gw = sinkhorn_experts_backward_weight(gy, x, offsets, tokens) if ctx.needs_input_grad[1] else None
        return gx, gw, None, None, None


def sinkhorn_expert_product(x, weight, offsets, tokens=None, slots=None):
    """Each expert's rows times its matrix, [R, N]; differentiable with respect to x and weight [E, N, K].

    With tokens [R] and slots [T, k] of a Routing, x is [T, K] and its rows are gathered; without both, x is [R, K],
    in the rows' order.  Rows from offsets[E] on are zero."""
    if (tokens is None) != (slots is None):
        raise ValueError("tokens and slots go together")
    x, weight = x.contiguous(), weight.contiguous()
    if slots is not None:
        if slots.dim() != 2 or slots.shape[0] != x.shape[0] or slots.numel() != tokens.numel():
            raise ValueError(f"slots must be [T, k] with T = {x.shape[0]}, T k = {tokens.numel()}, "
                             f"got {list(slots.shape)}")
    if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad):
        return _ExpertProduct.apply(x, weight, offsets, tokens, slots)
    return sinkhorn_experts_forward(x, weight, offsets, tokens)


# ---- dropout ----

def _dropout(x, p, seed, offset, residual, stream=None):
    lib = load_library()
    _typed(x, "x")
    if residual is not None:
        _typed(residual, "residual", (x.dtype,)), _shape(residual, x.shape, "residual")
        _like(residual, x, "residual")
    args = _counter(p, seed, offset)
    with _on(stream):
        y = torch.empty_like(x)
    _call(lib.sinkhorn_dropout, x.device, stream, x.numel(), _DTYPE[x.dtype], _ptr(x), _ptr(residual), _ptr(y), *args)
    return y


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, offset):
        ctx.p, ctx.seed, ctx.offset = p, seed, offset
        return _dropout(x, p, seed, offset, residual)

    @staticmethod
    def backward(ctx, gy):
        gx = _dropout(gy.contiguous(), ctx.p, ctx.seed, ctx.offset, None) if ctx.needs_input_grad[0] else None
        return gx, gy if ctx.needs_input_grad[1] else None, None, None, None


def sinkhorn_dropout(x, p, seed, offset=0, residual=None, stream=None):
    """residual + dropout(x), differentiable with respect to x and residual.  An element is dropped with probability
    p (to 16 bits) by a generator keyed with seed (64 bits) and counted by offset (64 bits) and the element's number
    in x, so the mask is never stored: the same seed and offset drop the same elements.  A dropped element adds
    nothing, whatever it holds."""
    x = x.contiguous()
    residual = None if residual is None else residual.contiguous()
    if torch.is_grad_enabled() and (x.requires_grad or (residual is not None and residual.requires_grad)):
        if stream is not None:
            raise ValueError("a differentiable call runs on the current stream")
        return _Dropout.apply(x, residual, p, seed, offset)
    return _dropout(x, p, seed, offset, residual, stream)


# ---- combination of expert rows ----

def _combine_args(z, weights, slots):
    _typed(z, "z")
    _dev(slots, "slots", torch.int32), _like(slots, z, "slots")
    if z.dim() != 2 or slots.dim() != 2 or z.shape[0] != slots.numel():
        raise ValueError(f"z must be [T k, D] and slots [T, k], got {list(z.shape)} {list(slots.shape)}")
    _dev(weights, "weights"), _shape(weights, slots.shape, "weights"), _like(weights, z, "weights")
    T, k = slots.shape
    return SkCombine(T, z.shape[1], max(k, 1) if T == 0 else k, _DTYPE[z.dtype])


def sinkhorn_combine_forward(z, weights, slots, residual=None, p=0.0, seed=0, offset=0, stream=None):
    """y [T, D] = residual + dropout(sum_s weights[t, s] z[slots[t, s]])."""
    lib = load_library()
    c = _combine_args(z, weights, slots)
    args = _counter(p, seed, offset)
    if residual is not None:
        _typed(residual, "residual", (z.dtype,)), _shape(residual, (c.T, c.D), "residual")
        _like(residual, z, "residual")
    with _on(stream):
        y = torch.empty((c.T, c.D), device=z.device, dtype=z.dtype)
    _call(lib.sinkhorn_combine_forward, z.device, stream, ctypes.byref(c), _ptr(z), _ptr(weights), _ptr(slots),
          _ptr(residual), _ptr(y), *args)
    return y


def sinkhorn_combine_backward(z, weights, slots, offsets, grad_y, p=0.0, seed=0, offset=0, stream=None):
    """(grad_z [T k, D], grad_weights [T, k]); offsets as from the router (its last entry: the rows in use)."""
    lib = load_library()
    c = _combine_args(z, weights, slots)
    args = _counter(p, seed, offset)
    _typed(grad_y, "grad_y", (z.dtype,)), _shape(grad_y, (c.T, c.D), "grad_y"), _like(grad_y, z, "grad_y")
    _dev(offsets, "offsets", torch.int32), _like(offsets, z, "offsets")
    with _on(stream):
        gz = torch.empty_like(z)
        gw = torch.empty_like(weights)
    used = ctypes.c_void_p(offsets.data_ptr() + 4 * (offsets.numel() - 1))
    _call(lib.sinkhorn_combine_backward, z.device, stream, ctypes.byref(c), _ptr(z), _ptr(weights), _ptr(slots), used,
          _ptr(grad_y), _ptr(gz), _ptr(gw), *args)
    return gz, gw


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, z, weights, slots, offsets, residual, p, seed, offset):
        ctx.save_for_backward(z, weights, slots, offsets)
        ctx.drop = (p, seed, offset)
        return sinkhorn_combine_forward(z, weights, slots, residual, p, seed, offset)

    @staticmethod
    def backward(ctx, gy):
        z, weights, slots, offsets = ctx.saved_tensors
        gz = gw = None
        if ctx.needs_input_grad[0] or ctx.needs_input_grad[1]:
            gz, gw = sinkhorn_combine_backward(z, weights, slots, offsets, gy.contiguous(), *ctx.drop)
        return gz, gw, None, None, gy if ctx.needs_input_grad[4] else None, None, None, None


def sinkhorn_expert_combine(z, weights, slots, offsets, residual=None, p=0.0, seed=0, offset=0):
    """residual + dropout(weighted sum of each token's expert rows), [T, D]; differentiable with respect to z
    [T k, D], weights [T, k] and residual.  slots and offsets are a Routing's; p, seed and offset as in
    sinkhorn_dropout, over the elements of the result."""
    z, weights = z.contiguous(), weights.contiguous()
    residual = None if residual is None else residual.contiguous()
    if torch.is_grad_enabled() and (z.requires_grad or weights.requires_grad or
                                    (residual is not None and residual.requires_grad)):
        return _Combine.apply(z, weights, slots, offsets, residual, p, seed, offset)
    return sinkhorn_combine_forward(z, weights, slots, residual, p, seed, offset)
