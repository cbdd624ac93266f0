"""Rows in 8 bits: packing, the experts' products of packed rows for serving, and activations and products that keep
their rows in 8 bits for the backward pass.  Marshalling and autograd wrappers of the C ABI; every step runs in the HIP
library.

    w8 = sk.sinkhorn_pack(w)                                      # once; w [E, N, K]
    h = sk.sinkhorn_expert_product_packed(x, w8, r.offsets, r.tokens)

    h = sk.sinkhorn_expert_product_kept(x, w1, r.offsets, r.tokens, r.slots)          # in training
    z = sk.sinkhorn_expert_product_kept(h, w2, r.offsets, activation="silu", gated=True)
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple

import torch

from ._binding import SinkhornError, SkPacking, _dev, _int32, load_library
from .routed import (_call, _DTYPE, _experts, _experts_sizes, _first_order, _match, _on_stream, _ptr, _recorded,
                     _rows_in_order, _rows_of, _run_experts, _run_experts_input, _run_experts_weight, _typed)

KEPT_BLOCK = 128  # columns under one scale of a kept row
_ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


class Packed(NamedTuple):
    """Rows in 8 bits: row r of `columns` is scales[r] times values[r, :columns] (block = 0), or each `block` columns of
    it a scale of their own times their values."""
    values: torch.Tensor  # [..., P] int8, P = columns up to whole 16, zeros past the columns
    scales: torch.Tensor  # [...] float32, or [..., ceil(columns / block)]
    columns: int
    block: int = 0


@functools.lru_cache(maxsize=1024)
def _packing(rows, columns, block, dtype):
    if not 0 <= rows < 1 << 62:
        raise SinkhornError(-2, f"{rows} rows")
    return ctypes.byref(SkPacking(rows, *_int32(columns), block, dtype))


def _pitch(columns):
    return (columns + 15) // 16 * 16


def _row_count(shape):
    n = 1
    for s in shape:
        n *= s
    return n


def _block(block):
    if block not in (0, KEPT_BLOCK):
        raise ValueError(f"block must be 0 (a scale a row) or {KEPT_BLOCK}, got {block}")
    return int(block)


def _scales_shape(lead, columns, block):
    return (*lead, (columns + block - 1) // block) if block else tuple(lead)


def _new_packed(x, block):
    *lead, columns = x.shape
    return Packed(torch.empty((*lead, _pitch(columns)), device=x.device, dtype=torch.int8),
                  torch.empty(_scales_shape(lead, columns, block), device=x.device, dtype=torch.float32), columns,
                  block)


def _columns(x, name):
    _typed(x, name)
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"{name} must be [..., columns], got {list(x.shape)}")


def _check_packed(p, name, block=None):
    """A Packed of the shapes that its columns and block say; gives the shape of its values."""
    if not isinstance(p, Packed):
        raise TypeError(f"{name} must be a Packed")
    values, scales, columns, own = p
    _block(own)
    if block is not None and own != block:
        raise ValueError(f"{name} must have a scale for {block or 'each row'}, got block = {own}")
    _dev(values, f"{name}.values", torch.int8)
    shape = values.shape
    if len(shape) < 1 or columns < 1 or shape[-1] != _pitch(columns):
        raise ValueError(f"{name}.values must be [..., {_pitch(columns)}] for {columns} columns, got {list(shape)}")
    if values.data_ptr() % 16:
        raise ValueError(f"{name}.values must be aligned to 16 bytes")
    _match(scales, f"{name}.scales", values, _scales_shape(shape[:-1], columns, own), torch.float32)
    return shape


def _run_pack(x, block):
    p = _new_packed(x, block)
    _call(load_library().sinkhorn_pack, x.device,
          _packing(_row_count(x.shape[:-1]), p.columns, block, _DTYPE[x.dtype]), x.data_ptr(), p.values.data_ptr(),
          p.scales.data_ptr())
    return p


class _Constant(torch.autograd.Function):
    """A call without a gradient: its result counts as computed from the inputs, and who differentiates it gets an
    error, not a gradient without this path's part."""

    @staticmethod
    def forward(ctx, call, name, *inputs):
        ctx.name = name
        return call(*inputs)

    @staticmethod
    def backward(ctx, *grads):
        raise NotImplementedError(f"{ctx.name} has no gradient")


@_on_stream
def sinkhorn_pack(x, block=0) -> Packed:
    """Rows of x [..., columns] in 8 bits (see Packed and include/sinkhorn.h): a scale for each row, or for each 128
    columns of a row (block = 128).  float32, bfloat16 or float16.  No gradient.  stream=: as in sinkhorn_forward."""
    x = x.detach().contiguous()
    _columns(x, "x")
    return _run_pack(x, _block(block))


def _run_unpack(p, dtype):
    lead = p.values.shape[:-1]
    y = torch.empty((*lead, p.columns), device=p.values.device, dtype=dtype)
    _call(load_library().sinkhorn_unpack, y.device, _packing(_row_count(lead), p.columns, p.block, _DTYPE[dtype]),
          p.values.data_ptr(), p.scales.data_ptr(), y.data_ptr())
    return y


@_on_stream
def sinkhorn_unpack(packed, dtype=torch.float32):
    """The values that packed rows stand for, [..., columns], rounded to dtype.  No gradient."""
    _check_packed(packed, "packed")
    if dtype not in _DTYPE:
        raise TypeError(f"dtype must be one of {[str(d) for d in _DTYPE]}, got {dtype}")
    return _run_unpack(packed, dtype)


# ---- products of rows in 8 bits ----

@_on_stream
def sinkhorn_expert_product_packed(x, weight, offsets=None, tokens=None, dtype=None):
    """Each expert's rows times its matrix in 8-bit whole numbers, [R, N]: with a scale for each row of x and each of
    the weight's output channels.

    x [T, K] in 16 or 32 bits, which the call packs, or a Packed of it; weight a Packed of [E, N, K]; with tokens [R] of
    a Routing the rows are gathered, without them x is [R, K] in the rows' order.  Rows from offsets[E] on are zero.
    Without offsets the weight is a Packed of [N, K] (or [1, N, K]) and every row is multiplied by it.  The sums are
    exact; dtype is the result's (float32, bfloat16 or float16; default: x's, bfloat16 for a Packed).  For serving: it
    has no gradient, and asking for one raises.  stream=: as in sinkhorn_forward."""
    shape = _check_packed(weight, "weight", 0)
    if len(shape) == 2 and offsets is None:
        shape = (1, *shape)
    if len(shape) != 3 or (offsets is None and shape[0] != 1):
        raise ValueError(f"weight must be packed from [E, N, K] (without offsets from [N, K]), got values "
                         f"{list(weight.values.shape)}")
    E, N, K = shape[0], shape[1], weight.columns
    if isinstance(x, Packed):
        rows, given, default = x.values, x.scales, torch.bfloat16
        lead = _check_packed(x, "x", 0)[:-1]
        columns = x.columns
    else:
        rows = given = x = x.contiguous()
        default = _typed(x, "x").dtype
        *lead, columns = x.shape if x.dim() else (0,)
    if len(lead) != 1 or columns != K:
        raise ValueError(f"x must have rows of {K} columns, got {[*lead, columns]}")
    _match(weight.values, "weight", rows)
    dtype = default if dtype is None else dtype
    if dtype not in _DTYPE:
        raise TypeError(f"dtype must be one of {[str(d) for d in _DTYPE]}, got {dtype}")
    if offsets is not None:
        _match(offsets, "offsets", rows, (E + 1,), torch.int32)
    T = lead[0]
    if tokens is None:
        T, k = _rows_in_order(T)
    else:
        if offsets is None:
            raise ValueError("tokens go with offsets")
        _match(tokens, "tokens", rows, None, torch.int32)
        k = _rows_of(tokens.numel(), T, "tokens")
    call = x, weight, offsets, tokens, lead[0], (T, k, E, K, N, _DTYPE[dtype]), dtype
    if _recorded(given, weight.scales):
        return _Constant.apply(functools.partial(_run_packed_product, *call), "sinkhorn_expert_product_packed", given,
                               weight.scales)
    return _run_packed_product(*call)


def _run_packed_product(x, weight, offsets, tokens, rows, sizes, dtype, *_):
    dev, lib = weight.values.device, load_library()
    if isinstance(x, Packed):
        values, scales = x.values.data_ptr(), x.scales.data_ptr()
    else:  # the scales behind the values
        wide = _pitch(x.shape[1])
        space = torch.empty((rows * (wide + 4),), device=dev, dtype=torch.int8)
        values = space.data_ptr()
        scales = values + rows * wide
        _call(lib.sinkhorn_pack, dev, _packing(rows, x.shape[1], 0, _DTYPE[x.dtype]), x.data_ptr(), values, scales)
    y = torch.empty((sizes[0] * sizes[1], sizes[4]), device=dev, dtype=dtype)
    _call(lib.sinkhorn_experts_forward_packed, dev, _experts(*sizes)[0], values, scales, weight.values.data_ptr(),
          weight.scales.data_ptr(), _ptr(offsets), _ptr(tokens), y.data_ptr())
    return y


# ---- activations, and products that keep their rows in 8 bits ----

def _kind(activation, gated, columns):
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {list(_ACTIVATIONS)}, got {activation!r}")
    if gated and columns % 2:
        raise ValueError(f"a gated activation takes an even number of columns, got {columns}")
    return _ACTIVATIONS[activation], int(bool(gated))


def _run_activation(x, kind, gated, keep):
    """(activated rows, Packed of x or None)."""
    *lead, columns = x.shape
    y = torch.empty((*lead, columns // 2 if gated else columns), device=x.device, dtype=x.dtype)
    p = _new_packed(x, KEPT_BLOCK) if keep else None
    _call(load_library().sinkhorn_activation_forward, x.device,
          _packing(_row_count(lead), columns, KEPT_BLOCK, _DTYPE[x.dtype]), kind, gated, x.data_ptr(), y.data_ptr(),
          _ptr(p and p.values), _ptr(p and p.scales))
    return y, p


def _run_activation_backward(p, kind, gated, dtype, gy, wants_y):
    """(activated rows again or None, gradient of x or None)."""
    *lead, _ = p.values.shape
    made = {"device": p.values.device, "dtype": dtype}
    y = torch.empty((*lead, p.columns // 2 if gated else p.columns), **made) if wants_y else None
    gx = torch.empty((*lead, p.columns), **made) if gy is not None else None
    _call(load_library().sinkhorn_activation_backward, p.values.device,
          _packing(_row_count(lead), p.columns, KEPT_BLOCK, _DTYPE[dtype]), kind, gated, p.values.data_ptr(),
          p.scales.data_ptr(), _ptr(gy), _ptr(y), _ptr(gx))
    return y, gx


class _Activation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, kind, gated):
        y, p = _run_activation(x, kind, gated, True)
        ctx.save_for_backward(p.values, p.scales)
        ctx.call = kind, gated, x.dtype, p.columns
        return y

    @staticmethod
    @_first_order
    def backward(ctx, gy):
        kind, gated, dtype, columns = ctx.call
        p = Packed(*ctx.saved_tensors, columns, KEPT_BLOCK)
        return _run_activation_backward(p, kind, gated, dtype, gy.contiguous(), False)[1], None, None


def sinkhorn_activation(x, activation, gated=False):
    """act(x), or with gated act(x[..., :K]) x[..., K:] of the two halves of the columns; act is "none", "relu", "silu"
    or "gelu" (by the error function).  Differentiable with respect to x, which is kept in 8 bits with a scale for each
    128 columns of a row: the derivative is taken at those values.  float32, bfloat16 or float16, in 32 bits."""
    x = x.contiguous()
    _columns(x, "x")
    kind, gated = _kind(activation, gated, x.shape[-1])
    if _recorded(x):
        return _Activation.apply(x, kind, gated)
    return _run_activation(x, kind, gated, False)[0]


class _KeptProduct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, offsets, tokens, slots, kind, gated, sizes):
        plain = not kind and not gated
        if not ctx.needs_input_grad[1] and plain:
            a, p = x, None  # the gradient of x needs the weight alone
        elif plain:
            a, p = x, _run_pack(x, KEPT_BLOCK)
        else:
            a, p = _run_activation(x, kind, gated, True)
        ctx.save_for_backward(weight, offsets, tokens, slots, p and p.values, p and p.scales)
        ctx.call = kind, gated, x.shape[1], x.dtype, sizes
        return _run_experts(a, weight, offsets, tokens, sizes)

    @staticmethod
    @_first_order
    def backward(ctx, gy):
        weight, offsets, tokens, slots, values, scales = ctx.saved_tensors
        kind, gated, columns, dtype, sizes = ctx.call
        gy, need_x, need_w = gy.contiguous(), *ctx.needs_input_grad[:2]
        p = None if values is None else Packed(values, scales, columns, KEPT_BLOCK)
        gx = _run_experts_input(gy, weight, offsets, slots, sizes) if need_x else None
        a = gw = None
        if kind or gated:
            a, gx = _run_activation_backward(p, kind, gated, dtype, gx, need_w)
        elif need_w:
            a = _run_unpack(p, dtype)
        if need_w:
            gw = _run_experts_weight(gy, a, offsets, tokens, sizes)
        return gx, gw, None, None, None, None, None, None


def sinkhorn_expert_product_kept(x, weight, offsets, tokens=None, slots=None, activation="none", gated=False):
    """As sinkhorn_expert_product, of the activated rows act(x) (as sinkhorn_activation; x has 2 K columns where gated),
    with x kept in 8 bits for the backward pass instead of 16, a scale for each 128 columns of a row; the activated rows
    are not kept.  The result is of x as given; the gradients take x at the values kept, activated again and rounded to
    x's type."""
    if (tokens is None) != (slots is None):
        raise ValueError("tokens and slots go together")
    x, weight = x.contiguous(), weight.contiguous()
    _columns(x, "x")
    kind, gated = _kind(activation, gated, x.shape[-1])
    sizes = _experts_sizes(x, weight, offsets, tokens, 1 + gated)
    if slots is not None:
        T, k = sizes[:2]
        _match(slots, "slots", x, (T, k) if T else (0, *slots.shape[1:2]), torch.int32)
    if _recorded(x, weight):
        return _KeptProduct.apply(x, weight, offsets, tokens, slots, kind, gated, sizes)
    a = _run_activation(x, kind, gated, False)[0] if kind or gated else x
    return _run_experts(a, weight, offsets, tokens, sizes)
