"""Rows in 8 bits: packing, the experts' products of packed rows for serving, and activations and products that keep
their rows in 8 bits for the backward pass.  Every step runs in the HIP library, through its calls on torch tensors.

    w8 = sk.sinkhorn_pack(w)                                      # once; w [E, N, K]
    h = sk.sinkhorn_expert_product_packed(x, w8, r.offsets, r.tokens)

    h = sk.sinkhorn_expert_product_kept(x, w1, r.offsets, r.tokens, r.slots)          # in training
    z = sk.sinkhorn_expert_product_kept(h, w2, r.offsets, activation="silu", gated=True)
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from ._binding import load_torch_library
from .routed import _on_stream

_ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


class Packed(NamedTuple):
    """Rows in 8 bits: row r of `columns` is scales[r] times values[r, :columns] (block = 0), or each `block` columns of
    it a scale of their own times their values."""
    values: torch.Tensor  # [..., P] int8, P = columns up to whole 16, zeros past the columns
    scales: torch.Tensor  # [...] float32, or [..., ceil(columns / block)]
    columns: int
    block: int = 0


@_on_stream
def sinkhorn_pack(x, block=0) -> Packed:
    """Rows of x [..., columns] in 8 bits (see Packed and include/sinkhorn.h): a scale for each row, or for each 128
    columns of a row (block = 128).  float32, bfloat16 or float16.  A constant: no gradient goes through it.  stream=: as
    in sinkhorn_forward."""
    values, scales = load_torch_library().pack(x, block)
    return Packed(values, scales, x.shape[-1], block)


@_on_stream
def sinkhorn_unpack(packed, dtype=torch.float32):
    """The values that packed rows stand for, [..., columns], rounded to dtype.  No gradient goes through it."""
    return load_torch_library().unpack(packed, dtype)


@_on_stream
def sinkhorn_expert_product_packed(x, weight, offsets=None, tokens=None, dtype=None):
    """Each expert's rows times its matrix in 8-bit whole numbers, [R, N]: with a scale for each row of x and each of
    the weight's output channels.

    x [T, K] in 16 or 32 bits, which the call packs, or a Packed of it; weight a Packed of [E, N, K]; with tokens [R] of
    a Routing the rows are gathered, without them x is [R, K] in the rows' order.  Rows from offsets[E] on are zero.
    Without offsets the weight is a Packed of [N, K] (or [1, N, K]) and every row is multiplied by it.  The sums are
    exact; dtype is the result's (float32, bfloat16 or float16; default: x's, bfloat16 for a Packed).  For serving: it
    has no gradient, and asking for one raises.  stream=: as in sinkhorn_forward."""
    if isinstance(x, Packed):
        return load_torch_library().product_packed(None, x, weight, offsets, tokens, dtype)
    return load_torch_library().product_packed(x, None, weight, offsets, tokens, dtype)


def sinkhorn_activation(x, activation, gated=False):
    """act(x), or with gated act(x[..., :K]) x[..., K:] of the two halves of the columns; act is "none", "relu", "silu"
    or "gelu" (by the error function).  Differentiable with respect to x, which is kept in 8 bits with a scale for each
    128 columns of a row: the derivative is taken at those values.  float32, bfloat16 or float16, in 32 bits."""
    return load_torch_library().activation(x, _ACTIVATIONS.get(activation, -1), bool(gated))


def sinkhorn_expert_product_kept(x, weight, offsets, tokens=None, slots=None, activation="none", gated=False):
    """As sinkhorn_expert_product, of the activated rows act(x) (as sinkhorn_activation; x has 2 K columns where gated),
    with x kept in 8 bits for the backward pass instead of 16, a scale for each 128 columns of a row; the activated rows
    are not kept.  The result is of x as given, its activated rows rounded to x's type (in float16 one past 65504 is
    infinite); the gradients take x at the values kept, activated again and rounded to x's type.  Between the product and
    the activation's derivative the rows' gradient is rounded to bfloat16, too; in float16, which has not the range for it,
    it stays in 32 bits there."""
    return load_torch_library().product_kept(x, weight, offsets, tokens, slots, _ACTIVATIONS.get(activation, -1),
                                             bool(gated))
