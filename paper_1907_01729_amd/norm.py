"""The norms around a block, fused with its gate and its residual.  Marshalling and autograd wrappers of the C ABI; every
step runs in the HIP library.

    n = sk.sinkhorn_norm(x, sk.Norm(w1))                          # in front of the first block
    z = block(n)                                                  # e.g. a layer of routed experts
    x, n = sk.sinkhorn_residual_norm(z, x, gate=g, after=sk.Norm(w2), before=sk.Norm(w3))   # and of the next
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple

import torch

from ._binding import SkNorms, _int32, load_library
from .routed import _call, _contiguous, _DTYPE, _first_order, _match, _on_stream, _ptr, _recorded, _typed, _workspace


class Norm(NamedTuple):
    """A norm over the columns: (x - m) / sqrt(mean((x - m)^2) + eps) weight + bias, with m the mean where center is
    true and 0 (root mean square) where it is not."""
    weight: torch.Tensor | None = None  # [N], of the rows' type or float32
    bias: torch.Tensor | None = None    # [N], as weight
    eps: float = 1e-6
    center: bool = False


class NormGradients(NamedTuple):
    """What sinkhorn_residual_norm_backward gives; None: not asked for, or nothing to take it of."""
    h: torch.Tensor | None
    residual: torch.Tensor | None
    gate: torch.Tensor | None
    after_weight: torch.Tensor | None
    after_bias: torch.Tensor | None
    before_weight: torch.Tensor | None
    before_bias: torch.Tensor | None


_NO_GATE, _ROWS, _COLUMNS, _FULL = range(4)


@functools.lru_cache(maxsize=1024)
def _norms(T, N, dtype, wdtype, gate, gdtype, after, before, scale, eps_after, eps_before):
    p = SkNorms(*_int32(T, N), dtype, wdtype, gate, gdtype, after, before, scale, eps_after, eps_before)
    ref = ctypes.byref(p)
    return ref, int(load_library().sinkhorn_norm_workspace_bytes(ref))


def _rows(x, name):
    _typed(x, name)
    if x.dim() != 2:
        raise ValueError(f"{name} must be [T, N], got {list(x.shape)}")
    return x.shape


def _kind(norm):
    return 0 if norm is None else 2 if norm.center else 1


def _parameter(t, name, x, N, found):
    """Checks a weight or bias; gives its type, which is the type of all of them."""
    _typed(t, name)
    _match(t, name, x)
    if t.dim() != 1 or t.shape[0] != N:
        raise ValueError(f"{name} must be [{N}], got {list(t.shape)}")
    if t.dtype != x.dtype and t.dtype != torch.float32:
        raise TypeError(f"{name} must be {x.dtype} or float32, got {t.dtype}")
    if found is not None and t.dtype != found:
        raise TypeError(f"all weights and biases must have one type, got {found} and {t.dtype}")
    return t.dtype


def _parameters(x, N, *norms):
    """Checks the named norms' weights and biases and gives their type."""
    found = None
    for name, norm in norms:
        if norm is None:
            continue
        if norm.weight is not None:
            found = _parameter(norm.weight, name + ".weight", x, N, found)
        if norm.bias is not None:
            found = _parameter(norm.bias, name + ".bias", x, N, found)
    return _DTYPE[x.dtype if found is None else found]


def _gate(gate, x):
    """(shape, type) of a gate as the library names them."""
    if gate is None:
        return _NO_GATE, 0
    _typed(gate, "gate")
    _match(gate, "gate", x)
    T, N = x.shape
    if gate.dtype != x.dtype and gate.dtype != torch.float32:
        raise TypeError(f"gate must be {x.dtype} or float32, got {gate.dtype}")
    for kind, shape in ((_FULL, (T, N)), (_ROWS, (T, 1)), (_COLUMNS, (1, N))):
        if tuple(gate.shape) == shape:
            return kind, _DTYPE[gate.dtype]
    raise ValueError(f"gate must be [{T}, {N}], [{T}, 1] or [1, {N}], got {list(gate.shape)}")


def _as_contiguous(norm):
    if norm is None or ((norm.weight is None or norm.weight.is_contiguous()) and
                        (norm.bias is None or norm.bias.is_contiguous())):
        return norm
    return norm._replace(weight=_contiguous(norm.weight), bias=_contiguous(norm.bias))


def _of(norm, what):
    return None if norm is None else getattr(norm, what)


# ---- the norm alone ----

def _norm_sizes(x, norm):
    T, N = _rows(x, "x")
    dtype = _DTYPE[x.dtype]
    return T, N, dtype, _parameters(x, N, ("norm", norm)), 0, 0, 0, _kind(norm), 1.0, 0.0, float(norm.eps)


def _run_norm(x, norm, sizes, with_stats):
    y = torch.empty_like(x)
    stats = torch.empty((sizes[0], 4), device=x.device, dtype=torch.float32) if with_stats else None
    _call(load_library().sinkhorn_norm_forward, x.device, _norms(*sizes)[0], x.data_ptr(), _ptr(norm.weight),
          _ptr(norm.bias), y.data_ptr(), _ptr(stats))
    return y, stats


@_on_stream
def sinkhorn_norm_forward(x, norm=Norm()):
    """(norm of x [T, N], stats); stats goes to sinkhorn_norm_backward.  stream=: as in sinkhorn_forward."""
    return _run_norm(x, norm, _norm_sizes(x, norm), True)


@_on_stream
def sinkhorn_norm_backward(x, norm, stats, grad_y, workspace=None):
    """(grad_x, grad_weight, grad_bias) from the norm's gradient; None for what the norm does not have."""
    sizes = _norm_sizes(x, norm)
    _match(stats, "stats", x, (sizes[0], 4), torch.float32)
    _match(grad_y, "grad_y", x, x.shape, x.dtype)
    return _run_norm_backward(x, norm, stats, grad_y, sizes, (True, norm.weight is not None, norm.bias is not None),
                              workspace)


def _run_norm_backward(x, norm, stats, gy, sizes, wanted, workspace=None):
    ref, need = _norms(*sizes)
    gx = torch.empty_like(x) if wanted[0] else None
    gw = torch.empty_like(norm.weight) if wanted[1] else None
    gb = torch.empty_like(norm.bias) if wanted[2] else None
    scratch = _workspace(workspace, need, x.device) if wanted[1] or wanted[2] else None
    _call(load_library().sinkhorn_norm_backward, x.device, ref, x.data_ptr(), _ptr(norm.weight), stats.data_ptr(),
          gy.data_ptr(), _ptr(gx), _ptr(gw), _ptr(gb), _ptr(scratch), need)
    return gx, gw, gb


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, norm, sizes):
        norm = norm._replace(weight=weight, bias=bias)
        y, stats = _run_norm(x, norm, sizes, True)
        ctx.save_for_backward(x, weight, bias, stats)
        ctx.call = norm._replace(weight=None, bias=None), sizes
        return y

    @staticmethod
    @_first_order
    def backward(ctx, gy):
        x, weight, bias, stats = ctx.saved_tensors
        norm, sizes = ctx.call
        return (*_run_norm_backward(x, norm._replace(weight=weight, bias=bias), stats, gy.contiguous(), sizes,
                                    ctx.needs_input_grad[:3]), None, None)


def sinkhorn_norm(x, norm=Norm()):
    """Norm of the rows of x [T, N], differentiable with respect to x and the norm's weight and bias.  float32, bfloat16
    or float16; statistics and sums in 32 bits, one rounding."""
    x, norm = x.contiguous(), _as_contiguous(norm)
    sizes = _norm_sizes(x, norm)
    if _recorded(x, norm.weight, norm.bias):
        return _Norm.apply(x, norm.weight, norm.bias, norm._replace(weight=None, bias=None), sizes)
    return _run_norm(x, norm, sizes, False)[0]


# ---- a block's end ----

def _residual_sizes(h, gate, scale, after, before):
    T, N = _rows(h, "h")
    kind, gdtype = _gate(gate, h)
    return (T, N, _DTYPE[h.dtype], _parameters(h, N, ("after", after), ("before", before)), kind, gdtype, _kind(after),
            _kind(before), float(scale), 0.0 if after is None else float(after.eps),
            0.0 if before is None else float(before.eps))


def _run_residual(h, residual, gate, after, before, sizes, with_stats):
    out, normed = torch.empty_like(h), None if before is None else torch.empty_like(h)
    stats = torch.empty((sizes[0], 4), device=h.device, dtype=torch.float32) if with_stats else None
    _call(load_library().sinkhorn_residual_norm_forward, h.device, _norms(*sizes)[0], h.data_ptr(),
          residual.data_ptr(), _ptr(gate), _ptr(_of(after, "weight")), _ptr(_of(after, "bias")),
          _ptr(_of(before, "weight")), _ptr(_of(before, "bias")), out.data_ptr(), _ptr(normed), _ptr(stats))
    return out, normed, stats


@_on_stream
def sinkhorn_residual_norm_forward(h, residual, gate=None, scale=1.0, after=None, before=None):
    """(out, next, stats) of a block's end: see sinkhorn_residual_norm; stats goes to
    sinkhorn_residual_norm_backward.  stream=: as in sinkhorn_forward."""
    sizes = _residual_sizes(h, gate, scale, after, before)
    _match(residual, "residual", h, h.shape, h.dtype)
    return _run_residual(h, residual, gate, after, before, sizes, True)


@_on_stream
def sinkhorn_residual_norm_backward(h, out, stats, grad_out=None, grad_next=None, gate=None, scale=1.0, after=None,
                                    before=None, workspace=None):
    """NormGradients from those of out and next (each may be None); those of h and residual are one tensor where out is
    their plain sum."""
    sizes = _residual_sizes(h, gate, scale, after, before)
    _match(out, "out", h, h.shape, h.dtype)
    _match(stats, "stats", h, (sizes[0], 4), torch.float32)
    for t, name in ((grad_out, "grad_out"), (grad_next, "grad_next")):
        if t is not None:
            _match(t, name, h, h.shape, h.dtype)
    wanted = (True, True, *(t is not None for t in (gate, _of(after, "weight"), _of(after, "bias"),
                                                    _of(before, "weight"), _of(before, "bias"))))
    return _run_residual_backward(h, out, gate, after, before, stats, grad_out, grad_next, sizes, wanted, workspace)


def _run_residual_backward(h, out, gate, after, before, stats, g_out, g_next, sizes, wanted, workspace=None):
    ref, need = _norms(*sizes)
    rows = next(t for t in (h, out, g_out) if t is not None)
    like = (rows, rows, gate, _of(after, "weight"), _of(after, "bias"), _of(before, "weight"), _of(before, "bias"))
    grads = [torch.empty_like(t) if w else None for t, w in zip(like, wanted)]
    # Where out = residual + h both have one gradient: it is written once, and is one tensor for both, as of a sum.
    same = after is None and gate is None and sizes[8] == 1.0 and wanted[0] and wanted[1]
    if same:
        grads[0] = None
    sums = any(wanted[3:]) or (wanted[2] and sizes[4] == _COLUMNS)
    scratch = _workspace(workspace, need, stats.device) if sums else None
    _call(load_library().sinkhorn_residual_norm_backward, stats.device, ref, _ptr(h), _ptr(out), _ptr(gate),
          _ptr(_of(after, "weight")), _ptr(_of(after, "bias")), _ptr(_of(before, "weight")), stats.data_ptr(),
          _ptr(g_out), _ptr(g_next), *(_ptr(g) for g in grads), _ptr(scratch), need)
    if same:
        grads[0] = grads[1]
    return NormGradients(*grads)


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, residual, gate, after_w, after_b, before_w, before_b, after, before, sizes):
        after = None if after is None else after._replace(weight=after_w, bias=after_b)
        before = None if before is None else before._replace(weight=before_w, bias=before_b)
        out, normed, stats = _run_residual(h, residual, gate, after, before, sizes, True)
        # Without a norm after the block its output is needed for the gate's gradient alone; without one before the
        # next, the sum is not needed.
        keep_h = after is not None or ctx.needs_input_grad[2]
        ctx.save_for_backward(h if keep_h else None, out if before is not None else None, gate, after_w, after_b,
                              before_w, before_b, stats)
        ctx.norms = after is not None, before is not None
        ctx.sizes = sizes
        ctx.set_materialize_grads(False)  # no zeros for outputs without a gradient
        return (out,) if before is None else (out, normed)

    @staticmethod
    @_first_order
    def backward(ctx, g_out, g_next=None):
        if g_out is None and g_next is None:
            return (None,) * 10
        h, out, gate, after_w, after_b, before_w, before_b, stats = ctx.saved_tensors
        after = Norm(after_w, after_b) if ctx.norms[0] else None
        before = Norm(before_w, before_b) if ctx.norms[1] else None
        return (*_run_residual_backward(h, out, gate, after, before, stats, _contiguous(g_out), _contiguous(g_next),
                                        ctx.sizes, ctx.needs_input_grad[:7]), None, None, None)


def sinkhorn_residual_norm(h, residual, gate=None, scale=1.0, after=None, before=None):
    """The end of a block, and the norm in front of the next:

        out = scale residual + gate after(h),   next = before(out)

    h and residual [T, N]; gate [T, N], [T, 1] or [1, N] (of h's type or float32) or None; after and before a Norm or
    None: without after, h itself is gated; without before, out alone is returned, else (out, next).  Differentiable
    with respect to h, residual, the gate and the norms' weights and biases; scale is a number.  float32, bfloat16 or
    float16, in 32 bits, one rounding of each result; next is the norm of the rounded sum."""
    h, residual, gate = h.contiguous(), residual.contiguous(), _contiguous(gate)
    after, before = _as_contiguous(after), _as_contiguous(before)
    sizes = _residual_sizes(h, gate, scale, after, before)
    _match(residual, "residual", h, h.shape, h.dtype)
    parameters = (_of(after, "weight"), _of(after, "bias"), _of(before, "weight"), _of(before, "bias"))
    if _recorded(h, residual, gate, *parameters):
        plain = lambda n: None if n is None else n._replace(weight=None, bias=None)  # noqa: E731
        got = _ResidualNorm.apply(h, residual, gate, *parameters, plain(after), plain(before), sizes)
        return got[0] if before is None else got
    out, normed, _ = _run_residual(h, residual, gate, after, before, sizes, False)
    return out if before is None else (out, normed)
