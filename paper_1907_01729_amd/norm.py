"""The norms around a block, fused with its gate and its residual.  Every step runs in the HIP library: the raw calls go
to its C ABI from here, the differentiable ones through its calls on torch tensors.

    n = sk.sinkhorn_norm(x, sk.Norm(w1))                          # in front of the first block
    z = block(n)                                                  # e.g. a layer of routed experts
    x, n = sk.sinkhorn_residual_norm(z, x, gate=g, after=sk.Norm(w2), before=sk.Norm(w3))   # and of the next
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple

import torch

from ._binding import SkNorms, _int32, load_library, load_torch_library
from .routed import _call, _DTYPE, _match, _on_stream, _ptr, _typed, _workspace


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


_PROXY = torch._C._TorchDispatchModeKey.PROXY


def _not_traced(fn):
    """Refuses fn within torch.jit.trace and make_fx, which record its allocations alone: a replay would give out memory
    that nobody wrote."""
    @functools.wraps(fn)
    def call(*args, **kwargs):
        if torch._C._is_tracing() or torch._C._get_dispatch_mode(_PROXY) is not None:
            raise NotImplementedError(f"{fn.__name__} cannot be traced")
        return fn(*args, **kwargs)
    return call


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


def _pointers(norm):
    return (None, None) if norm is None else (_ptr(norm.weight), _ptr(norm.bias))


# ---- the norm alone ----

def _norm_sizes(x, norm):
    T, N = _rows(x, "x")
    dtype = _DTYPE[x.dtype]
    return T, N, dtype, _parameters(x, N, ("norm", norm)), 0, 0, 0, _kind(norm), 1.0, 0.0, float(norm.eps)


@_on_stream
@_not_traced
def sinkhorn_norm_forward(x, norm=Norm()):
    """(norm of x [T, N], stats); stats goes to sinkhorn_norm_backward.  stream=: as in sinkhorn_forward."""
    sizes = _norm_sizes(x, norm)
    y, stats = torch.empty_like(x), torch.empty((sizes[0], 4), device=x.device, dtype=torch.float32)
    _call(load_library().sinkhorn_norm_forward, x.device, _norms(*sizes)[0], x.data_ptr(), _ptr(norm.weight),
          _ptr(norm.bias), y.data_ptr(), stats.data_ptr())
    return y, stats


@_on_stream
@_not_traced
def sinkhorn_norm_backward(x, norm, stats, grad_y, workspace=None):
    """(grad_x, grad_weight, grad_bias) from the norm's gradient; None for what the norm does not have."""
    sizes = _norm_sizes(x, norm)
    _match(stats, "stats", x, (sizes[0], 4), torch.float32)
    _match(grad_y, "grad_y", x, x.shape, x.dtype)
    ref, need = _norms(*sizes)
    gx, gw, gb = (None if t is None else torch.empty_like(t) for t in (x, norm.weight, norm.bias))
    scratch = _workspace(workspace, need, x.device)
    _call(load_library().sinkhorn_norm_backward, x.device, ref, x.data_ptr(), _ptr(norm.weight), stats.data_ptr(),
          grad_y.data_ptr(), gx.data_ptr(), _ptr(gw), _ptr(gb), _ptr(scratch), need)
    return gx, gw, gb


def sinkhorn_norm(x, norm=Norm()):
    """Norm of the rows of x [T, N], differentiable with respect to x and the norm's weight and bias.  float32, bfloat16
    or float16; statistics and sums in 32 bits, one rounding."""
    return load_torch_library().norm(x, norm)


# ---- a block's end ----

def _residual_sizes(h, gate, scale, after, before):
    T, N = _rows(h, "h")
    kind, gdtype = _gate(gate, h)
    return (T, N, _DTYPE[h.dtype], _parameters(h, N, ("after", after), ("before", before)), kind, gdtype, _kind(after),
            _kind(before), float(scale), 0.0 if after is None else float(after.eps),
            0.0 if before is None else float(before.eps))


@_on_stream
@_not_traced
def sinkhorn_residual_norm_forward(h, residual, gate=None, scale=1.0, after=None, before=None):
    """(out, next, stats) of a block's end: see sinkhorn_residual_norm; stats goes to
    sinkhorn_residual_norm_backward.  stream=: as in sinkhorn_forward."""
    sizes = _residual_sizes(h, gate, scale, after, before)
    _match(residual, "residual", h, h.shape, h.dtype)
    out, normed = torch.empty_like(h), None if before is None else torch.empty_like(h)
    stats = torch.empty((sizes[0], 4), device=h.device, dtype=torch.float32)
    _call(load_library().sinkhorn_residual_norm_forward, h.device, _norms(*sizes)[0], h.data_ptr(),
          residual.data_ptr(), _ptr(gate), *_pointers(after), *_pointers(before), out.data_ptr(), _ptr(normed),
          stats.data_ptr())
    return out, normed, stats


@_on_stream
@_not_traced
def sinkhorn_residual_norm_backward(h, out, stats, grad_out=None, grad_next=None, gate=None, scale=1.0, after=None,
                                    before=None, workspace=None):
    """NormGradients from those of out and next (each may be None)."""
    sizes = _residual_sizes(h, gate, scale, after, before)
    _match(out, "out", h, h.shape, h.dtype)
    _match(stats, "stats", h, (sizes[0], 4), torch.float32)
    for t, name in ((grad_out, "grad_out"), (grad_next, "grad_next")):
        if t is not None:
            _match(t, name, h, h.shape, h.dtype)
    ref, need = _norms(*sizes)
    parameters = [t for n in (after, before) for t in ((None, None) if n is None else (n.weight, n.bias))]
    grads = [None if t is None else torch.empty_like(t) for t in (h, h, gate, *parameters)]
    scratch = _workspace(workspace, need, h.device)
    _call(load_library().sinkhorn_residual_norm_backward, h.device, ref, h.data_ptr(), out.data_ptr(), _ptr(gate),
          *_pointers(after), _pointers(before)[0], stats.data_ptr(), _ptr(grad_out), _ptr(grad_next),
          *(_ptr(g) for g in grads), _ptr(scratch), need)
    return NormGradients(*grads)


def sinkhorn_residual_norm(h, residual, gate=None, scale=1.0, after=None, before=None):
    """The end of a block, and the norm in front of the next:

        out = scale residual + gate after(h),   next = before(out)

    h and residual [T, N]; gate [T, N], [T, 1] or [1, N] (of h's type or float32) or None; after and before a Norm or
    None: without after, h itself is gated; without before, out alone is returned, else (out, next).  Differentiable
    with respect to h, residual, the gate and the norms' weights and biases; scale is a number.  float32, bfloat16 or
    float16, in 32 bits, one rounding of each result; next is the norm of the rounded sum."""
    got = load_torch_library().residual_norm(h, residual, gate, scale, after, before)
    return got[0] if before is None else tuple(got)
