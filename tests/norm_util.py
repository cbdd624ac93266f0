"""The norms around a block in 64 bits, on the CPU, from their formulas, with bounds on what 32 bits and one rounding of
each result may be off by."""
import torch

from routed_util import rounding

U = 2.0 ** -24
# Roundings on the way to a sum of up to 65536 columns: 3 in the tree of eight, up to 8 over a lane's chunks, 6 over the
# wavefront, 15 over the wavefronts, and the mean, the square and eps: 37 units of the sum of absolute terms.  The root
# halves a relative error and adds its own two units.
D = 40


def double(t):
    return None if t is None else t.detach().cpu().double()


def statistics(x, eps, center):
    """(x without its mean, r, and X with |error of xh| <= D U X)."""
    m = x.mean(1, keepdim=True) if center else torch.zeros_like(x[:, :1])
    r = 1 / torch.sqrt((x - m).square().mean(1, keepdim=True) + eps)
    far = (x.abs() + x.abs().mean(1, keepdim=True)) * r if center else torch.zeros_like(x)
    return x - m, r, ((x - m) * r).abs() + far


def forward(x, w, b, eps, center, dtype):
    """(norm, bound)."""
    d, r, X = statistics(x, eps, center)
    w = 1.0 if w is None else w
    y = d * r * w
    absw = abs(w) if isinstance(w, float) else w.abs()
    off = 2 * D * U * X * absw
    if b is not None:
        y = y + b
        off = off + 2 * U * b.abs()
    return y, off + rounding(y, dtype)


def backward(x, w, eps, center, gy, gy_off=None):
    """Gradients of x, w and b in 64 bits from gy (off by gy_off), with bounds that leave out the results' rounding.
    The terms of d - mean(d) - xh mean(d xh) are each off by the D roundings of a sum and by X where xh enters."""
    z, r, X = statistics(x, eps, center)
    xh = z * r
    gy_off = torch.zeros_like(gy) if gy_off is None else gy_off
    w = torch.ones_like(x[:1]) if w is None else w
    d, d_off = gy * w, gy_off * w.abs()
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    gx = r * (d - (mean(d) if center else 0) - xh * mean(d * xh))
    size = d.abs() + (mean(d.abs()) if center else 0) + X * mean(d.abs() * X)
    off = r * (4 * D * U * size + d_off + (mean(d_off) if center else 0) + X * mean(d_off * X))
    T = x.shape[0]
    gw, gw_off = (gy * xh).sum(0), ((D + T) * U * gy.abs() * X + D * U * gy.abs() * X + gy_off * X).sum(0)
    gb, gb_off = gy.sum(0), ((D + T) * U * gy.abs() + gy_off).sum(0)
    return {"x": (gx, off), "w": (gw, gw_off), "b": (gb, gb_off)}


def close(got, want, off, dtype=None):
    """got within off of want, and a rounding to dtype."""
    got = got.detach().cpu()
    dtype = dtype or got.dtype
    assert got.dtype == dtype and got.shape == want.shape, (got.dtype, got.shape, want.shape)
    far = (got.double() - want).abs()
    limit = off + rounding(want, dtype) + 1e-300
    assert bool((far <= limit).all()), float((far / limit).max())
