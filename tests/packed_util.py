"""Rows in 8 bits and the activations in 64 bits, on the CPU, from their definitions."""
import math

import torch


def pack(x, block=0):
    """(values as float64 whole numbers, scales in 32 bits) of the rows of x; block as in sinkhorn_pack."""
    x = x.detach().cpu()
    *lead, columns = x.shape
    width = block or columns
    blocks = -(-columns // width)
    v = torch.zeros(*lead, blocks * width, dtype=torch.float64)
    v[..., :columns] = x.double()
    v = v.view(*lead, blocks, width)
    most = v.abs().amax(-1)
    bad = ~torch.isfinite(v).all(-1)
    s = torch.where(bad, torch.full_like(most, math.nan), most / 127).float()  # one rounding: 53 bits hold the quotient's
    d = s.double()[..., None]
    q = torch.where((d > 0), torch.round(v / torch.where(d > 0, d, torch.ones_like(d))), torch.zeros_like(v))
    q = q.clamp(-127, 127).reshape(*lead, blocks * width)[..., :columns]
    return q, s if block else s.reshape(*lead)


def unpack(q, s, block=0):
    """s q in 64 bits."""
    if not block:
        return q * s.double()[..., None]
    return q * s.double().repeat_interleave(block, -1)[..., :q.shape[-1]]


def activate(x, kind, gated):
    """act(x), or act(v) u of x = (v, u); x in 64 bits."""
    v, u = x.chunk(2, -1) if gated else (x, None)
    a = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t / (1 + torch.exp(-t)),
         "gelu": lambda t: 0.5 * t * torch.special.erfc(-t / math.sqrt(2))}[kind](v)
    return a * u if gated else a
