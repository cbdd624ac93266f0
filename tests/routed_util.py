"""Definitions of the routed-layer operators in 64 bits, on the CPU, for the tests."""
import numpy as np
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12}  # half a step, relative
FLOOR = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # half a step at 0


def rounding(ref, dtype):
    """The error of one rounding of ref to dtype: half a step is at most 2 UNIT |ref| (just above a power of two)."""
    return 2 * UNIT[dtype] * ref.abs() + FLOOR[dtype]


def route(logits, k, bias=None, mask=None, renormalize=True):
    """The router's outputs; logits a tensor on the CPU (any type), weights and losses in 64 bits and differentiable
    with respect to the double copy that is returned as the last entry."""
    T, E = logits.shape
    l = logits.detach().double().requires_grad_()
    score = logits.detach().float()
    if bias is not None:
        score = score + bias
    score = score.numpy()
    live = np.ones(T, dtype=bool) if mask is None else mask.numpy().copy()
    live &= ~np.all(logits.float().numpy() == -np.inf, axis=1)
    experts = np.full((T, k), -1, dtype=np.int32)
    for t in np.nonzero(live)[0]:
        can = [e for e in range(E) if score[t, e] > -np.inf]
        for s, e in enumerate(sorted(can, key=lambda e: (-score[t, e], e))[:k]):
            experts[t, s] = e
    flat = experts.reshape(-1)
    counts = np.array([(flat == e).sum() for e in range(E)], dtype=np.int32)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    order = np.argsort(np.where(flat < 0, E, flat), kind="stable")
    tokens = np.where(flat[order] >= 0, order // k, -1).astype(np.int32)
    slots = np.full(T * k, -1, dtype=np.int32)
    slots[order] = np.arange(T * k)
    slots[flat < 0] = -1
    n = max(1, int(live.sum()))
    rows = torch.from_numpy(np.nonzero(live)[0])
    weights = torch.zeros(T, k, dtype=torch.float64)
    ll = l[rows]
    p = torch.softmax(ll, 1)
    ch = torch.from_numpy(experts).long()[rows]
    has = ch >= 0
    if renormalize:
        picked = torch.where(has, ll.gather(1, ch.clamp(min=0)), torch.full_like(ch, -np.inf, dtype=torch.float64))
        none = ~has.any(1, keepdim=True)
        w = torch.where(has, torch.softmax(torch.where(none, torch.zeros_like(picked), picked), 1),
                        torch.zeros(1, dtype=torch.float64))
    else:
        w = torch.where(has, p.gather(1, ch.clamp(min=0)), torch.zeros(1, dtype=torch.float64))
    weights = weights.index_copy(0, rows, w)
    f = torch.from_numpy(counts).double() / (k * n)
    balance = E * (f * p.sum(0)).sum() / n
    z = torch.logsumexp(ll, 1).square().sum() / n
    return dict(weights=weights, experts=torch.from_numpy(experts), counts=torch.from_numpy(counts),
                offsets=torch.from_numpy(offsets), tokens=torch.from_numpy(tokens),
                slots=torch.from_numpy(slots).reshape(T, k), balance=balance, z_loss=z, logits=l)


def order_of(experts, E):
    """(offsets, tokens, slots) of given experts [T, k] (-1: none), as int32 tensors."""
    T, k = experts.shape
    flat = experts.reshape(-1).numpy()
    counts = np.bincount(flat[flat >= 0], minlength=E)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    order = np.argsort(np.where(flat < 0, E, flat), kind="stable")
    slots = np.empty(T * k, dtype=np.int32)
    slots[order] = np.arange(T * k, dtype=np.int32)
    slots[flat < 0] = -1
    tokens = np.where(flat[order] >= 0, order // k, -1).astype(np.int32)
    return torch.from_numpy(offsets), torch.from_numpy(tokens), torch.from_numpy(slots.reshape(T, k))


def philox(block, offset, seed):
    """Philox4x32-10: four words for each block number (uint64 array)."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    block = np.asarray(block, dtype=np.uint64)
    c = [block & low, block >> u(32), np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & low, (a >> u(32)) ^ c[3] ^ u(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1)


def keep(first, n, p, seed, offset):
    """(keep as booleans, scale) of the elements first .. first + n."""
    threshold = min(int(p * 65536 + 0.5), 65535)
    i = np.arange(first, first + n, dtype=np.uint64)
    words = philox(np.unique(i // np.uint64(8)), offset, seed)
    at = (i // np.uint64(8) - np.uint64(first // 8)).astype(np.int64)
    j = (i % np.uint64(8)).astype(np.int64)
    u = (words[at, j // 2] >> (16 * (j % 2)).astype(np.uint64)) & np.uint64(0xFFFF)
    return torch.from_numpy(u >= threshold), 65536 / (65536 - threshold)


def products(x, w, offsets, tokens, gy=None):
    """y and, with gy, the gradient of x's rows as they are gathered [R, K], of x and of w, in 64 bits; and the sums
    of absolute products that bound the rounding of sums in 32 bits (named abs_*)."""
    E, N, K = w.shape
    R = tokens.numel() if tokens is not None else x.shape[0]
    out = {}
    for name, (X, W, G) in {"": (x, w, gy), "abs_": (x.abs(), w.abs(), None if gy is None else gy.abs())}.items():
        X, W = X.double(), W.double()
        y = torch.zeros(R, N, dtype=torch.float64)
        gx, gw = torch.zeros_like(X), torch.zeros_like(W)
        for e in range(E):
            lo, hi = int(offsets[e]), int(offsets[e + 1])
            if lo == hi:
                continue
            rows = tokens[lo:hi].long() if tokens is not None else torch.arange(lo, hi)
            y[lo:hi] = X[rows] @ W[e].t()
            if G is not None:
                g = G[lo:hi].double()
                gx.index_add_(0, rows, g @ W[e])
                gw[e] = g.t() @ X[rows]
        out.update({name + "y": y, name + "gx": gx, name + "gw": gw})
    return out
