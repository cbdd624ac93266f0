"""The three terms of the router's gradient in 64 bits, each with a bound of its own: at many tokens those of the losses
are a thousandth of the weights' term, and a bound for the sum would hide them."""
import torch

import routed_util as ref

U = 2.0 ** -24  # half a step of 32 bits, relative


def terms(logits, k, want, mask, renormalize, gw, gb, gz, count_of=None, tokens=None):
    """{output: (its term of the gradient, bound)} for incoming gradients gw [T, k], gb and gz; want is the routing.
    count_of and tokens replace the counts and the number of live tokens, to plant a mistake.

    p (a quotient of exponentials of arguments up to 60) is off by `slack` of itself, as its test has it; the factors of
    a term by the roundings that are counted beside them, its sums by one for each step (16 to a lane, then a tree)."""
    T, E = logits.shape
    live = torch.ones(T, dtype=torch.bool) if mask is None else mask
    live = (live & (logits.float() > -torch.inf).any(1))[:, None]
    l = torch.where(live, logits.double(), torch.zeros(1, dtype=torch.float64))
    slack = (64 + 8 + torch.log2(torch.tensor(E + 1.0)).item()) * U
    p = torch.softmax(l, 1) * live
    n = max(1, int(live.sum())) if tokens is None else tokens
    counts = want["counts"].double() if count_of is None else count_of

    c = gb * E * counts / (k * n) / n
    size = p.new_tensor(abs(gb)) * E * counts / (k * n) / n
    mean = (p * size).sum(1, keepdim=True)
    balance = p * (c - (p * c).sum(1, keepdim=True))
    out = {"balance": (balance, p * size * (slack + 8 * U) + p * mean * (2 * slack + 32 * U))}

    lse = torch.logsumexp(l, 1, keepdim=True)
    top = l.amax(1, keepdim=True)
    out["z_loss"] = (2 * gz * lse * p / n,
                     2 * abs(gz) * p / n * (lse.abs() * (slack + 6 * U) + slack + 4 * U * (lse - top)))

    e, w = want["experts"].long(), want["weights"].detach()
    g = torch.where(e >= 0, gw.double(), torch.zeros(1, dtype=torch.float64))
    spread = lambda t: torch.zeros(T, E + 1, dtype=torch.float64).scatter(1, torch.where(e >= 0, e, E), t)[:, :E]  # noqa: E731
    wg, size = (w * g).sum(1, keepdim=True), (w * g.abs()).sum(1, keepdim=True)
    if renormalize:
        grad, bound = spread(w * (g - wg)), spread(w * g.abs() * (slack + 4 * U) + w * size * (2 * slack + 12 * U))
    else:
        grad = spread(w * g) - p * wg
        bound = spread(w * g.abs()) * (slack + 4 * U) + p * size * (2 * slack + 12 * U)
    out["weights"] = (grad, bound)
    return {name: (v, b + ref.rounding(v, logits.dtype)) for name, (v, b) in out.items()}


SIZES = [(1, 3, 2), (60, 64, 4), (1000, 7, 3), (700, 300, 16), (2500, 256, 8), (4500, 100, 4), (9000, 40, 2),
         (17000, 6, 2), (40000, 12, 3)]


def case(T, E, k, dtype):
    """(logits, mask, routing, incoming gradients) of a size."""
    g = torch.Generator().manual_seed(T + E)
    logits = (1.5 * torch.randn(T, E, generator=g) + 0.5 * torch.randn(E, generator=g)).to(dtype)
    mask = torch.rand(T, generator=g) < 0.9
    mask[0] = True
    renormalize = k % 2 == 0
    want = ref.route(logits, k, None, mask, renormalize)
    return logits, mask, renormalize, want, torch.randn(T, k, generator=g), 3.7, -0.9
