"""A layer of routed experts in front of a label loss, trained on made-up data.

    python examples/routed_layer.py [--steps N] [--no-balance] [--block]

Each step: router logits from the features; the Sinkhorn potentials of the cost -logits between the tokens and the
experts (uniform masses) give each expert the offset under which the experts are taken evenly; the router takes two
experts a token with it; the experts' two products with a ReLU between; the weighted sum with dropout on top of the
features; a linear head; and the Wasserstein loss between the predicted and the given label histograms.

With --block the layer is a block of a deeper network: a norm in front of it and one behind it, a gate and a scaled
residual fused with the next norm, a gated activation between the products, and the products' rows kept in 8 bits for the
backward pass; and it is served with its weights in 8 bits at the end.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1907_01729_amd as sk  # noqa: E402


class RoutedLayer(torch.nn.Module):
    def __init__(self, dim, hidden, experts, k=2, p=0.1, lam=0.3, n_iter=30):
        super().__init__()
        half = dict(device="cuda", dtype=torch.bfloat16)
        self.gate = torch.nn.Parameter(torch.randn(experts, dim, device="cuda") / dim ** 0.5)
        self.w1 = torch.nn.Parameter(torch.randn(experts, hidden, dim, **half) / dim ** 0.5)
        self.w2 = torch.nn.Parameter(torch.randn(experts, dim, hidden, **half) / hidden ** 0.5)
        self.k, self.p, self.lam, self.n_iter = k, p, lam, n_iter

    def even_bias(self, logits):
        """lam * beta of the entropic transport between tokens and experts: [E]."""
        T, E = logits.shape
        mu, nu = logits.new_full((1, T), 1 / T), logits.new_full((1, E), 1 / E)
        return self.lam * sk.sinkhorn_forward(mu, nu, -logits.detach(), self.lam, self.n_iter)["beta"][0]

    def forward(self, x, seed, balanced=True):
        logits = x.float() @ self.gate.t()
        r = sk.sinkhorn_route(logits, self.k, bias=self.even_bias(logits) if balanced else None)
        h = torch.relu(sk.sinkhorn_expert_product(x, self.w1, r.offsets, r.tokens, r.slots))
        z = sk.sinkhorn_expert_product(h, self.w2, r.offsets)
        p = self.p if self.training else 0.0
        return sk.sinkhorn_expert_combine(z, r.weights, r.slots, r.offsets, residual=x, p=p, seed=seed), r


class RoutedBlock(RoutedLayer):
    """out = scale x + gate norm(layer(norm(x))), and the norm of out that the next block begins with."""

    def __init__(self, dim, hidden, experts, scale=0.9, **other):
        super().__init__(dim, 2 * hidden, experts, **other)  # twice the columns: values and their gates
        half = dict(device="cuda", dtype=torch.bfloat16)
        self.w2 = torch.nn.Parameter(torch.randn(experts, dim, hidden, **half) / hidden ** 0.5)
        self.first, self.after, self.before = (torch.nn.Parameter(torch.ones(dim, **half)) for _ in range(3))
        self.open = torch.nn.Parameter(torch.full((1, dim), 0.5, device="cuda"))
        self.scale = scale

    def end(self, z, x):
        return sk.sinkhorn_residual_norm(z, x, self.open, self.scale, sk.Norm(self.after), sk.Norm(self.before))

    def route(self, n, balanced):
        logits = n.float() @ self.gate.t()
        return sk.sinkhorn_route(logits, self.k, bias=self.even_bias(logits) if balanced else None)

    def forward(self, x, seed, balanced=True):
        n = sk.sinkhorn_norm(x, sk.Norm(self.first))
        r = self.route(n, balanced)
        h = sk.sinkhorn_expert_product_kept(n, self.w1, r.offsets, r.tokens, r.slots)
        z = sk.sinkhorn_expert_product_kept(h, self.w2, r.offsets, activation="silu", gated=True)
        p = self.p if self.training else 0.0
        z = sk.sinkhorn_expert_combine(z, r.weights, r.slots, r.offsets, p=p, seed=seed)
        return self.end(z, x)[1], r

    def packed(self):
        """The experts' weights in 8 bits, for serve."""
        return sk.sinkhorn_pack(self.w1), sk.sinkhorn_pack(self.w2)

    @torch.no_grad()
    def serve(self, x, packed, balanced=True):
        """As forward without dropout, with the experts' products in 8 bits."""
        n = sk.sinkhorn_norm(x, sk.Norm(self.first))
        r = self.route(n, balanced)
        h = sk.sinkhorn_expert_product_packed(n, packed[0], r.offsets, r.tokens)
        z = sk.sinkhorn_expert_product_packed(sk.sinkhorn_activation(h, "silu", gated=True), packed[1], r.offsets)
        return self.end(sk.sinkhorn_expert_combine(z, r.weights, r.slots, r.offsets), x)[1]


def main(steps=40, balanced=True, tokens=1024, dim=256, experts=16, classes=20, say=print, block=False):
    torch.manual_seed(0)
    layer = (RoutedBlock if block else RoutedLayer)(dim, 2 * dim, experts)
    head = torch.nn.Linear(dim, classes, device="cuda")
    opt = torch.optim.AdamW([*layer.parameters(), *head.parameters()], lr=2e-3)
    line = torch.linspace(0, 1, classes, device="cuda")
    cost = (line[:, None] - line[None, :]).square().contiguous()
    # Features with a common direction, so that unbalanced logits favour some experts; labels that depend on them.
    features = torch.randn(tokens, dim, device="cuda") + 0.7 * torch.randn(dim, device="cuda")
    target = torch.softmax(3 * (features @ torch.randn(dim, classes, device="cuda")) / dim ** 0.5, 1)
    losses, spread = [], []
    for step in range(steps):
        y, r = layer(features.bfloat16(), seed=step, balanced=balanced)
        predicted = torch.softmax(head(y.float()), 1)
        label = sk.sinkhorn_loss(predicted, target, cost, lam=0.05, n_iter=50).mean()
        loss = label + 0.01 * r.balance + 1e-4 * r.z_loss
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(label.detach()))
        spread.append(float(r.counts.max()) * experts / (tokens * layer.k))
        if say and step % 10 == 0:
            say(f"step {step}: label loss {losses[-1]:.5f}, balance {float(r.balance.detach()):.4f}, "
                f"fullest expert {spread[-1]:.2f} times the mean")
    if block and say:
        layer.eval()
        x = features.bfloat16()
        with torch.no_grad():
            want = layer(x, 0, balanced)[0].float()
        off = (layer.serve(x, layer.packed(), balanced).float() - want).norm() / want.norm()
        say(f"served in 8 bits: {float(off):.4f} of the result's norm away")
    return losses, spread


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--steps", type=int, default=40)
    a.add_argument("--no-balance", action="store_true")
    a.add_argument("--block", action="store_true")
    a = a.parse_args()
    main(a.steps, not a.no_balance, block=a.block)
