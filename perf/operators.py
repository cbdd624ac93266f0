"""Operators of a routed layer of experts: the calls a program makes of them, over the range of sizes it has.

Each case is a dict of plain values.  `kind` names the operator:

  route    experts of each token from its logits, their weights, the counts and the balance loss, and the order
           of the (token, slot) pairs by expert; "train" adds the gradient of the logits
  experts  the product of each expert's rows with that expert's matrix; "train" adds both gradients
  combine  the weighted sum of a token's expert rows, dropped out, on top of a residual; "train" adds the gradients
           of the rows and of the weights
  dropout  dropout from a counter-based generator, on top of a residual or alone; "train" adds the gradient

The plain forms below compute in 32 bits with elementary operations and round once at the end.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # four requests answered a token at a time: latency
        {"name": "route_step", "kind": "route", "T": 4, "E": 64, "k": 4, "type": "bf16", "bias": True, "masked": False,
         "renormalize": True, "train": False},
        # a training step of a layer with few experts
        {"name": "route_train", "kind": "route", "T": 8192, "E": 64, "k": 2, "type": "bf16", "bias": True,
         "masked": False, "renormalize": True, "train": True},
        # many fine experts, a long batch with padding
        {"name": "route_wide", "kind": "route", "T": 65536, "E": 256, "k": 8, "type": "fp32", "bias": True,
         "masked": True, "renormalize": True, "train": True},
        # the experts' products of four single tokens: the chosen weights are read once
        {"name": "experts_step", "kind": "experts", "T": 4, "E": 64, "k": 4, "K": 2048, "N": 1024, "type": "bf16",
         "masked": False, "train": False},
        # ragged: an odd batch, sizes that no tile divides, unrouted tokens
        {"name": "experts_ragged", "kind": "experts", "T": 777, "E": 12, "k": 3, "K": 1000, "N": 520, "type": "fp16",
         "masked": True, "train": True},
        # a training step, few large experts
        {"name": "experts_train", "kind": "experts", "T": 4096, "E": 8, "k": 2, "K": 2048, "N": 4096, "type": "bf16",
         "masked": False, "train": True},
        # a training step, many experts: the largest
        {"name": "experts_many", "kind": "experts", "T": 16384, "E": 64, "k": 4, "K": 2048, "N": 2048, "type": "bf16",
         "masked": False, "train": True},
        # the layer's output for four single tokens
        {"name": "combine_step", "kind": "combine", "T": 4, "D": 2048, "k": 4, "type": "bf16", "p": 0.0,
         "masked": False, "train": False},
        # the layer's output in training
        {"name": "combine_train", "kind": "combine", "T": 16384, "D": 2048, "k": 4, "type": "bf16", "p": 0.1,
         "masked": False, "train": True},
        # dropout of a small batch of features before a label loss
        {"name": "dropout_small", "kind": "dropout", "T": 64, "D": 1000, "type": "fp32", "p": 0.5, "residual": False,
         "train": True},
        # dropout on top of a residual in a large training step
        {"name": "dropout_train", "kind": "dropout", "T": 16384, "D": 4096, "type": "bf16", "p": 0.1,
         "residual": True, "train": True},
        # odd rows: no row begins where a vector load could
        {"name": "dropout_odd", "kind": "dropout", "T": 4099, "D": 1001, "type": "fp16", "p": 0.2, "residual": True,
         "train": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "experts", "combine", "dropout"])
    if kind == "route":
        E = _log(rng, 2, 256)
        train = rng.random() < 0.7
        return {"kind": kind, "T": _log(rng, 1, 65536), "E": E, "k": rng.randint(1, min(8, E)),
                "type": rng.choice(["fp32", "bf16", "fp16"]), "bias": rng.random() < 0.5, "masked": rng.random() < 0.5,
                "renormalize": rng.random() < 0.7, "train": train}
    if kind == "experts":
        E = _log(rng, 2, 64)
        T = _log(rng, 1, 16384)
        sizes = [(_log(rng, 64, 2048) + 7) // 8 * 8 for _ in range(2)]
        if rng.random() < 0.2:  # a row that no vector load divides
            sizes[rng.randint(0, 1)] -= rng.randint(1, 7)
        return {"kind": kind, "T": T, "E": E, "k": rng.randint(1, min(4, E)), "K": sizes[0], "N": sizes[1],
                "type": rng.choice(["bf16", "bf16", "fp16"]), "masked": rng.random() < 0.3,
                "train": T > 64 and rng.random() < 0.8}
    if kind == "combine":
        return {"kind": kind, "T": _log(rng, 1, 16384), "D": _log(rng, 64, 2048), "k": rng.randint(1, 4),
                "type": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "p": rng.choice([0.0, 0.1, 0.25]),
                "masked": rng.random() < 0.3, "train": rng.random() < 0.7}
    return {"kind": kind, "T": _log(rng, 1, 16384), "D": _log(rng, 64, 4096),
            "type": rng.choice(["fp32", "bf16", "fp16"]), "p": rng.choice([0.05, 0.1, 0.3, 0.5]),
            "residual": rng.random() < 0.5, "train": rng.random() < 0.7}


# ---- inputs ----

def _order(experts, E):
    """Offsets, tokens and slots of the pairs in the order (expert, token, slot); pairs without an expert come last."""
    T, k = experts.shape
    flat = experts.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    counts = torch.zeros(E + 1, dtype=torch.int64, device=flat.device).scatter_add_(0, key, torch.ones_like(key))[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=flat.device)
    offsets[1:] = torch.cumsum(counts, 0)
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=flat.device)
    slots = torch.where(flat < 0, -1, place).reshape(T, k)
    tokens = torch.where(key[order] < E, order // k, -1)
    return counts.int(), offsets.int(), tokens.int(), slots.int()


def _routed(gen, T, E, k, masked):
    """Experts of each token as a trained router picks them: some experts are wanted more than others."""
    want = 0.3 * torch.randn(E, generator=gen, device="cuda")
    experts = torch.topk(torch.randn(T, E, generator=gen, device="cuda") + want, k, dim=1).indices.int()
    if masked:
        gone = torch.rand(T, generator=gen, device="cuda") < 0.1
        experts = torch.where(gone[:, None], torch.full_like(experts, -1), experts)
    return experts


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *n: torch.randn(*n, generator=gen, device="cuda")  # noqa: E731
    typ = _TYPES[case["type"]]
    s = {"case": case}
    T = case["T"]
    if case["kind"] == "route":
        E, k = case["E"], case["k"]
        s["logits"] = (1.5 * randn(T, E) + 0.5 * randn(E)).to(typ).requires_grad_(case["train"])
        s["bias"] = 0.4 * randn(E) if case["bias"] else None
        s["mask"] = torch.rand(T, generator=gen, device="cuda") >= 0.1 if case["masked"] else None
        if case["train"]:
            s["g_weights"], s["g_balance"], s["g_z"] = randn(T, k), 0.01 * T * (1 + randn(()).abs()), 0.001 * T * (
                1 + randn(()).abs())
        return s
    if case["kind"] == "experts":
        E, K, N = case["E"], case["K"], case["N"]
        s["experts"] = _routed(gen, T, E, case["k"], case["masked"])
        counts, s["offsets"], s["tokens"], s["slots"] = _order(s["experts"], E)
        s["most"] = int(counts.max())  # the plain form's padded rows of an expert
        s["x"] = randn(T, K).to(typ).requires_grad_(case["train"])
        s["w"] = (randn(E, N, K) / math.sqrt(K)).to(typ).requires_grad_(case["train"])
        if case["train"]:
            s["gy"] = randn(T * case["k"], N).to(typ)
        return s
    D = case["D"]
    s["seed"] = int(torch.randint(0, 1 << 62, (1,), generator=gen, device="cuda"))
    s["offset"] = int(torch.randint(0, 1 << 20, (1,), generator=gen, device="cuda"))
    if case["kind"] == "combine":
        k = case["k"]
        E = 16
        experts = _routed(gen, T, E, k, case["masked"])
        _, s["offsets"], s["tokens"], s["slots"] = _order(experts, E)
        s["z"] = randn(T * k, D).to(typ).requires_grad_(case["train"])
        s["weights"] = torch.softmax(randn(T, k), 1).requires_grad_(case["train"])
        s["residual"] = randn(T, D).to(typ)
    else:
        s["x"] = randn(T, D).to(typ).requires_grad_(case["train"])
        s["residual"] = randn(T, D).to(typ) if case["residual"] else None
    if case["train"]:
        s["gy"] = randn(T, D).to(typ)
    return s


# ---- one pass ----

def run(state):
    return (_own if own else _plain)[state["case"]["kind"]](state)


def _own_route(s):
    import paper_1907_01729_amd as sk
    c = s["case"]
    r = sk.sinkhorn_route(s["logits"], c["k"], bias=s["bias"], mask=s["mask"], renormalize=c["renormalize"])
    out = {n: getattr(r, n) for n in ("weights", "experts", "counts", "offsets", "tokens", "slots", "balance", "z_loss")}
    if c["train"]:
        out["grad"], = torch.autograd.grad((r.weights, r.balance, r.z_loss), (s["logits"],),
                                           (s["g_weights"], s["g_balance"], s["g_z"]))
    return out


def _own_experts(s):
    import paper_1907_01729_amd as sk
    y = sk.sinkhorn_expert_product(s["x"], s["w"], s["offsets"], s["tokens"], s["slots"])
    out = {"y": y}
    if s["case"]["train"]:
        out["grad_x"], out["grad_w"] = torch.autograd.grad(y, (s["x"], s["w"]), s["gy"])
    return out


def _own_combine(s):
    import paper_1907_01729_amd as sk
    y = sk.sinkhorn_expert_combine(s["z"], s["weights"], s["slots"], s["offsets"], residual=s["residual"],
                                   p=s["case"]["p"], seed=s["seed"], offset=s["offset"])
    out = {"y": y}
    if s["case"]["train"]:
        out["grad_z"], out["grad_weights"] = torch.autograd.grad(y, (s["z"], s["weights"]), s["gy"])
    return out


def _own_dropout(s):
    import paper_1907_01729_amd as sk
    y = sk.sinkhorn_dropout(s["x"], s["case"]["p"], s["seed"], s["offset"], residual=s["residual"])
    out = {"y": y}
    if s["case"]["train"]:
        out["grad_x"], = torch.autograd.grad(y, (s["x"],), s["gy"])
    return out


def _plain_route(s):
    with torch.no_grad():
        c = s["case"]
        T, E, k = c["T"], c["E"], c["k"]
        l = s["logits"].float()
        live = torch.ones(T, dtype=torch.bool, device=l.device) if s["mask"] is None else s["mask"]
        top = l.amax(1)
        live = live & (top > -math.inf)
        e = torch.exp(l - top[:, None])
        p = torch.where(live[:, None], e / e.sum(1, keepdim=True), 0.0)
        lse = torch.where(live, top + torch.log(e.sum(1)), 0.0)
        score = l if s["bias"] is None else l + s["bias"]
        order = torch.sort(score, dim=1, descending=True, stable=True)
        can = (order.values[:, :k] > -math.inf) & live[:, None]
        chosen = order.indices[:, :k]
        experts = torch.where(can, chosen, -1)
        lc = torch.where(can, l.gather(1, chosen), -math.inf)
        if c["renormalize"]:
            w = torch.where(can, torch.exp(lc - lc.amax(1, keepdim=True)), 0.0)
            w = torch.where(can, w / w.sum(1, keepdim=True), 0.0)
        else:
            w = torch.where(can, p.gather(1, chosen), 0.0)
        counts, offsets, tokens, slots = _order(experts, E)
        n = live.sum().clamp(min=1).float()
        f = counts.float() / (k * n)
        out = {"weights": w, "experts": experts.int(), "counts": counts, "offsets": offsets, "tokens": tokens,
               "slots": slots, "balance": E * (f * (p.sum(0) / n)).sum(),
               "z_loss": lse.square().sum() / n}
        if c["train"]:
            g = s["g_weights"]
            coef = s["g_balance"] * E / n * f
            grad = p * (coef - (p * coef).sum(1, keepdim=True)) + (2 * s["g_z"] / n) * lse[:, None] * p
            wg = (w * g).sum(1, keepdim=True)
            if c["renormalize"]:
                grad = grad.scatter_add(1, chosen, torch.where(can, w * (g - wg), 0.0))
            else:
                grad = (grad - p * wg).scatter_add(1, chosen, torch.where(can, w * g, 0.0))
            out["grad"] = grad.to(s["logits"].dtype)
        return out


def _plain_experts(s):
    with torch.no_grad():
        c = s["case"]
        T, E, k, K, N = (c[n] for n in ("T", "E", "k", "K", "N"))
        R, typ = T * k, s["x"].dtype
        offsets, tokens, slots = s["offsets"].long(), s["tokens"].long(), s["slots"].long()
        rows = torch.arange(R, device=tokens.device)
        of = torch.searchsorted(offsets[1:], rows, right=True).clamp(max=E - 1)  # the expert of each row
        used = tokens >= 0
        xr = torch.where(used[:, None], s["x"].float()[tokens.clamp(min=0)], 0.0)
        if R <= E:  # few rows: each with its own copy of its matrix
            w = s["w"][of].float()
            out = {"y": torch.matmul(w, xr[:, :, None])[:, :, 0].to(typ)}
            if not c["train"]:
                return out
        w = s["w"].float()
        most = s["most"]
        at = torch.where(used, of * most + rows - offsets[of], E * most)  # the row's place among its expert's padded rows
        # each expert's rows, padded to as many as any has; unused rows land on a last place, which is cut off
        padded = lambda v: torch.zeros(E * most + 1, v.shape[1], device=v.device).index_copy(  # noqa: E731
            0, at, v)[:-1].view(E, most, -1)
        xp = padded(xr)
        y = torch.bmm(xp, w.transpose(1, 2).contiguous()).view(E * most, N)
        y = torch.where(used[:, None], y[at.clamp(max=E * most - 1)], 0.0)
        out = {"y": y.to(typ)}
        if c["train"]:
            gp = padded(torch.where(used[:, None], s["gy"].float(), 0.0))
            gr = torch.bmm(gp, w).view(E * most, K)[at.clamp(max=E * most - 1)]
            gx = torch.where((slots >= 0)[:, :, None], gr[slots.clamp(min=0)], 0.0).sum(1)
            out["grad_x"] = gx.to(typ)
            out["grad_w"] = torch.bmm(gp.transpose(1, 2).contiguous(), xp).to(typ)
        return out


def _mul32(a, b):
    """High and low 32 bits of a * b; a: int64 tensor of 32-bit values, b: a 32-bit constant."""
    low, high = (a & 0xFFFF) * b, (a >> 16) * b
    mid = (low >> 16) + (high & 0xFFFFFFFF)
    return ((high >> 32 << 16) + (mid >> 16)) & 0xFFFFFFFF, ((mid << 16) | (low & 0xFFFF)) & 0xFFFFFFFF


def _plain_keep(n, p, seed, offset, device):
    """scale * keep of n elements: the ten rounds of the generator, eight elements from a block of four words."""
    threshold = min(int(p * 65536 + 0.5), 65535)
    block = torch.arange((n + 7) // 8, device=device, dtype=torch.int64)
    a, b = block & 0xFFFFFFFF, block >> 32
    c, d = torch.full_like(a, offset & 0xFFFFFFFF), torch.full_like(a, offset >> 32)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        h0, l0 = _mul32(a, 0xD2511F53)
        h1, l1 = _mul32(c, 0xCD9E8D57)
        a, b, c, d = h1 ^ b ^ k0, l1, h0 ^ d ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack((a, b, c, d), 1)
    halves = torch.stack((words & 0xFFFF, words >> 16), 2).reshape(-1)[:n]
    return torch.where(halves >= threshold, 65536 / (65536 - threshold), 0.0).float()


def _plain_combine(s):
    with torch.no_grad():
        c = s["case"]
        T, D = c["T"], c["D"]
        slots = s["slots"].long()
        has = (slots >= 0)[:, :, None]
        z = torch.where(has, s["z"].float()[slots.clamp(min=0)], 0.0)  # [T, k, D]
        w = s["weights"]
        keep = (_plain_keep(T * D, c["p"], s["seed"], s["offset"], z.device).view(T, D) if c["p"] > 0 else
                torch.ones(1, 1, device=z.device))
        out = {"y": (s["residual"].float() + keep * (w[:, :, None] * z).sum(1)).to(s["z"].dtype)}
        if c["train"]:
            g = keep * s["gy"].float()
            gz = torch.zeros(T * c["k"] + 1, D, device=z.device)
            gz[torch.where(slots >= 0, slots, T * c["k"]).reshape(-1)] = (w[:, :, None] * g[:, None, :]).reshape(-1, D)
            out["grad_z"] = gz[:-1].to(s["z"].dtype)
            out["grad_weights"] = (g[:, None, :] * z).sum(2)
        return out


def _plain_dropout(s):
    with torch.no_grad():
        c = s["case"]
        x = s["x"]
        keep = _plain_keep(x.numel(), c["p"], s["seed"], s["offset"], x.device).view(x.shape)
        y = keep * x.float()
        out = {"y": (y if s["residual"] is None else y + s["residual"].float()).to(x.dtype)}
        if c["train"]:
            out["grad_x"] = (keep * s["gy"].float()).to(x.dtype)
        return out


_own = {"route": _own_route, "experts": _own_experts, "combine": _own_combine, "dropout": _own_dropout}
_plain = {"route": _plain_route, "experts": _plain_experts, "combine": _plain_combine, "dropout": _plain_dropout}


# ---- what a pass cannot do without ----

def work(case):
    T, b = case["T"], 4 if case["type"] == "fp32" else 2
    both = case["train"]
    if case["kind"] == "route":
        E, k = case["E"], case["k"]
        return {"bytes": T * E * b * (3 if both else 1) + T * k * (24 if both else 16) + 12 * E,
                "flops": T * E * (20 if both else 10)}
    if case["kind"] == "experts":
        E, k, K, N = (case[n] for n in ("E", "k", "K", "N"))
        R = T * k
        step = T * K * b + min(E, R) * N * K * b + R * N * b
        return {"bytes": step * (3 if both else 1), "flops": 2 * R * N * K * (3 if both else 1)}
    D = case["D"]
    if case["kind"] == "combine":
        R = T * case["k"]
        return {"bytes": R * (D * b + 8) + 2 * T * D * b + (T * D * b + 2 * R * D * b + R * 12 if both else 0),
                "flops": R * D * (5 if both else 2)}
    n = T * D
    return {"bytes": n * b * ((3 if case["residual"] else 2) + (2 if both else 0)), "flops": n * (4 if both else 2)}


# ---- the definitions in 64 bits ----

def _exact_keep(n, p, seed, offset):
    threshold = min(int(p * 65536 + 0.5), 65535)
    u = np.uint64
    low = u(0xFFFFFFFF)
    block = np.arange(-(-n // 8), dtype=np.uint64)
    ctr = [block & low, block >> u(32), np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        first, second = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        ctr = [(second >> u(32)) ^ ctr[1] ^ u(key[0]), second & low, (first >> u(32)) ^ ctr[3] ^ u(key[1]), first & low]
        key = [(key[0] + 0x9E3779B9) % 2**32, (key[1] + 0xBB67AE85) % 2**32]
    bits = np.empty((len(block), 8), dtype=np.uint16)
    for j in range(8):
        bits[:, j] = ((ctr[j // 2] >> u(16 * (j % 2))) & u(0xFFFF)).astype(np.uint16)
    return torch.from_numpy((bits.reshape(-1)[:n] >= threshold).astype(np.float64) * (65536 / (65536 - threshold)))


def _exact_route(s):
    c = s["case"]
    E, k = c["E"], c["k"]
    l = s["logits"].detach().double().cpu().numpy()
    score = s["logits"].detach().float().cpu().numpy()  # the order is defined by the sum in 32 bits
    if s["bias"] is not None:
        score = score + s["bias"].cpu().numpy()
    live = np.ones(len(l), dtype=bool) if s["mask"] is None else s["mask"].cpu().numpy()
    e = np.exp(l)  # these logits are far from the range's ends
    total = e.sum(1)
    p = e / total[:, None]
    chosen = np.argsort(-score, axis=1, kind="stable")[:, :k]
    picked = np.take_along_axis(p, chosen, 1) * live[:, None]
    w = picked / picked.sum(1, keepdims=True).clip(1e-300) if c["renormalize"] else picked
    n = max(1, int(live.sum()))
    counts = np.bincount(chosen[live].reshape(-1), minlength=E)
    f = counts / (k * n)
    out = {"weights": w, "experts": None, "counts": None, "offsets": None, "tokens": None, "slots": None,
           "balance": np.array(E * (f * p[live].sum(0)).sum() / n), "z_loss": np.array((np.log(total[live]) ** 2).sum() / n)}
    if c["train"]:
        g = s["g_weights"].double().cpu().numpy()
        dp = np.tile(float(s["g_balance"]) * E * f / n, (len(l), 1))  # d / d p
        if not c["renormalize"]:
            np.add.at(dp, (np.arange(len(l))[:, None], chosen), g)
        else:
            sums = np.take_along_axis(p, chosen, 1).sum(1, keepdims=True)
            np.add.at(dp, (np.arange(len(l))[:, None], chosen), (g - (w * g).sum(1, keepdims=True)) / sums)
        through_lse = 2 * float(s["g_z"]) / n * np.log(total)[:, None]  # lse's gradient is p
        grad = p * (dp - (p * dp).sum(1, keepdims=True)) + through_lse * p
        out["grad"] = grad * live[:, None]
    return {n: v if v is None else torch.from_numpy(np.asarray(v)) for n, v in out.items()}


def _exact_experts(s):
    c = s["case"]
    x, w = s["x"].detach().double(), s["w"].detach().double()
    y = torch.zeros(c["T"] * c["k"], c["N"], dtype=torch.float64, device=x.device)
    gx, gw = torch.zeros_like(x), torch.zeros_like(w)
    bounds = s["offsets"].tolist()
    for e in range(c["E"]):
        lo, hi = bounds[e], bounds[e + 1]
        if lo == hi:
            continue
        mine = s["tokens"][lo:hi].long()
        y[lo:hi] = x[mine] @ w[e].t().contiguous()
        if c["train"]:
            g = s["gy"][lo:hi].double()
            gx.index_add_(0, mine, g @ w[e])
            gw[e] = g.t().contiguous() @ x[mine]
    return {"y": y, "grad_x": gx, "grad_w": gw} if c["train"] else {"y": y}


def _exact_combine(s):
    c = s["case"]
    T, D, k = c["T"], c["D"], c["k"]
    keep = _exact_keep(T * D, c["p"], s["seed"], s["offset"]).view(T, D).cuda() if c["p"] > 0 else 1.0
    z, w = s["z"].detach().double(), s["weights"].detach().double()
    total = torch.zeros(T, D, dtype=torch.float64, device=z.device)
    gz, gw = torch.zeros_like(z), torch.zeros_like(w)
    for j in range(k):
        at = s["slots"][:, j].long()
        rows = (at >= 0).nonzero()[:, 0]
        at = at[rows]
        total[rows] += w[rows, j, None] * z[at]
        if c["train"]:
            g = (keep * s["gy"].double())[rows]
            gz[at] = w[rows, j, None] * g
            gw[rows, j] = (g * z[at]).sum(1)
    y = s["residual"].double() + keep * total
    return {"y": y, "grad_z": gz, "grad_weights": gw} if c["train"] else {"y": y}


def _exact_dropout(s):
    c = s["case"]
    x = s["x"].detach().double()
    keep = _exact_keep(x.numel(), c["p"], s["seed"], s["offset"]).view(x.shape).to(x.device)
    out = {"y": keep * x + (0 if s["residual"] is None else s["residual"].double())}
    if c["train"]:
        out["grad_x"] = keep * s["gy"].double()
    return out


def exact(case, seed):
    return {"route": _exact_route, "experts": _exact_experts, "combine": _exact_combine,
            "dropout": _exact_dropout}[case["kind"]](prepare(case, seed))
