"""Operators around a layer of routed experts: the norms of its block, and its products in 8 bits.

Each case is a dict of plain values.  `kind` names the operator:

  norm    a norm over the columns (root mean square, or mean and variance); "train" adds its gradients
  block   the end of a block: its output normed, gated and added to the scaled residual, and the next block's norm of
          that sum; "train" adds every gradient
  packed  the experts' products in 8-bit whole numbers, with a scale for each token and each output channel: the
          tokens' rows are rounded to 8 bits within the call, the weights are kept so
  kept    the experts' product of activated rows in training, with the rows kept in 8 bits for the backward pass (a
          scale for each 128 columns of a row); "train" adds the gradients of the rows and of the weights

The plain forms below compute in 32 bits (64 where a value is rounded to 8 bits) with elementary operations and round
once at the end.
"""
import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_EPS = 1e-5
_BLOCK = 128  # columns under one scale of a kept row


def listed():
    return [
        # four requests answered a token at a time: the norm in front of the layer, latency
        {"name": "norm_step", "kind": "norm", "T": 4, "N": 2048, "type": "bf16", "center": False, "train": False},
        # a training step's norm in 32 bits over wide rows, with mean and bias
        {"name": "norm_wide", "kind": "norm", "T": 4096, "N": 8192, "type": "fp32", "center": True, "train": True},
        # four single tokens at a block's end: both norms, latency
        {"name": "block_step", "kind": "block", "T": 4, "N": 2048, "type": "bf16", "after": True, "before": True,
         "gate": "none", "scale": 1.0, "center": False, "train": False},
        # a training step with norms on both sides of the block and a gate for each token
        {"name": "block_train", "kind": "block", "T": 8192, "N": 2048, "type": "bf16", "after": True, "before": True,
         "gate": "token", "scale": 0.7, "center": False, "train": True},
        # a long batch, the plain residual with the next block's norm alone
        {"name": "block_long", "kind": "block", "T": 65536, "N": 2048, "type": "bf16", "after": False, "before": True,
         "gate": "none", "scale": 1.0, "center": False, "train": True},
        # rows that no vector load divides, a gate for each element, means and biases
        {"name": "block_odd", "kind": "block", "T": 4099, "N": 1001, "type": "fp16", "after": True, "before": True,
         "gate": "full", "scale": 0.5, "center": True, "train": True},
        # four single tokens: the chosen experts' weights are read once
        {"name": "packed_step", "kind": "packed", "T": 4, "E": 64, "k": 4, "K": 2048, "N": 1024, "type": "bf16",
         "masked": False},
        # a long prompt through many experts
        {"name": "packed_long", "kind": "packed", "T": 16384, "E": 64, "k": 4, "K": 2048, "N": 2048, "type": "bf16",
         "masked": False},
        # odd sizes, tokens without an expert, ragged experts
        {"name": "packed_odd", "kind": "packed", "T": 777, "E": 12, "k": 3, "K": 1003, "N": 517, "type": "fp16",
         "masked": True},
        # the first product of a layer in training: tokens gathered, the input kept in 8 bits
        {"name": "kept_gather", "kind": "kept", "T": 8192, "E": 16, "k": 2, "K": 2048, "N": 2048, "type": "bf16",
         "act": "none", "gated": False, "masked": False, "train": True},
        # the second product: the gated activation of rows in order, which are kept in 8 bits instead of 16
        {"name": "kept_gated", "kind": "kept", "T": 32768, "E": 16, "k": 1, "K": 1024, "N": 2048, "type": "bf16",
         "act": "silu", "gated": True, "masked": False, "train": True},
        # odd sizes
        {"name": "kept_odd", "kind": "kept", "T": 501, "E": 5, "k": 3, "K": 345, "N": 203, "type": "fp16",
         "act": "gelu", "gated": False, "masked": True, "train": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "block", "packed", "kept"])
    typ = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind in ("norm", "block"):
        N = _log(rng, 16, 8192)
        T = _log(rng, 1, min(65536, (1 << 25) // N))
        train = rng.random() < 0.7
        case = {"kind": kind, "T": T, "N": N, "type": typ, "center": rng.random() < 0.4, "train": train}
        if kind == "block":
            after, before = rng.choice([(True, True), (True, False), (False, True)])
            case.update(after=after, before=before, gate=rng.choice(["none", "token", "channel", "full"]),
                        scale=rng.choice([1.0, 0.5, 0.81]))
        return case
    typ = rng.choice(["bf16", "bf16", "fp16"])
    E = _log(rng, 1, 64)
    k = rng.randint(1, min(4, E))
    sizes = [(_log(rng, 64, 2048) + 15) // 16 * 16 for _ in range(2)]
    if rng.random() < 0.25:  # a row that no vector load divides
        sizes[rng.randint(0, 1)] -= rng.randint(1, 15)
    case = {"kind": kind, "T": _log(rng, 1, 8192 if kind == "packed" else 4096), "E": E, "k": k, "K": sizes[0], "N": sizes[1], "type": typ,
            "masked": rng.random() < 0.3}
    if kind == "kept":
        case.update(act=rng.choice(["none", "relu", "silu", "gelu"]), gated=rng.random() < 0.4,
                    train=rng.random() < 0.8)
    return case


# ---- inputs ----

def _order(experts, E):
    """Offsets, tokens and slots of the pairs in the order (expert, token, slot); pairs without an expert come last."""
    T, k = experts.shape
    flat = experts.reshape(-1)
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    counts = torch.zeros(E + 1, dtype=torch.int64, device=flat.device).scatter_add_(0, key, torch.ones_like(key))[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=flat.device)
    offsets[1:] = torch.cumsum(counts, 0)
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=flat.device)
    slots = torch.where(flat < 0, -1, place).reshape(T, k)
    tokens = torch.where(key[order] < E, order // k, -1)
    return max(1, int(counts.max())), offsets.int(), tokens.int(), slots.int()


def _round8(x, columns):
    """(whole numbers of 8 bits, scales) of x's rows, with a scale for every `columns` columns."""
    *lead, K = x.shape
    blocks = -(-K // columns)
    x = torch.nn.functional.pad(x.float(), (0, blocks * columns - K)).view(*lead, blocks, columns)
    s = (x.abs().amax(-1).double() / 127).float()
    q = torch.round(x.double() / torch.where(s > 0, s, 1.0).double()[..., None]).float()  # next to a half: in 64 bits
    return q, s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *n: torch.randn(*n, generator=gen, device="cuda")  # noqa: E731
    typ, train = _TYPES[case["type"]], case.get("train", False)
    leaf = lambda t: t.to(typ).requires_grad_(train)  # noqa: E731
    s = {"case": case}
    T, N = case["T"], case["N"]
    # activations: some columns are far larger than the others
    rows = lambda R, C: randn(R, C) * torch.exp(0.7 * randn(C))  # noqa: E731
    if case["kind"] in ("norm", "block"):
        def parameters(name):
            s[name + "_w"] = leaf(1 + 0.2 * randn(N))
            s[name + "_b"] = leaf(0.2 * randn(N)) if case["center"] else None
        if case["kind"] == "norm":
            s["x"] = leaf(rows(T, N) + (0.5 if case["center"] else 0.0))
            parameters("norm")
            if train:
                s["gy"] = randn(T, N).to(typ)
            return s
        s["h"], s["residual"] = leaf(rows(T, N)), leaf(2 * rows(T, N))
        shape = {"none": None, "token": (T, 1), "channel": (1, N), "full": (T, N)}[case["gate"]]
        s["gate"] = None if shape is None else torch.sigmoid(randn(*shape))
        if shape is not None:  # a router's gate has 32 bits, as its weights have
            s["gate"] = s["gate"].to(torch.float32 if case["gate"] == "token" else typ).requires_grad_(train)
        for name in ("after", "before"):
            if case[name]:
                parameters(name)
        if train:
            s["g_out"], s["g_next"] = randn(T, N).to(typ), randn(T, N).to(typ) if case["before"] else None
        return s
    E, K, k = case["E"], case["K"], case["k"]
    # experts of each token as a trained router picks them: some are wanted more than others
    want = 0.3 * randn(E)
    experts = torch.topk(randn(T, E) + want, k, dim=1).indices
    if case["masked"]:
        gone = torch.rand(T, generator=gen, device="cuda") < 0.1
        experts = torch.where(gone[:, None], -1, experts)
    s["most"], s["offsets"], s["tokens"], s["slots"] = _order(experts, E)  # most: the plain form's rows of an expert
    if k == 1:  # rows in order already
        s["tokens"], s["slots"] = None, None
    w = randn(E, N, K) / math.sqrt(K)
    if case["kind"] == "packed":
        s["x"] = rows(T, K).to(typ)
        q, scales = _round8(w * torch.exp(0.3 * randn(E, N, 1)), K)
        # laid out once, as a program does that serves them: rows of whole 16 bytes, zeros at their end
        s["values"] = torch.nn.functional.pad(q.view(E, N, K), (0, -K % 16)).to(torch.int8)
        s["scales"] = scales.view(E, N)
        return s
    s["x"] = leaf(rows(T, K * (2 if case["gated"] else 1)))
    s["w"] = leaf(w)
    if train:
        s["gy"] = randn(T * k, N).to(typ)
    return s


# ---- one pass ----

def run(state):
    return (_own if own else _plain)[state["case"]["kind"]](state)


def _leaves(s, *names):
    return {n: s[n] for n in names if s.get(n) is not None}


def _own_norm(s):
    import paper_1907_01729_amd as sk
    y = sk.sinkhorn_norm(s["x"], sk.Norm(s["norm_w"], s["norm_b"], _EPS, s["case"]["center"]))
    out = {"y": y}
    if s["case"]["train"]:
        leaves = _leaves(s, "x", "norm_w", "norm_b")
        grads = torch.autograd.grad(y, tuple(leaves.values()), s["gy"])
        out.update(("grad_" + n, g) for n, g in zip(leaves, grads))
    return out


def _own_block(s):
    import paper_1907_01729_amd as sk
    c = s["case"]
    norm = {n: sk.Norm(s[n + "_w"], s[n + "_b"], _EPS, c["center"]) if c[n] else None for n in ("after", "before")}
    y = sk.sinkhorn_residual_norm(s["h"], s["residual"], gate=s["gate"], scale=c["scale"], **norm)
    y = y if c["before"] else (y,)
    out = dict(zip(("out", "next"), y))
    if c["train"]:
        leaves = _leaves(s, "h", "residual", "gate", "after_w", "after_b", "before_w", "before_b")
        grads = torch.autograd.grad(y, tuple(leaves.values()), (s["g_out"], s["g_next"])[:len(y)])
        out.update(("grad_" + n, g) for n, g in zip(leaves, grads))
    return out


def _own_packed(s):
    import paper_1907_01729_amd as sk
    weight = sk.Packed(s["values"], s["scales"], s["case"]["K"], 0)
    return {"y": sk.sinkhorn_expert_product_packed(s["x"], weight, s["offsets"], s["tokens"])}


def _own_kept(s):
    import paper_1907_01729_amd as sk
    c = s["case"]
    y = sk.sinkhorn_expert_product_kept(s["x"], s["w"], s["offsets"], s["tokens"], s["slots"], activation=c["act"],
                                        gated=c["gated"])
    out = {"y": y}
    if c["train"]:
        out["grad_x"], out["grad_w"] = torch.autograd.grad(y, (s["x"], s["w"]), s["gy"])
    return out


def _centred(x, center):
    """x without its mean, and the inverse of its root mean square."""
    if center:
        x = x - x.mean(1, keepdim=True)
    return x, torch.rsqrt(x.square().mean(1, keepdim=True) + _EPS)


def _normed(xh, w, b):
    y = xh * w.to(xh.dtype)
    return y if b is None else y + b.to(xh.dtype)


def _norm_grad(gy, xh, r, w, center):
    """Gradient of x from that of the norm."""
    g = gy * w.to(xh.dtype)
    gx = g - xh * (g * xh).mean(1, keepdim=True)
    if center:
        gx = gx - g.mean(1, keepdim=True)
    return r * gx


def _norm_sums(out, s, name, gy, xh):
    out[f"grad_{name}_w"] = (gy * xh).sum(0).to(s[name + "_w"].dtype)
    if s[name + "_b"] is not None:
        out[f"grad_{name}_b"] = gy.sum(0).to(s[name + "_b"].dtype)


def _plain_norm(s):
    with torch.no_grad():
        c, typ = s["case"], s["x"].dtype
        x, r = _centred(s["x"].float(), c["center"])
        xh = x * r
        out = {"y": _normed(xh, s["norm_w"], s["norm_b"]).to(typ)}
        if c["train"]:
            gy = s["gy"].float()
            out["grad_x"] = _norm_grad(gy, xh, r, s["norm_w"], c["center"]).to(typ)
            _norm_sums(out, s, "norm", gy, xh)
        return out


def _plain_block(s):
    with torch.no_grad():
        c, typ = s["case"], s["h"].dtype
        n = s["h"].float()
        if c["after"]:
            h, rh = _centred(n, c["center"])
            hh = h * rh
            n = _normed(hh, s["after_w"], s["after_b"])
        gate = 1.0 if s["gate"] is None else s["gate"].float()
        y = (c["scale"] * s["residual"].float() + gate * n).to(typ)
        out = {"out": y}
        if c["before"]:
            o, ro = _centred(y.float(), c["center"])
            oh = o * ro
            out["next"] = _normed(oh, s["before_w"], s["before_b"]).to(typ)
        if not c["train"]:
            return out
        g = s["g_out"].float()
        if c["before"]:
            gn = s["g_next"].float()
            g = g + _norm_grad(gn, oh, ro, s["before_w"], c["center"])
        dn = gate * g
        dh = _norm_grad(dn, hh, rh, s["after_w"], c["center"]) if c["after"] else dn
        out["grad_h"], out["grad_residual"] = dh.to(typ), (c["scale"] * g).to(typ)
        if s["gate"] is not None:
            d = g * n
            d = {"token": lambda: d.sum(1, keepdim=True), "channel": lambda: d.sum(0, keepdim=True),
                 "full": lambda: d}[c["gate"]]()
            out["grad_gate"] = d.to(s["gate"].dtype)
        if c["after"]:
            _norm_sums(out, s, "after", dn, hh)
        if c["before"]:
            _norm_sums(out, s, "before", gn, oh)
        return out


def _rows(s, E, R):
    """Of each row: its expert, its source row, whether it has any, and its place among the experts' padded rows."""
    offsets, most = s["offsets"].long(), s["most"]
    row = torch.arange(R, device=offsets.device)
    of = torch.searchsorted(offsets[1:], row, right=True).clamp(max=E - 1)
    used = row < offsets[-1]
    src = row if s["tokens"] is None else s["tokens"].long().clamp(min=0)
    return of, src, used, torch.where(used, of * most + row - offsets[of], E * most)


def _padded(v, at, E, most):
    """Each expert's rows, padded to as many as any has; unused rows land on a last place, which is cut off."""
    return torch.zeros(E * most + 1, v.shape[1], device=v.device).index_copy(0, at, v)[:-1].view(E, most, -1)


def _plain_packed(s):
    with torch.no_grad():
        c, typ = s["case"], s["x"].dtype
        E, K, R = c["E"], c["K"], c["T"] * c["k"]
        q, sx = _round8(s["x"], K)
        of, src, used, at = _rows(s, E, R)
        xr = torch.where(used[:, None], q.view(-1, K)[src], 0.0)
        if R <= E:  # few rows: each with its own copy of its matrix
            y = torch.matmul(s["values"][of][:, :, :K].float(), xr[:, :, None])[:, :, 0]
        else:
            w = s["values"][:, :, :K].float()
            y = torch.bmm(_padded(xr, at, E, s["most"]), w.transpose(1, 2).contiguous())
            y = y.view(E * s["most"], -1)[at.clamp(max=E * s["most"] - 1)]
        y = torch.where(used[:, None], y * sx[src] * s["scales"][of], 0.0)
        return {"y": y.to(typ)}


def _act(kind, x):
    """The activation and its derivative."""
    if kind == "none":
        return x, torch.ones_like(x)
    if kind == "relu":
        return torch.where(x > 0, x, 0.0), (x > 0).to(x.dtype)
    if kind == "silu":
        p = 1 / (1 + torch.exp(-x))
        return x * p, p * (1 + x * (1 - p))
    p = 0.5 * (1 + torch.erf(x / math.sqrt(2)))
    return x * p, p + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


def _activated(c, x):
    """The activated rows, and what carries their gradient to x's columns."""
    if not c["gated"]:
        a, d = _act(c["act"], x)
        return a, lambda g: g * d
    v, u = x.split(c["K"], dim=1)
    a, d = _act(c["act"], v)
    return a * u, lambda g: torch.cat((g * u * d, g * a), 1)


def _plain_kept(s):
    with torch.no_grad():
        c, typ = s["case"], s["x"].dtype
        T, E, k, K = (c[n] for n in ("T", "E", "k", "K"))
        R, most = T * k, s["most"]
        of, src, used, at = _rows(s, E, R)
        place = at.clamp(max=E * most - 1)
        a, _ = _activated(c, s["x"].float())
        w = s["w"].float()
        rows = lambda v: torch.where(used[:, None], v, 0.0)  # noqa: E731
        y = torch.bmm(_padded(rows(a[src]), at, E, most), w.transpose(1, 2).contiguous()).view(E * most, -1)
        out = {"y": rows(y[place]).to(typ)}
        if c["train"]:
            q, sc = _round8(s["x"], _BLOCK)
            x = (q * sc[..., None]).view(T, -1)[:, :s["x"].shape[1]]
            a, back = _activated(c, x)
            gp = _padded(rows(s["gy"].float()), at, E, most)
            gr = rows(torch.bmm(gp, w).view(E * most, K)[place])
            if s["slots"] is not None:
                slots = s["slots"].long()
                gr = torch.where((slots >= 0)[:, :, None], gr[slots.clamp(min=0)], 0.0).sum(1)
            out["grad_x"] = back(gr).to(typ)
            out["grad_w"] = torch.bmm(gp.transpose(1, 2).contiguous(),
                                      _padded(rows(a[src]), at, E, most)).to(typ)
        return out


_own = {"norm": _own_norm, "block": _own_block, "packed": _own_packed, "kept": _own_kept}
_plain = {"norm": _plain_norm, "block": _plain_block, "packed": _plain_packed, "kept": _plain_kept}


# ---- the definitions in 64 bits ----

def _double(t):
    return None if t is None else t.detach().double()


def _exact_norm(x, w, b, center):
    mean = x.mean(1, keepdim=True) if center else torch.zeros_like(x[:, :1])
    z = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + _EPS)
    return z * w + (0 if b is None else b)


def _exact_rounded(x, columns):
    """x rounded to 8 bits, as the values that these stand for."""
    out = torch.empty_like(x, dtype=torch.float64)
    for lo in range(0, x.shape[-1], columns):
        part = x[..., lo:lo + columns].double()
        scale = (part.abs().amax(-1, keepdim=True) / 127).float().double()
        out[..., lo:lo + columns] = torch.where(scale > 0, torch.round(part / scale.clamp(min=1e-300)) * scale, 0.0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("norm", "block"):
        return _exact_block(s)
    T, E, k, N = (case[n] for n in ("T", "E", "k", "N"))
    offsets = s["offsets"].tolist()
    source = torch.arange(T, device="cuda") if s["tokens"] is None else s["tokens"].long()
    y = torch.zeros(T * k, N, dtype=torch.float64, device="cuda")
    if case["kind"] == "packed":
        x = _exact_rounded(s["x"], case["K"])
        for e in range(E):
            if offsets[e] < offsets[e + 1]:
                rows = slice(offsets[e], offsets[e + 1])
                w = s["values"][e, :, :case["K"]].double() * s["scales"][e].double()[:, None]
                y[rows] = x[source[rows]] @ w.t()
        return {"y": y}
    act = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}

    def activated(x):
        if not case["gated"]:
            return act[case["act"]](x)
        return act[case["act"]](x[:, :case["K"]]) * x[:, case["K"]:]

    w = _double(s["w"])
    x = _exact_rounded(s["x"].detach(), _BLOCK).requires_grad_()
    with torch.enable_grad():
        kept = activated(x)
    a = activated(_double(s["x"]))
    out = {"y": y}
    gw, ga = torch.zeros_like(w), torch.zeros_like(a)
    for e in range(E):
        rows = slice(offsets[e], offsets[e + 1])
        src = source[rows]
        y[rows] = a[src] @ w[e].t()
        if case["train"]:
            g = s["gy"][rows].double()
            gw[e] = g.t() @ kept.detach()[src]
            ga.index_add_(0, src, g @ w[e])
    if case["train"]:
        out["grad_x"], = torch.autograd.grad(kept, x, ga)
        out["grad_w"] = gw
    return out


def _exact_block(s):
    """By differentiation of the definition; the sum that the next norm takes is the one that the block gives out."""
    c = s["case"]
    names = [n for n in ("x", "h", "residual", "gate", "norm_w", "norm_b", "after_w", "after_b", "before_w", "before_b")
             if s.get(n) is not None]
    v = {n: _double(s[n]).requires_grad_(c["train"]) for n in names}
    with torch.enable_grad():
        if c["kind"] == "norm":
            y = (_exact_norm(v["x"], v["norm_w"], v.get("norm_b"), c["center"]),)
            out, g = {"y": y[0].detach()}, (s.get("gy"),)
        else:
            n = _exact_norm(v["h"], v["after_w"], v.get("after_b"), c["center"]) if c["after"] else v["h"]
            total = c["scale"] * v["residual"] + v.get("gate", 1.0) * n
            y = (total,)
            if c["before"]:
                given = total + (total.detach().to(s["h"].dtype).double() - total.detach())
                y += (_exact_norm(given, v["before_w"], v.get("before_b"), c["center"]),)
            out, g = dict(zip(("out", "next"), (t.detach() for t in y))), (s.get("g_out"), s.get("g_next"))[:len(y)]
        if c["train"]:
            grads = torch.autograd.grad(y, tuple(v.values()), tuple(t.double() for t in g))
            order = _leaves(s, *(("x", "norm_w", "norm_b") if c["kind"] == "norm" else
                                 ("h", "residual", "gate", "after_w", "after_b", "before_w", "before_b")))
            found = dict(zip(v, grads))
            out.update(("grad_" + n, found[n]) for n in order)
    return out


# ---- what a pass cannot do without ----

def work(case):
    T, N, size = case["T"], case["N"], 4 if case["type"] == "fp32" else 2
    train = case.get("train", False)
    if case["kind"] == "norm":
        # x and y; and in training x, gy and gx (parameters are small beside them)
        return {"bytes": T * N * size * (5 if train else 2) + N * size, "flops": T * N * (14 if train else 4)}
    if case["kind"] == "block":
        full = 1 if case["gate"] == "full" else 0
        arrays = 3 + case["before"] + full  # h, residual, out, next, gate
        if train:  # h (for the norm after, or the gate), out (for the norm before), their gradients and the gate's
            arrays += (1 if case["after"] or case["gate"] != "none" else 0) + 2 * case["before"] + 3 + 2 * full
        per = 4 * (case["after"] + case["before"]) + 3
        return {"bytes": T * N * size * arrays, "flops": T * N * per * (3 if train else 1)}
    E, K, R = case["E"], case["K"], T * case["k"]
    used = min(E, E * (1 - (1 - case["k"] / E) ** T))
    if case["kind"] == "packed":
        return {"bytes": int(T * K * size + used * N * (K + 4) + R * N * size), "flops": 2 * R * K * N}
    wide = 2 * K if case["gated"] else K
    forward = T * wide * size + used * N * K * size + R * N * size
    if not train:
        return {"bytes": int(forward), "flops": 2 * R * K * N}
    kept = T * wide + 4 * T * -(-wide // _BLOCK)  # written, and read again
    back = R * N * size + used * N * K * size + T * wide * size + E * N * K * size
    return {"bytes": int(forward + 2 * kept + back), "flops": 6 * R * K * N}
