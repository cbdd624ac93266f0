"""Routed-layer operators on the GPU against their definitions in 64 bits: router, experts' products, dropout,
combination.  Tolerances: one rounding to the output's type plus what sums in 32 bits can lose."""
import math

import numpy as np
import pytest
import torch

import paper_1907_01729_amd as sk
import routed_util as ref
from routed_util import rounding

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
E32 = 2.0 ** -24  # unit roundoff of 32 bits


def gen(seed):
    return torch.Generator().manual_seed(seed)


def within(got, want, bound):
    """|got - want| <= bound; a result past the type's largest number is infinite."""
    want = want.detach().double()
    past = torch.isinf(want.to(got.dtype))
    got = got.detach().double().cpu()
    assert got.shape == want.shape
    err = torch.where(past & (got == torch.sign(want) * math.inf), torch.zeros_like(want), (got - want).abs())
    bad = ~(err <= bound)
    assert not bad.any(), (int(bad.sum()), err[bad][:4], want[bad][:4], (bound + torch.zeros_like(err))[bad][:4])


def shifted(t):
    """The same contiguous values where no vector load can begin."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    flat[1:] = t.reshape(-1).cuda()
    return flat[1:].view(t.shape)


# ---- router ----

def make_logits(T, E, dtype, seed, scale=1.5):
    g = gen(seed)
    return (scale * torch.randn(T, E, generator=g) + 0.5 * torch.randn(E, generator=g)).to(dtype)


def check_route(logits, k, bias=None, mask=None, renormalize=True, dev_logits=None):
    dl = (logits.cuda() if dev_logits is None else dev_logits).requires_grad_()
    r = sk.sinkhorn_route(dl, k, bias=None if bias is None else bias.cuda(),
                          mask=None if mask is None else mask.cuda(), renormalize=renormalize)
    want = ref.route(logits, k, bias, mask, renormalize)
    for n in ("experts", "counts", "offsets", "tokens", "slots"):
        assert torch.equal(getattr(r, n).cpu(), want[n]), n
    # A weight is a quotient of exponentials whose arguments (at most 60 here, after the scaling to base 2) are
    # rounded to 32 bits: 60 E32, a few more roundings, and the sum's.
    E = logits.shape[1]
    slack = (64 + 8 + math.log2(E + 1)) * E32
    within(r.weights, want["weights"], slack * want["weights"].detach() + 1e-30)
    T = max(1, logits.shape[0])
    sums = slack + 2 * (math.log2(T + 1) + 32 + 16) * E32  # chains of up to 32, then trees and strands
    within(r.balance, want["balance"], sums * want["balance"].detach().abs() + 1e-30)
    within(r.z_loss, want["z_loss"], sums * want["z_loss"].detach().abs() + 16 * E32)
    g = gen(99)
    gw = torch.randn(logits.shape[0], k, generator=g)
    gb, gz = torch.tensor(3.7), torch.tensor(-0.9)
    got, = torch.autograd.grad((r.weights, r.balance, r.z_loss), (dl,), (gw.cuda(), gb.cuda(), gz.cuda()))
    total = (want["weights"] * gw).sum() + gb.double() * want["balance"] + gz.double() * want["z_loss"]
    grad, = torch.autograd.grad(total, (want["logits"],))
    grad = torch.nan_to_num(grad, nan=0.0)  # 0 * inf of -inf logits in the reference
    assert got.dtype == logits.dtype
    # each term of the gradient is a product of factors with the weights' slack; the terms that cancel are at most
    # the largest incoming gradient times a weight
    size = (gw.abs().amax() * 2 + 4 * abs(float(gb)) + 60 * abs(float(gz)) + 1).double()
    within(got, grad, rounding(grad, logits.dtype) + 4 * slack * size)
    return r


ROUTE_SIZES = [(1, 1, 1), (1, 8, 8), (3, 2, 1), (5, 64, 4), (64, 64, 2), (65, 64, 2), (129, 5, 2), (777, 60, 6),
               (300, 256, 8), (130, 300, 16), (70, 1000, 16), (1000, 7, 3), (333, 128, 1), (20, 512, 5), (9, 17, 16),
               (257, 250, 7)]


@pytest.mark.parametrize("T,E,k", ROUTE_SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_route(T, E, k, dtype):
    g = gen(T + E)
    check_route(make_logits(T, E, dtype, T * 7 + E), k, bias=0.4 * torch.randn(E, generator=g),
                mask=torch.rand(T, generator=g) < 0.8, renormalize=bool(k % 2))


@pytest.mark.parametrize("T,E,k", [(40, 64, 4), (333, 100, 8), (700, 256, 2), (90, 600, 4)])
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_without_bias_or_mask_and_unaligned(T, E, k, renormalize):
    l = make_logits(T, E, F32, 5)
    check_route(l, k, renormalize=renormalize)
    check_route(l, k, renormalize=renormalize, dev_logits=shifted(l))
    h = make_logits(T, E, BF16, 6)
    check_route(h, k, renormalize=renormalize, dev_logits=shifted(h))


def test_route_many_tokens():
    """Long runs and many blocks: ranks, block starts and offsets."""
    r = check_route(make_logits(40000, 12, BF16, 1, scale=0.3), 3)
    assert int(r.counts.sum()) == 120000


def test_route_ties_go_to_the_lowest_expert():
    l = torch.randint(0, 3, (500, 64), generator=gen(2)).float()
    check_route(l, 8)
    check_route(torch.zeros(70, 256), 16)
    check_route(torch.zeros(3, 9), 9)


def test_route_masked_logits_and_empty_rows():
    """Rows without a logit above -inf, experts that are out by their logit or bias, masks of the lowest value, fewer
    experts than slots, garbage in masked rows."""
    l = make_logits(200, 33, F32, 3)
    l[::7] = -math.inf
    l[1::7, 5:] = -math.inf  # five experts for eight slots
    l[2::7, ::2] = torch.finfo(F32).min
    l[3::7, 1:] = torch.finfo(F32).min  # one ordinary logit
    l[4::7] = torch.finfo(F32).min  # all at the lowest value: a live row
    bias = 0.1 * torch.randn(33, generator=gen(4))
    bias[0] = bias[32] = -math.inf
    # z would be the square of 3e38: only the integers, the weights and that nothing is NaN elsewhere
    r = sk.sinkhorn_route(l.cuda(), 8, bias=bias.cuda())
    want = ref.route(l, 8, bias)
    for n in ("experts", "counts", "offsets", "tokens", "slots"):
        assert torch.equal(getattr(r, n).cpu(), want[n]), n
    within(r.weights, want["weights"], 1e-5 * want["weights"].detach() + 1e-30)
    assert not torch.isnan(r.weights).any() and torch.isfinite(r.balance)
    mask = torch.ones(200, dtype=torch.bool)
    mask[4::7] = False
    l[4::7] = math.nan
    l[2::7, ::2] = -math.inf
    l[3::7, 1:] = -math.inf
    check_route(l, 8, bias=bias, mask=mask)
    check_route(l, 8, mask=mask, renormalize=False)


def test_route_nothing_live():
    l = make_logits(50, 16, F32, 8)
    for logits, mask in ((l, torch.zeros(50, dtype=torch.bool)), (torch.full_like(l, -math.inf), None)):
        d = logits.cuda().requires_grad_()
        r = sk.sinkhorn_route(d, 2, mask=None if mask is None else mask.cuda())
        assert (r.experts == -1).all() and (r.slots == -1).all() and (r.tokens == -1).all()
        assert not r.counts.any() and not r.offsets.any() and not r.weights.any()
        assert float(r.balance.detach()) == 0 and float(r.z_loss.detach()) == 0
        g, = torch.autograd.grad((r.weights.sum(), r.balance, r.z_loss), (d,), (torch.ones((), device="cuda"),) * 3)
        assert (g == 0).all()
    r = sk.sinkhorn_route(torch.empty(0, 16, device="cuda"), 2)
    assert r.weights.shape == (0, 2) and not r.offsets.any() and float(r.balance) == 0


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_route_not_finite_shows_in_its_row_alone(bad):
    for T in (20, 3000):  # one block, many
        l = make_logits(T, 64, F32, 9)
        l[11, 7] = bad
        if math.isnan(bad):
            l[12] = -math.inf
            l[12, 3] = bad
        r = sk.sinkhorn_route(l.cuda(), 4)
        rows = [11, 12] if math.isnan(bad) else [11]
        for t in rows:
            taken = r.experts[t] >= 0
            assert torch.isnan(r.weights[t][taken]).all()
        rest = [t for t in range(T) if t not in rows]
        assert torch.isfinite(r.weights[rest]).all()
        assert torch.isnan(r.balance) and torch.isnan(r.z_loss)
        e = r.experts.cpu()
        assert int(e.min()) >= -1 and int(e.max()) < 64
        for t in rows:
            got = [v for v in e[t].tolist() if v >= 0]
            assert len(got) == len(set(got))


def test_route_partial_gradients():
    """Each of the three outputs alone, and none of them."""
    l = make_logits(100, 24, F32, 10)
    want = ref.route(l, 3)
    for name in ("weights", "balance", "z_loss"):
        d = l.cuda().requires_grad_()
        g, = torch.autograd.grad(getattr(sk.sinkhorn_route(d, 3), name).sum(), (d,))
        w, = torch.autograd.grad(want[name].sum(), (want["logits"],), retain_graph=True)
        within(g, w, 1e-5 * max(1.0, float(w.abs().max())))


def test_route_gradient_against_differences():
    """Directional differences of the operator's own outputs; logits far enough apart that the choice stays."""
    g = gen(12)
    T, E, k, h = 64, 32, 4, 2.0 ** -7
    l = torch.stack([torch.randperm(E, generator=g) for _ in range(T)]).float() * 0.125
    gw = torch.randn(T, k, generator=g)

    def value(x):
        r = sk.sinkhorn_route(x.cuda(), k)
        return float((r.weights.double().cpu() * gw).sum() + 5 * r.balance.double().cpu() + r.z_loss.double().cpu()
                     ), r.experts.cpu()
    d = l.cuda().requires_grad_()
    r = sk.sinkhorn_route(d, k)
    grad, = torch.autograd.grad((r.weights, r.balance, r.z_loss), (d,),
                                (gw.cuda(), torch.tensor(5.0, device="cuda"), torch.tensor(1.0, device="cuda")))
    for seed in range(4):
        v = torch.randn(T, E, generator=gen(100 + seed)).clamp(-3, 3)
        (up, eu), (down, ed) = value(l + h * v), value(l - h * v)
        assert torch.equal(eu, r.experts.cpu()) and torch.equal(ed, r.experts.cpu())
        diff = (up - down) / (2 * h)
        dot = float((grad.double().cpu() * v).sum())
        # outputs of a size of 50 are off by about 50 * 1e-6 / h; the third derivative gives h^2 of the slope's size
        assert abs(diff - dot) <= 0.01 + 1e-3 * abs(dot)


# ---- experts' products ----

def make_experts(T, k, E, seed, masked=False, only=None):
    g = gen(seed)
    score = torch.rand(T, E, generator=g)
    if only is not None:
        score[:, only] += 10
    experts = score.topk(k, dim=1).indices.int() if T else torch.empty(0, k, dtype=torch.int32)
    if masked:
        experts[torch.rand(T, generator=g) < 0.3] = -1
        experts[torch.rand(T, k, generator=g) < 0.1] = -1
    return ref.order_of(experts, E)


def check_products(T, k, E, K, N, dtype, seed=0, masked=False, only=None, gathered=True, shift=False):
    g = gen(seed + 1)
    offsets, tokens, slots = make_experts(T, k, E, seed, masked, only)
    rows = T if gathered else T * k
    x = torch.randn(rows, K, generator=g).to(dtype)
    w = (torch.randn(E, N, K, generator=g) / math.sqrt(K)).to(dtype)
    gy = torch.randn(T * k, N, generator=g).to(dtype)
    used = int(offsets[E])
    put = shifted if shift else (lambda t: t.cuda())
    dx, dw = put(x), put(w)
    dgy = gy.clone()
    dgy[used:] = math.nan  # rows of no expert take no part
    if gathered and T:
        routed = torch.zeros(T, dtype=torch.bool)
        routed[tokens[tokens >= 0].long()] = True
        dx[~routed.cuda()] = math.nan
    elif T:
        dx[used:] = math.nan
    dx.requires_grad_(), dw.requires_grad_()
    dev = lambda t: t.cuda()  # noqa: E731
    y = (sk.sinkhorn_expert_product(dx, dw, dev(offsets), dev(tokens), dev(slots)) if gathered else
         sk.sinkhorn_expert_product(dx, dw, dev(offsets)))
    gx, gw = torch.autograd.grad(y, (dx, dw), put(dgy))
    want = ref.products(x, w, offsets, tokens if gathered else None, gy)
    assert y.dtype == gx.dtype == gw.dtype == dtype
    # sums in 32 bits of n products in any order: at most n E32 of the sum of their absolute values (twice that, for
    # the matrix core's own rounding), then one rounding
    most = int((offsets[1:] - offsets[:-1]).max()) if E else 0
    within(y, want["y"], rounding(want["y"], dtype) + 2 * (K + 8) * E32 * want["abs_y"])
    within(gx, want["gx"], rounding(want["gx"], dtype) + 2 * (N + k + 8) * E32 * want["abs_gx"])
    within(gw, want["gw"], rounding(want["gw"], dtype) + 2 * (most + 8) * E32 * want["abs_gw"])
    assert (y[used:] == 0).all()


PRODUCTS = [
    # T, k, E, K, N
    (1, 1, 1, 1, 1), (1, 1, 4, 8, 8), (1, 4, 16, 64, 64), (3, 2, 8, 128, 72), (4, 4, 64, 256, 128),
    (16, 2, 3, 200, 136), (33, 1, 2, 64, 256), (64, 3, 5, 96, 80), (100, 2, 7, 264, 520), (257, 2, 4, 512, 256),
    (300, 4, 64, 128, 64), (513, 1, 1, 320, 192), (1000, 2, 3, 256, 384), (65, 16, 20, 48, 40), (2, 1, 200, 40, 24),
    (700, 2, 4, 1032, 264),
]


@pytest.mark.parametrize("T,k,E,K,N", PRODUCTS)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_products(T, k, E, K, N, dtype):
    check_products(T, k, E, K, N, dtype, seed=T + K)


@pytest.mark.parametrize("T,k,E,K,N", [(5, 2, 4, 33, 17), (130, 2, 3, 77, 130), (300, 1, 2, 250, 63), (1, 2, 9, 7, 5),
                                       (260, 3, 5, 129, 264), (260, 3, 5, 264, 129)])
def test_products_odd_sizes(T, k, E, K, N):
    check_products(T, k, E, K, N, BF16, seed=3)
    check_products(T, k, E, K, N, F16, seed=4, masked=True)


@pytest.mark.parametrize("T,k,E,K,N", [(200, 3, 6, 128, 256), (40, 2, 32, 64, 48), (4, 4, 8, 512, 64), (900, 1, 2, 64, 72)])
def test_products_unrouted_tokens(T, k, E, K, N):
    check_products(T, k, E, K, N, BF16, seed=5, masked=True)


def test_products_one_expert_has_all_rows():
    check_products(400, 1, 16, 192, 128, BF16, only=3)
    check_products(400, 1, 16, 192, 128, F16, only=15)


@pytest.mark.parametrize("T,k,E,K,N", [(300, 2, 4, 128, 96), (3, 2, 16, 256, 64), (129, 2, 5, 33, 40)])
def test_products_rows_in_order(T, k, E, K, N):
    check_products(T, k, E, K, N, BF16, gathered=False, masked=True)


def test_products_unaligned():
    check_products(150, 2, 4, 128, 64, BF16, shift=True)
    check_products(3, 2, 4, 128, 64, F16, shift=True)


def test_products_nothing_to_do():
    w = torch.randn(4, 32, 16, device="cuda").to(BF16).requires_grad_()
    x = torch.empty(0, 16, device="cuda", dtype=BF16).requires_grad_()
    off = torch.zeros(5, dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    y = sk.sinkhorn_expert_product(x, w, off, none, none.view(0, 2))
    assert y.shape == (0, 32)
    gx, gw = torch.autograd.grad(y.sum(), (x, w))
    assert gx.shape == (0, 16) and (gw == 0).all()


def test_products_gradient_against_differences():
    """The operator is linear in x and in w: the difference is its value, up to the results' rounding."""
    offsets, tokens, slots = (t.cuda() for t in make_experts(90, 2, 5, 21))
    g = gen(22)
    x = torch.randn(90, 64, generator=g).to(F16).cuda().requires_grad_()
    w = (torch.randn(5, 48, 64, generator=g) / 8).to(F16).cuda().requires_grad_()
    gy = torch.randn(180, 48, generator=g).to(F16).cuda()
    y = sk.sinkhorn_expert_product(x, w, offsets, tokens, slots)
    gx, gw = torch.autograd.grad(y, (x, w), gy)
    with torch.no_grad():
        for t, grad, call in ((x, gx, lambda v: sk.sinkhorn_expert_product(v, w, offsets, tokens, slots)),
                              (w, gw, lambda v: sk.sinkhorn_expert_product(x, v, offsets, tokens, slots))):
            step = torch.randn(t.shape, generator=g).cuda().to(F16) * 0.25
            up, down = t + step, t - step
            moved = (up.double() - down.double())  # the step as it is after rounding
            diff = ((call(up).double() - call(down).double()) * gy.double()).sum()
            dot = (grad.double() * moved).sum()
            size = (grad.double().abs() * moved.abs()).sum() + (y.double().abs() * gy.double().abs()).sum()
            assert abs(float(diff - dot)) <= 2.0 ** -10 * float(size)


# ---- dropout ----

def test_generator_known_answers():
    """Published answers of Philox4x32-10, on the oracle; the GPU is compared with it below."""
    f = lambda b, o, s: [int(v) for v in ref.philox(np.array([b], dtype=np.uint64), o, s)[0]]  # noqa: E731
    assert f(0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    full = (1 << 64) - 1
    assert f(full, full, full) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2048, 2049, 100003])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999999])
def test_dropout(n, dtype, p):
    g = gen(n)
    x, r = torch.randn(n, generator=g).to(dtype), torch.randn(n, generator=g).to(dtype)
    seed, offset = (1 << 63) + 12345 + n, (5 << 32) + 7
    keep, scale = ref.keep(0, n, p, seed, offset)
    kept = torch.where(keep, x.double() * scale, torch.zeros(1, dtype=torch.float64))
    for put in (lambda t: t.cuda(), shifted):
        dx, dr = put(x).requires_grad_(), put(r).requires_grad_()
        y = sk.sinkhorn_dropout(dx, p, seed, offset, residual=dr)
        # the product with the scale (itself rounded), the sum, the output's rounding
        within(y, kept + r.double(), rounding(kept + r.double(), dtype) + 4 * E32 * (kept.abs() + r.double().abs()))
        gy = torch.randn(n, generator=g).to(dtype)
        gx, gr = torch.autograd.grad(y, (dx, dr), put(gy))
        want = torch.where(keep, gy.double() * scale, torch.zeros(1, dtype=torch.float64))
        within(gx, want, rounding(want, dtype) + 4 * E32 * want.abs())
        assert torch.equal(gr.cpu(), gy)
        alone = sk.sinkhorn_dropout(dx.detach(), p, seed, offset)
        within(alone, kept, rounding(kept, dtype) + 4 * E32 * kept.abs())


def test_dropout_rate_and_independence():
    n, p = 1 << 22, 0.3
    one = torch.ones(n, device="cuda")
    a, b, c = (sk.sinkhorn_dropout(one, p, s, o) for s, o in ((1, 0), (2, 0), (1, 1)))
    for y in (a, b, c):  # six standard deviations of a binomial rate
        assert abs(float((y == 0).double().mean()) - p) < 6 * math.sqrt(p * (1 - p) / n) + 2.0 ** -16
    for u, v in ((a, b), (a, c)):
        both = float(((u == 0) & (v == 0)).double().mean())
        assert abs(both - p * p) < 6 * math.sqrt(p * p / n) + 2.0 ** -15
    assert torch.equal(a, sk.sinkhorn_dropout(one, p, 1, 0))


def test_dropout_of_values_that_are_not_finite():
    n = 4096
    x = torch.full((n,), math.nan)
    x[::3] = math.inf
    keep, _ = ref.keep(0, n, 0.5, 3, 0)
    y = sk.sinkhorn_dropout(x.cuda(), 0.5, 3, residual=torch.ones(n, device="cuda")).cpu()
    assert (y[~keep] == 1).all()
    assert not torch.isfinite(y[keep]).any()


def test_dropout_past_32_bits():
    """Elements past 2^32 and blocks past 2^29: numbers in 64 bits."""
    n = (1 << 32) + 4099
    x = torch.ones(n, device="cuda", dtype=BF16)
    y = sk.sinkhorn_dropout(x, 0.25, 77, 9)
    for first in (0, (1 << 31) - 512, (1 << 32) - 512, n - 1000):
        keep, scale = ref.keep(first, 1000, 0.25, 77, 9)
        got = y[first:first + 1000].double().cpu()
        assert torch.equal(got > 0, keep)
    del x, y


# ---- combination ----

def check_combine(T, D, k, dtype, p, seed=0, masked=True, residual=True, shift=False):
    g = gen(seed + T + D)
    _, tokens, slots = make_experts(T, k, 16 if k <= 16 else k, seed, masked)
    offsets = torch.tensor([0, int((slots >= 0).sum())], dtype=torch.int32)
    z = torch.randn(T * k, D, generator=g).to(dtype)
    w = torch.softmax(torch.randn(T, k, generator=g), 1)
    r = torch.randn(T, D, generator=g).to(dtype) if residual else None
    gy = torch.randn(T, D, generator=g).to(dtype)
    put = shifted if shift else (lambda t: t.cuda())
    dz = z.clone()
    dz[int(offsets[-1]):] = math.nan  # rows that no slot names
    dz = put(dz).requires_grad_()
    dw = w.cuda().requires_grad_()
    dr = None if r is None else put(r).requires_grad_()
    y = sk.sinkhorn_expert_combine(dz, dw, slots.cuda(), offsets.cuda(), residual=dr, p=p, seed=11, offset=3)
    keep, scale = ref.keep(0, T * D, p, 11, 3)
    keep = keep.view(T, D).double() * scale if int(p * 65536 + 0.5) else torch.ones(T, D, dtype=torch.float64)
    has = (slots >= 0)[:, :, None].double()
    zs = z.double()[slots.clamp(min=0).long()] * has  # [T, k, D]
    wd = w.double()[:, :, None]
    mix = keep * (wd * zs).sum(1)
    size = keep * (wd * zs).abs().sum(1)
    base = torch.zeros(T, D, dtype=torch.float64) if r is None else r.double()
    within(y, base + mix, rounding(base + mix, dtype) + (k + 4) * E32 * (size + base.abs()))
    inputs = (dz, dw) if dr is None else (dz, dw, dr)
    got = torch.autograd.grad(y, inputs, put(gy))
    gd = keep * gy.double()
    gz = torch.zeros(T * k, D, dtype=torch.float64)
    live = slots >= 0
    gz[slots[live].long()] = (wd * gd[:, None, :])[live]
    within(got[0], gz, rounding(gz, dtype) + 4 * E32 * gz.abs())
    gw = (gd[:, None, :] * zs).sum(2)
    # a lane's chain, then a tree over the wavefront
    within(got[1], gw, (D / 64 + 16) * E32 * (gd[:, None, :] * zs).abs().sum(2) + 1e-30)
    if dr is not None:
        assert torch.equal(got[2].cpu(), gy)


@pytest.mark.parametrize("T,D,k", [(1, 1, 1), (1, 8, 2), (4, 2048, 4), (3, 7, 2), (50, 520, 3), (9, 1001, 4),
                                   (300, 64, 16), (33, 136, 5), (1000, 24, 2), (5, 4096, 8)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_combine(T, D, k, dtype, p):
    check_combine(T, D, k, dtype, p)


def test_combine_without_residual_and_unaligned():
    check_combine(40, 256, 2, BF16, 0.1, residual=False)
    check_combine(40, 256, 2, BF16, 0.1, shift=True)
    check_combine(40, 250, 3, F32, 0.1, residual=False, shift=True)
    check_combine(40, 64, 1, F16, 0.0, masked=False)


def test_combine_gradient_against_differences():
    g = gen(31)
    _, _, slots = make_experts(60, 3, 8, 31)
    offsets = torch.tensor([180], dtype=torch.int32, device="cuda")
    z = torch.randn(180, 72, generator=g).cuda().requires_grad_()
    w = torch.softmax(torch.randn(60, 3, generator=g), 1).cuda().requires_grad_()
    gy = torch.randn(60, 72, generator=g).cuda()
    call = lambda a, b: sk.sinkhorn_expert_combine(a, b, slots.cuda(), offsets, p=0.2, seed=5)  # noqa: E731
    gz, gw = torch.autograd.grad(call(z, w), (z, w), gy)
    with torch.no_grad():
        dz, dw = torch.randn(180, 72, generator=g).cuda(), torch.randn(60, 3, generator=g).cuda()
        for up, down, dot in ((call(z + dz, w), call(z - dz, w), (gz.double() * dz.double()).sum()),
                              (call(z, w + dw), call(z, w - dw), (gw.double() * dw.double()).sum())):
            diff = ((up.double() - down.double()) * gy.double()).sum() / 2  # linear in each
            assert abs(float(diff - dot)) <= 1e-5 * float((up.abs() * gy.abs()).double().sum())


# ---- how they run ----

def layer(x, logits, w1, w2, bias, seed):
    r = sk.sinkhorn_route(logits, 2, bias=bias)
    h = torch.relu(sk.sinkhorn_expert_product(x, w1, r.offsets, r.tokens, r.slots))
    z = sk.sinkhorn_expert_product(h, w2, r.offsets)
    return sk.sinkhorn_expert_combine(z, r.weights, r.slots, r.offsets, residual=x, p=0.1, seed=seed), r


def layer_inputs(T, seed):
    g = gen(seed)
    return (torch.randn(T, 64, generator=g).to(BF16).cuda(), torch.randn(T, 8, generator=g).to(BF16).cuda(),
            (torch.randn(8, 96, 64, generator=g) / 8).to(BF16).cuda(),
            (torch.randn(8, 64, 96, generator=g) / 10).to(BF16).cuda(), (0.1 * torch.randn(8, generator=g)).cuda())


def test_same_bits_twice():
    for T in (3, 700):
        args = layer_inputs(T, 1)
        leaves = [args[0].requires_grad_(), args[1].requires_grad_(), args[2].requires_grad_(), args[3].requires_grad_()]
        runs = []
        for _ in range(2):
            y, r = layer(*args, 5)
            runs.append([y, *r, *torch.autograd.grad((y.float().square().mean() + r.balance + r.z_loss), leaves)])
        for a, b in zip(*runs):
            assert torch.equal(a, b)


def test_on_another_stream():
    args = layer_inputs(500, 2)
    want, _ = layer(*args, 5)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got, _ = layer(*args, 5)
    side.synchronize()
    assert torch.equal(got, want)
    y = sk.sinkhorn_experts_forward(args[0], args[2], torch.tensor([0, 9, 9, 9, 9, 9, 9, 9, 500], device="cuda",
                                                                   dtype=torch.int32))
    torch.cuda.synchronize()
    z = sk.sinkhorn_experts_forward(args[0], args[2], torch.tensor([0, 9, 9, 9, 9, 9, 9, 9, 500], device="cuda",
                                                                   dtype=torch.int32), stream=side)
    side.synchronize()
    assert torch.equal(y, z)


@pytest.mark.parametrize("T", [4, 600])
def test_in_a_graph(T):
    """Captured once, replayed on new inputs with the program's own work between, against the eager result."""
    x, logits, w1, w2, bias = layer_inputs(T, 3)
    with torch.no_grad():
        layer(x, logits, w1, w2, bias, 9)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, r = layer(x, logits, w1, w2, bias, 9)
        for seed in range(4):
            nx, nl, *_ = layer_inputs(T, 40 + seed)
            x.copy_(nx), logits.copy_(nl)
            graph.replay()
            torch.cuda.synchronize()
            want, wr = layer(x, logits, w1, w2, bias, 9)
            assert torch.equal(y, want)
            for a, b in zip(r, wr):
                assert torch.equal(a, b)


def test_refusals_of_gpu_tensors():
    x, logits, w1, w2, bias = layer_inputs(10, 4)
    r = sk.sinkhorn_route(logits, 2)
    with pytest.raises(TypeError):
        sk.sinkhorn_route(logits.double(), 2)
    for k in (0, 9, -1):
        with pytest.raises(sk.SinkhornError):
            sk.sinkhorn_route(logits, k)
    with pytest.raises(ValueError):
        sk.sinkhorn_route(logits[0], 2)
    with pytest.raises(ValueError):
        sk.sinkhorn_route(logits, 2, bias=bias[:3])
    with pytest.raises(TypeError):
        sk.sinkhorn_route(logits, 2, mask=torch.ones(10, device="cuda"))
    with pytest.raises(sk.SinkhornError):
        sk.sinkhorn_route(torch.zeros(2, 1025, device="cuda"), 2)
    with pytest.raises(TypeError):
        sk.sinkhorn_expert_product(x.float(), w1.float(), r.offsets, r.tokens, r.slots)
    with pytest.raises(TypeError):
        sk.sinkhorn_expert_product(x.half(), w1, r.offsets, r.tokens, r.slots)
    with pytest.raises(ValueError):
        sk.sinkhorn_expert_product(x, w2, r.offsets, r.tokens, r.slots)
    with pytest.raises(ValueError):
        sk.sinkhorn_expert_product(x, w1, r.offsets, r.tokens)
    with pytest.raises(ValueError):
        sk.sinkhorn_expert_product(x, w1, r.offsets[:-1], r.tokens, r.slots)
    with pytest.raises(ValueError):
        sk.sinkhorn_expert_product(x[:9], w1, r.offsets, r.tokens, r.slots)
    with pytest.raises(ValueError):
        sk.sinkhorn_expert_product(x, w1[0], r.offsets, r.tokens, r.slots)
    with pytest.raises(TypeError):
        sk.sinkhorn_expert_product(x, w1, r.offsets.long(), r.tokens, r.slots)
    for p in (-0.1, 1.0, 1.5, math.nan):
        with pytest.raises(ValueError):
            sk.sinkhorn_dropout(x, p, 1)
    with pytest.raises(ValueError):
        sk.sinkhorn_dropout(x, 0.1, 1, residual=x[:3])
    with pytest.raises(TypeError):
        sk.sinkhorn_dropout(x, 0.1, 1, residual=x.float())
    z = torch.zeros(20, 64, device="cuda", dtype=BF16)
    with pytest.raises(ValueError):
        sk.sinkhorn_expert_combine(z[:19], r.weights, r.slots, r.offsets)
    with pytest.raises(ValueError):
        sk.sinkhorn_expert_combine(z, r.weights[:, :1], r.slots, r.offsets)
    with pytest.raises(ValueError):
        sk.sinkhorn_expert_combine(z, r.weights, r.slots, r.offsets, residual=x[:, :63])
    with pytest.raises(TypeError):
        sk.sinkhorn_expert_combine(z, r.weights, r.slots.long(), r.offsets)


@pytest.mark.parametrize("T,E,k", [(2500, 256, 8), (4500, 100, 4), (9000, 40, 2), (17000, 6, 2)])
def test_route_work_groups_of_many_threads(T, E, k):
    """Enough tokens for work-groups of 1024 threads, at each number of lanes to a token."""
    check_route(make_logits(T, E, BF16, T), k, mask=torch.rand(T, generator=gen(T)) < 0.9)


@pytest.mark.parametrize("T,k,E,K,N", [(3000, 2, 2, 64, 72), (5000, 1, 1, 136, 80), (9000, 1, 3, 128, 128)])
def test_products_weight_gradient_in_parts(T, k, E, K, N):
    """Small matrices over many rows, one expert's share much larger than another's."""
    check_products(T, k, E, K, N, BF16, seed=8, masked=True)


def test_products_large_tiles():
    """Enough rows and columns for the largest tiles, in each direction, with edges."""
    check_products(4200, 2, 2, 264, 2056, BF16, seed=9, masked=True)
    check_products(4200, 2, 2, 2056, 264, F16, seed=10)
    check_products(600, 1, 33, 1032, 1000, BF16, seed=11)


def test_products_odd_sizes_large_tiles():
    check_products(3000, 2, 3, 1033, 1031, BF16, seed=12, masked=True)
    check_products(2500, 1, 2, 262, 1027, F16, seed=13, gathered=False)


@pytest.mark.parametrize("T", [800_000, 1_200_000])
def test_products_of_long_inputs(T):
    """Inputs past 2^31 and past 2^32 bytes: rows near the end, forward and weight gradient."""
    K, N, E = 2048, 64, 4
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, K, generator=g, device="cuda", dtype=BF16)
    w = (torch.randn(E, N, K, generator=g, device="cuda") / math.sqrt(K)).to(BF16)
    experts = torch.randint(0, E, (T, 1), generator=g, device="cuda").int().cpu()
    offsets, tokens, slots = (t.cuda() for t in ref.order_of(experts, E))
    y = sk.sinkhorn_experts_forward(x, w, offsets, tokens)
    some = torch.cat([torch.arange(0, 300), torch.arange(T // 2, T // 2 + 300), torch.arange(T - 300, T)]).cuda()
    rows = slots[some, 0].long()
    mine = experts.cuda()[some, 0].long()
    xs = x[some].double()
    want = torch.stack([torch.mv(w[e].double(), v) for e, v in zip(mine.tolist(), xs)])
    size = torch.stack([torch.mv(w[e].double().abs(), v.abs()) for e, v in zip(mine.tolist(), xs)])
    within(y[rows], want.cpu(), rounding(want.cpu(), BF16) + 2 * (K + 8) * E32 * size.cpu())
    gy = torch.zeros(T, N, device="cuda", dtype=BF16)
    gs = torch.randn(len(some), N, generator=g, device="cuda").to(BF16)
    gy[rows] = gs
    gw = sk.sinkhorn_experts_backward_weight(gy, x, offsets, tokens)
    want, size = torch.zeros(E, N, K, dtype=torch.float64), torch.zeros(E, N, K, dtype=torch.float64)
    for e in range(E):
        at = (mine == e).nonzero()[:, 0]
        want[e] = (gs[at].double().t().contiguous() @ xs[at]).cpu()
        size[e] = (gs[at].double().abs().t().contiguous() @ xs[at].abs()).cpu()
    # the other rows' products are zeros: they add nothing
    within(gw, want, rounding(want, BF16) + 2 * (len(some) + 8) * E32 * size)


def test_one_gradient_alone():
    args = layer_inputs(90, 6)
    x, w = args[0], args[2]
    r = sk.sinkhorn_route(args[1], 2)
    gy = torch.ones(180, 96, device="cuda", dtype=BF16)
    both = torch.autograd.grad(sk.sinkhorn_expert_product(x.requires_grad_(), w.requires_grad_(), r.offsets, r.tokens,
                                                          r.slots), (x, w), gy)
    gx, = torch.autograd.grad(sk.sinkhorn_expert_product(x, w.detach(), r.offsets, r.tokens, r.slots), (x,), gy)
    gw, = torch.autograd.grad(sk.sinkhorn_expert_product(x.detach(), w, r.offsets, r.tokens, r.slots), (w,), gy)
    assert torch.equal(gx, both[0]) and torch.equal(gw, both[1])
    z = torch.randn(180, 64, device="cuda")
    weights = r.weights.clone().requires_grad_()
    y = sk.sinkhorn_expert_combine(z, weights, r.slots, r.offsets, p=0.2, seed=3)
    g, = torch.autograd.grad(y.sum(), (weights,))
    _, want = sk.sinkhorn_combine_backward(z, weights.detach(), r.slots, r.offsets, torch.ones_like(y), 0.2, 3)
    assert torch.equal(g, want)


def test_no_second_derivative():
    x = torch.randn(8, device="cuda", requires_grad=True)
    g, = torch.autograd.grad((sk.sinkhorn_dropout(x, 0.1, 1) * x).sum(), (x,), create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
