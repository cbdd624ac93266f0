"""Rows in 8 bits: packing, products of packed rows, and activations and products that keep their rows in 8 bits."""
import math

import pytest
import torch

import packed_util as ref
import paper_1907_01729_amd as sk
from routed_util import order_of, products, rounding

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = 2.0 ** -24


def gen(seed):
    return torch.Generator().manual_seed(seed)


def make(*shape, seed, dtype=F32, by=1.0):
    return (by * torch.randn(*shape, generator=gen(seed))).to(dtype).cuda()


def rows(T, K, seed, dtype):
    """Columns of different sizes."""
    return (make(T, K, seed=seed) * torch.exp(0.7 * make(K, seed=seed + 1))).to(dtype)


def check_pack(x, block):
    p = sk.sinkhorn_pack(x, block)
    K = x.shape[-1]
    q, s = ref.pack(x, block)
    assert p.columns == K and p.block == block and p.values.dtype == torch.int8 and p.scales.dtype == F32
    assert p.values.shape == (*x.shape[:-1], -(-K // 16) * 16)
    values = p.values.cpu()
    assert torch.equal(values[..., :K].double(), q)
    assert not values[..., K:].any()
    assert torch.equal(p.scales.cpu().nan_to_num(-1.0), s.nan_to_num(-1.0))
    for dtype in (F32, BF16, F16):
        assert torch.equal(sk.sinkhorn_unpack(p, dtype).cpu().nan_to_num(7.0, 7.0, -7.0),
                           ref.unpack(q, s, block).float().to(dtype).nan_to_num(7.0, 7.0, -7.0))


SHAPES = [(1, 1), (5, 7), (3, 8), (2, 15), (9, 16), (4, 100), (70, 127), (3, 128), (33, 129), (2, 255), (5, 256), (7, 257),
          (64, 1000), (3, 1001), (2, 2048), (3, 8192), (2, 8193), (1, 20001), (600, 72)]


@pytest.mark.parametrize("T,K", SHAPES)
@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_pack(T, K, block, dtype):
    check_pack(rows(T, K, T + K, dtype), block)


@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_ties_and_their_neighbours(block, dtype):
    """Every multiple of half a step and what lies next to it, under scales that are powers of two and others."""
    half = torch.arange(-254, 255, dtype=torch.float64) / 2
    out = []
    for top in (127.0, 127.0 * 2.0 ** -9, 100.0, 3.1415927, 1.0, 0.3):
        s = float(torch.tensor(top / 127, dtype=torch.float64).float())
        v = (half * s).to(F32)
        near = torch.cat((v, torch.nextafter(v, torch.full_like(v, math.inf)),
                          torch.nextafter(v, torch.full_like(v, -math.inf))))
        near = near[near.abs() <= torch.tensor(top)]
        for part in near.split(127):
            row = torch.zeros(128)
            row[0] = top
            row[1:1 + len(part)] = part
            out.append(row)
    check_pack(torch.stack(out).to(dtype).cuda(), block)


@pytest.mark.parametrize("block", [0, 128])
def test_sizes_from_the_smallest_to_the_largest(block):
    """Scales that 32 bits hold with few bits, or not at all, and rows of zeros."""
    base = torch.randn(40, 130, generator=gen(1))
    base[:, 0] = 1.0 + torch.rand(40, generator=gen(2))
    x = torch.cat([base * 2.0 ** e for e in (-149, -147, -143, -142, -141, -130, -126, -100, -97, -96, -95, -60, 0, 60,
                                             120, 126)] + [torch.zeros(3, 130), -torch.zeros(1, 130)])
    x = x[torch.isfinite(x).all(1)]
    check_pack(x.cuda(), block)
    check_pack(x.to(BF16).cuda(), block)


@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_what_is_not_finite_stays_under_its_scale(block, dtype):
    x = rows(6, 300, 1, dtype)
    x[1, 5], x[2, 299], x[3, 130], x[4] = math.nan, math.inf, -math.inf, math.nan
    check_pack(x, block)


def test_leading_dimensions_strides_and_no_rows():
    w = make(3, 5, 40, seed=1, dtype=BF16)
    p = sk.sinkhorn_pack(w)
    assert p.values.shape == (3, 5, 48) and p.scales.shape == (3, 5)
    assert torch.equal(sk.sinkhorn_unpack(p), sk.sinkhorn_unpack(sk.sinkhorn_pack(w.view(15, 40))).view(3, 5, 40))
    a, b = sk.sinkhorn_pack(w.transpose(0, 1)), sk.sinkhorn_pack(w.transpose(0, 1).contiguous())
    assert torch.equal(a.values, b.values) and torch.equal(a.scales, b.scales)
    p = sk.sinkhorn_pack(w[:0], 128)
    assert p.scales.shape == (0, 5, 1) and sk.sinkhorn_unpack(p).shape == (0, 5, 40)
    p = sk.sinkhorn_pack(w[0, 0])
    assert p.values.shape == (48,) and p.scales.shape == ()
    odd = make(3 * 257 + 3, seed=1, dtype=BF16)[3:].view(3, 257)
    check_pack(odd, 0)
    check_pack(odd, 128)


def test_more_than_2_to_the_32_bytes():
    """Rows whose bytes 32 bits do not count: those at the end are their own."""
    K = 8192
    x = torch.zeros(300000, K, device="cuda", dtype=BF16)
    x[-3:] = rows(3, K, 1, BF16)
    for block in (0, 128):
        p = sk.sinkhorn_pack(x, block)
        q, s = ref.pack(x[-3:], block)
        assert torch.equal(p.values[-3:].cpu().double(), q) and torch.equal(p.scales[-3:].cpu(), s)
        assert not p.values[-6:-3].any()


# ---- products ----

def routed(T, E, k, seed, none=0.0):
    experts = torch.rand(T, E, generator=gen(seed)).topk(k, 1).indices.int()
    if none:
        experts[torch.rand(T, k, generator=gen(seed + 1)) < none] = -1
    return tuple(t.cuda() for t in order_of(experts, E))


def check_product(x, w, offsets, tokens, dtype=None, packed=False):
    """The product from the whole numbers and the scales in 64 bits; three roundings in 32 bits and one to the type.  The
    sum itself, up to 2^30, is exact until it becomes a 32-bit float."""
    w8 = sk.sinkhorn_pack(w)
    y = sk.sinkhorn_expert_product_packed(sk.sinkhorn_pack(x) if packed else x, w8, offsets, tokens, dtype)
    qx, sx = ref.pack(x)
    qw, sw = ref.pack(w)
    if qw.dim() == 2:
        qw, sw = qw[None], sw[None]
    E, N = sw.shape
    bounds = offsets.cpu().tolist() if offsets is not None else [0, x.shape[0]]
    R = tokens.numel() if tokens is not None else x.shape[0]
    src = tokens.cpu().long() if tokens is not None else torch.arange(R)
    want = torch.zeros(R, N, dtype=torch.float64)
    for e in range(E):
        lo, hi = bounds[e], bounds[e + 1]
        want[lo:hi] = (qx[src[lo:hi]] @ qw[e].t()) * sx[src[lo:hi]].double()[:, None] * sw[e].double()
    assert y.dtype == (dtype or (BF16 if packed else x.dtype)) and y.shape == want.shape
    far = (y.cpu().double() - want).abs()
    assert bool((far <= 4 * U * want.abs() + rounding(want, y.dtype)).all())
    return y


PRODUCTS = [
    # T, E, k, K, N: single tokens, each tile size, odd widths, experts without rows
    (1, 1, 1, 1, 1), (1, 4, 2, 16, 8), (4, 64, 4, 256, 96), (3, 5, 3, 100, 33), (7, 2, 1, 17, 1), (16, 16, 2, 2048, 40),
    (200, 4, 2, 65, 70), (150, 3, 1, 130, 7), (700, 5, 2, 1000, 517), (1000, 3, 2, 128, 1024), (1500, 2, 2, 513, 1536),
    (4096, 2, 2, 320, 4100),
]


@pytest.mark.parametrize("T,E,k,K,N", PRODUCTS)
@pytest.mark.parametrize("dtype,out", [(BF16, None), (F16, F32), (F32, BF16)])
def test_product(T, E, k, K, N, dtype, out):
    offsets, tokens, slots = routed(T, E, k, T + K, none=0.1)
    check_product(rows(T, K, 1, dtype), make(E, N, K, seed=2, by=K ** -0.5, dtype=BF16), offsets, tokens, out)


# Tiles of 64 with four buffers and (from 513 on) three, and of 128 with three (from 769 of 64 on): contractions of no whole
# step, one, and up to more than there are buffers.
@pytest.mark.parametrize("K", [1, 96, 128, 129, 256, 300, 384, 400, 512, 513, 640, 777])
@pytest.mark.parametrize("T,E,N", [(70, 2, 65), (2000, 1, 1400), (2000, 1, 1800)])
def test_every_number_of_steps(T, E, N, K):
    offsets, tokens, _ = routed(T, E, 1, K, none=0.05)
    x, w = rows(T, K, 1, BF16), make(E, N, K, seed=2, by=K ** -0.5, dtype=BF16)
    check_product(x, w, offsets, tokens, F32)
    check_product(x, w, torch.tensor([0, *[T // 2] * (E - 1), T - 3], dtype=torch.int32).cuda(), None, packed=True)


@pytest.mark.parametrize("K", [8, 64, 72, 128, 136, 192, 256, 320, 392])
@pytest.mark.parametrize("T,E,N", [(70, 2, 72), (2000, 1, 1400), (2000, 1, 1800)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_every_number_of_steps_in_16_bits(T, E, N, K, dtype):
    """The product forward, and the input gradient with K as its contraction (N a row's columns)."""
    offsets, tokens, slots = routed(T, E, 1, K, none=0.05)
    x, w = make(T, K, seed=1, dtype=dtype), make(E, N, K, seed=2, by=K ** -0.5, dtype=dtype)
    p = products(x.cpu(), w.cpu(), offsets.cpu(), tokens.cpu())
    y = sk.sinkhorn_expert_product(x, w, offsets, tokens, slots)
    far = (y.cpu().double() - p["y"]).abs()
    assert bool((far <= rounding(p["y"], dtype) + 2 * (K + 8) * U * p["abs_y"]).all())
    back, v, gy = w.mT.contiguous(), make(T, N, seed=3, dtype=dtype).requires_grad_(), x  # [E, K, N]
    o = offsets.clone()
    o[-1] = T - 5
    p = products(v.detach().cpu(), back.cpu(), o.cpu(), None, gy.cpu())
    gx, = torch.autograd.grad(sk.sinkhorn_expert_product(v, back, o), v, gy)
    far = (gx.cpu().double() - p["gx"]).abs()
    assert bool((far <= rounding(p["gx"], dtype) + 2 * (K + 8) * U * p["abs_gx"]).all())


@pytest.mark.parametrize("T,E,K,N", [(5, 3, 40, 24), (300, 4, 200, 130), (3000, 2, 256, 2048)])
def test_product_of_rows_in_order(T, E, K, N):
    offsets = torch.tensor([0] + sorted(torch.randint(0, T, (E,), generator=gen(3)).tolist()), dtype=torch.int32).cuda()
    y = check_product(rows(T, K, 1, BF16), make(E, N, K, seed=2, dtype=F16), offsets, None, F32, packed=True)
    assert not y[int(offsets[-1]):].any()


@pytest.mark.parametrize("T,K,N", [(1, 64, 24), (40, 1003, 65), (500, 129, 700), (2500, 512, 2304)])
@pytest.mark.parametrize("three", [True, False])
def test_product_with_one_matrix(T, K, N, three):
    w = make(*((1,) if three else ()), N, K, seed=2, dtype=BF16)
    check_product(rows(T, K, 1, BF16), w, None, None)
    check_product(rows(T, K, 1, BF16), w, None, None, F16, packed=True)


def test_the_largest_sum_is_exact():
    """K = 65536 products of 127 and 127: 2^30 and more, which a float holds with an error that shows."""
    K = 65536
    x = torch.full((130, K), 127.0, device="cuda", dtype=BF16)
    x[1::2, ::2] = -127.0
    x[1::2, 0] = 126.0
    w = torch.full((24, K), 127.0, device="cuda", dtype=BF16)
    w[1, 5] = 3.0
    y = sk.sinkhorn_expert_product_packed(x, sk.sinkhorn_pack(w), dtype=F32)
    s = float(torch.tensor(1.0))
    assert float(sk.sinkhorn_pack(x).scales[0]) == s
    want = (x.double().cpu() @ w.double().cpu().t()).float()
    assert torch.equal(y.cpu(), want)


def test_product_by_tiles_and_rows_agree():
    """The forms for few and for many rows give the same bits: the sums are exact."""
    E, K, N = 2, 384, 520
    w8 = sk.sinkhorn_pack(make(E, N, K, seed=2, dtype=BF16))
    x = rows(5000, K, 1, BF16)
    offsets = torch.tensor([0, 2600, 5000], dtype=torch.int32).cuda()
    y = sk.sinkhorn_expert_product_packed(x, w8, offsets)
    for lo, hi in ((0, 40), (2590, 2610), (4970, 5000)):
        off = torch.tensor([0, max(0, min(2600, hi) - lo), hi - lo], dtype=torch.int32).cuda()
        assert torch.equal(sk.sinkhorn_expert_product_packed(x[lo:hi], w8, off), y[lo:hi])
    off = torch.tensor([0, 100, 200], dtype=torch.int32).cuda()
    mid = torch.cat((x[2500:2600], x[2600:2700]))
    assert torch.equal(sk.sinkhorn_expert_product_packed(mid, w8, off), y[2500:2700])


def test_what_is_not_finite_in_a_product():
    """A token's NaN shows in its own rows, a channel's in its own column, and rows of no expert stay zero."""
    T, E, k, K, N = 90, 3, 2, 64, 40
    offsets, tokens, slots = routed(T, E, k, 1, none=0.2)
    x, w = rows(T, K, 1, BF16), make(E, N, K, seed=2, dtype=BF16)
    x[5, 3], x[6, 0] = math.nan, math.inf
    w[1, 7, 2] = math.nan
    y = sk.sinkhorn_expert_product_packed(x, sk.sinkhorn_pack(w), offsets, tokens).cpu()
    bad = (tokens.cpu() == 5) | (tokens.cpu() == 6)
    expert = torch.zeros(T * k, N, dtype=torch.bool)
    lo, hi = offsets[1:3].tolist()
    expert[lo:hi, 7] = True
    assert torch.equal(y.isnan(), bad[:, None] | expert)
    assert not y[int(offsets[-1]):].any()


def test_tokens_past_2_to_the_32_bytes():
    """Gathered rows whose bytes 32 bits do not count."""
    T, K, N = 280000, 16384, 136
    values = torch.zeros(T, K, device="cuda", dtype=torch.int8)
    scales = torch.ones(T, device="cuda")
    pick = torch.cat((torch.arange(0, 70), torch.arange(T - 100, T)))
    x = rows(len(pick), K, 1, BF16)
    p = sk.sinkhorn_pack(x)
    values[pick.cuda()], scales[pick.cuda()] = p.values, p.scales
    w8 = sk.sinkhorn_pack(make(2, N, K, seed=2, dtype=BF16))
    tokens = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    tokens[:len(pick)] = pick.int().cuda()
    offsets = torch.tensor([0, 90, len(pick)], dtype=torch.int32).cuda()
    got = sk.sinkhorn_expert_product_packed(sk.Packed(values, scales, K), w8, offsets, tokens)
    want = sk.sinkhorn_expert_product_packed(p, w8, offsets)
    assert torch.equal(got[:len(pick)], want) and not got[len(pick):].any()


def test_wrong_products():
    x, w = make(8, 32, seed=1, dtype=BF16), make(2, 16, 32, seed=2, dtype=BF16)
    w8 = sk.sinkhorn_pack(w)
    offsets = torch.tensor([0, 4, 8], dtype=torch.int32).cuda()
    odd = torch.empty(2 * 16 * 32 + 1, dtype=torch.int8, device="cuda")[1:].view(2, 16, 32)
    for call, error in ((lambda: sk.sinkhorn_expert_product_packed(x, w, offsets), TypeError),
                        (lambda: sk.sinkhorn_expert_product_packed(x, w8), ValueError),
                        (lambda: sk.sinkhorn_expert_product_packed(x[:, :16], w8, offsets), ValueError),
                        (lambda: sk.sinkhorn_expert_product_packed(x, w8, offsets[:2]), ValueError),
                        (lambda: sk.sinkhorn_expert_product_packed(x, w8, offsets.long()), TypeError),
                        (lambda: sk.sinkhorn_expert_product_packed(x, sk.sinkhorn_pack(w, 128), offsets), ValueError),
                        (lambda: sk.sinkhorn_expert_product_packed(sk.sinkhorn_pack(x, 128), w8, offsets), ValueError),
                        (lambda: sk.sinkhorn_expert_product_packed(x, w8._replace(values=odd), offsets), ValueError),
                        (lambda: sk.sinkhorn_expert_product_packed(x, w8._replace(columns=40), offsets), ValueError),
                        (lambda: sk.sinkhorn_expert_product_packed(x, w8._replace(scales=w8.scales[:1]), offsets), ValueError),
                        (lambda: sk.sinkhorn_expert_product_packed(x, w8, offsets, dtype=torch.float64), TypeError),
                        (lambda: sk.sinkhorn_expert_product_packed(x.cpu(), w8, offsets), TypeError),
                        (lambda: sk.sinkhorn_pack(x, 64), ValueError), (lambda: sk.sinkhorn_pack(x.int()), TypeError),
                        (lambda: sk.sinkhorn_unpack(w8, torch.int8), TypeError),
                        (lambda: sk.sinkhorn_pack(torch.zeros(3, 0, device="cuda")), ValueError)):
        with pytest.raises(error):
            call()


def test_a_gradient_through_a_packed_product_is_refused():
    x = make(8, 32, seed=1, dtype=BF16).requires_grad_()
    w8 = sk.sinkhorn_pack(make(16, 32, seed=2, dtype=BF16))
    y = sk.sinkhorn_expert_product_packed(x, w8)
    with torch.no_grad():
        assert torch.equal(sk.sinkhorn_expert_product_packed(x, w8), y)
    with pytest.raises(NotImplementedError):
        y.float().sum().backward()
    import torch.autograd.forward_ad as fwad
    with fwad.dual_level():
        dual = fwad.make_dual(x.detach(), torch.ones_like(x))
        with pytest.raises(RuntimeError, match="forward mode AD"):
            sk.sinkhorn_expert_product_packed(dual, w8)


# ---- activations ----

# Roundings in 32 bits of an activation's value and derivative, in units of the size of their terms: exp and erf within
# two units of their own, exp's argument rounded by half a unit of it, the quotient within two, and five products and
# sums; what enters a 1 + x (1 - p) or a 1 + erf is bounded by 1 + |x|.
ACT = 12 * U


def act_off(x, kind, gated):
    """Bounds of the activated rows, and of the two factors of their gradient."""
    v, u = x.chunk(2, -1) if gated else (x, torch.ones_like(x))
    return ACT * (1 + v.abs()) * (1 + v.abs()) * u.abs(), ACT * (1 + v.abs()) ** 2 * u.abs(), ACT * (1 + v.abs()) ** 2


def check_activation(x, kind, gated):
    x = x.clone().requires_grad_()
    y = sk.sinkhorn_activation(x, kind, gated)
    X = x.detach().cpu().double()
    want = ref.activate(X, kind, gated)
    off = act_off(X, kind, gated)[0]
    assert bool(((y.detach().cpu().double() - want).abs() <= off + rounding(want, x.dtype)).all())
    gy = make(*y.shape, seed=9, dtype=x.dtype)
    gx, = torch.autograd.grad(y, x, gy)
    kept = ref.unpack(*ref.pack(x, 128), 128).requires_grad_()
    a = ref.activate(kept, kind, gated)
    want, = torch.autograd.grad(a, kept, gy.cpu().double())
    G = gy.cpu().double().abs()
    _, d, e = act_off(kept.detach(), kind, gated)
    off = torch.cat((G * d, G * e), -1) if gated else G * d
    assert bool(((gx.cpu().double() - want).abs() <= off + rounding(want, x.dtype)).all())
    with torch.no_grad():
        assert torch.equal(sk.sinkhorn_activation(x, kind, gated), y)


@pytest.mark.parametrize("T,K", [(1, 1), (3, 5), (9, 8), (5, 60), (40, 128), (3, 200), (7, 256), (33, 1001), (2, 4096)])
@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_activation(T, K, kind, gated, dtype):
    check_activation(make(T, K * (1 + gated), seed=T + K, by=2.0, dtype=dtype), kind, gated)


@pytest.mark.parametrize("kind", ["relu", "silu", "gelu"])
def test_activation_far_from_zero(kind):
    x = torch.tensor([[-1e4, -200.0, -90.0, -87.0, -20.0, -5.0, -0.0, 0.0, 1e-30, 5.0, 20.0, 100.0, 1e4]], device="cuda")
    y = sk.sinkhorn_activation(x, kind)
    want = ref.activate(x.cpu().double(), kind, False)
    assert torch.isfinite(y).all()
    # exp's argument is rounded: its relative error there is |x| units
    assert bool(((y.cpu().double() - want).abs() <= 8 * U * (1 + x.cpu().double().abs()) * want.abs() + 1e-37).all())


def test_activation_of_more_dimensions():
    x = make(3, 4, 64, seed=1, dtype=BF16)
    assert torch.equal(sk.sinkhorn_activation(x, "silu", True),
                       sk.sinkhorn_activation(x.view(12, 64), "silu", True).view(3, 4, 32))
    assert sk.sinkhorn_activation(x[:0], "gelu").shape == (0, 4, 64)
    with pytest.raises(ValueError):
        sk.sinkhorn_activation(x[..., :5], "silu", True)
    with pytest.raises(ValueError):
        sk.sinkhorn_activation(x, "tanh")


# ---- products that keep their rows in 8 bits ----

def check_kept(T, E, k, K, N, kind, gated, dtype, in_order=False, none=0.1):
    """Forward against the product of the rows activated in 64 bits, gradients against those at the kept values.  The
    factors are activated rows rounded to 16 bits: half a step of each, beside the products' own sums."""
    if in_order:
        T, k = T * k, 1
        offsets = torch.tensor([0] + sorted(torch.randint(0, T + 1, (E,), generator=gen(3)).tolist()),
                               dtype=torch.int32).cuda()
        tokens = slots = None
    else:
        offsets, tokens, slots = routed(T, E, k, T + K, none=none)
    x = make(T, K * (1 + gated), seed=1, dtype=dtype).requires_grad_()
    w = make(E, N, K, seed=2, by=K ** -0.5, dtype=dtype).requires_grad_()
    gy = make(T * k, N, seed=3, dtype=dtype)
    y = sk.sinkhorn_expert_product_kept(x, w, offsets, tokens, slots, kind, gated)
    gx, gw = torch.autograd.grad(y, (x, w), gy)
    half = rounding(torch.ones(1, dtype=torch.float64), dtype)  # of a factor, relative (and below its range, absolute)
    o, t = offsets.cpu(), None if tokens is None else tokens.cpu()
    W, G = w.detach().cpu().double(), gy.cpu().double()
    X = x.detach().cpu().double()
    a = ref.activate(X, kind, gated)
    a_off = act_off(X, kind, gated)[0] + half * a.abs()
    p = products(a, W, o, t, G)
    sums = (K + N + T * k) * U  # at most so many roundings in a sum, of its absolute terms
    want = p["y"]
    off = products(a_off, W.abs(), o, t)["y"] + sums * p["abs_y"]
    assert bool(((y.detach().cpu().double() - want).abs() <= off + rounding(want, dtype)).all())
    kept = ref.unpack(*ref.pack(x, 128), 128).requires_grad_()
    b = ref.activate(kept, kind, gated)
    B = b.detach()
    b_off = act_off(kept.detach(), kind, gated)[0] + half * B.abs()
    p = products(B, W, o, t, G)
    off = products(b_off, W.abs(), o, t, G.abs())["gw"] + sums * p["abs_gw"]
    assert bool(((gw.cpu().double() - p["gw"]).abs() <= off + rounding(p["gw"], dtype)).all())
    # the gradient of the activated rows is rounded to 16 bits once before the activation's derivative
    ga = p["gx"]
    ga_off = sums * p["abs_gx"] + half * ga.abs() + 2.0 ** -25
    want, = torch.autograd.grad(b, kept, ga)
    _, d, e = act_off(kept.detach(), kind, gated)
    with torch.enable_grad():
        v = kept.detach().requires_grad_()
        slope = torch.autograd.grad(ref.activate(v, kind, gated).sum(), v)[0].abs()
    A = ga.abs()
    off = (torch.cat((A * d, A * e), -1) + torch.cat((ga_off, ga_off), -1) * slope) if gated else A * d + ga_off * slope
    assert bool(((gx.cpu().double() - want).abs() <= off + rounding(want, dtype)).all())
    with torch.no_grad():
        assert torch.equal(sk.sinkhorn_expert_product_kept(x, w, offsets, tokens, slots, kind, gated), y)


@pytest.mark.parametrize("T,E,k,K,N", [(1, 1, 1, 1, 1), (2, 3, 2, 8, 8), (5, 2, 1, 17, 9), (40, 4, 2, 64, 40),
                                       (70, 5, 3, 129, 33), (300, 3, 2, 256, 128), (600, 4, 2, 200, 136)])
@pytest.mark.parametrize("kind,gated", [("none", False), ("silu", True), ("gelu", False), ("relu", False), ("none", True)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_kept_product(T, E, k, K, N, kind, gated, dtype):
    check_kept(T, E, k, K, N, kind, gated, dtype)


@pytest.mark.parametrize("kind,gated", [("none", False), ("silu", True)])
@pytest.mark.parametrize("T,K,N", [(3, 24, 16), (500, 128, 200), (1000, 1024, 520)])
def test_kept_product_of_rows_in_order(T, K, N, kind, gated):
    check_kept(T, 4, 2, K, N, kind, gated, BF16, in_order=True)


def test_kept_rows_take_half_the_memory():
    """What a product keeps between its passes: its rows in 8 bits with their scales, and nothing else of that size."""
    T, K, N = 4096, 2048, 256
    w = make(2, N, K, seed=2, dtype=BF16).requires_grad_()
    offsets = torch.tensor([0, 1000, T], dtype=torch.int32).cuda()
    x = make(T, 2 * K, seed=1, dtype=BF16).requires_grad_()
    held = {}
    for name, gated, given in (("none", False, x[:, :K].contiguous()), ("silu", True, x)):
        before = torch.cuda.memory_allocated()
        y = sk.sinkhorn_expert_product_kept(given, w, offsets, activation=name, gated=gated)
        held[name] = torch.cuda.memory_allocated() - before - y.numel() * 2
        del y
    for name, columns in (("none", K), ("silu", 2 * K)):
        assert held[name] <= T * columns * (1 + 4 / 128) + (1 << 16), held


def test_kept_product_wants_one_gradient():
    x, w = make(90, 64, seed=1, dtype=BF16), make(3, 40, 32, seed=2, dtype=BF16)
    offsets = torch.tensor([0, 30, 50, 90], dtype=torch.int32).cuda()
    gy = make(90, 40, seed=3, dtype=BF16)
    for kind, gated in (("silu", True), ("none", False)):
        v = x if gated else x[:, :32].contiguous()

        def run(need_x, need_w):
            a, b = v.clone().requires_grad_(need_x), w.clone().requires_grad_(need_w)
            y = sk.sinkhorn_expert_product_kept(a, b, offsets, activation=kind, gated=gated)
            return torch.autograd.grad(y, [t for t in (a, b) if t.requires_grad], gy)
        both = run(True, True)
        assert torch.equal(run(True, False)[0], both[0]) and torch.equal(run(False, True)[0], both[1])


def test_kept_product_against_the_plain_one():
    """Without an activation the results are the product's own, and the gradient of the rows, too."""
    offsets, tokens, slots = routed(200, 4, 2, 5)
    x, w = rows(200, 96, 1, BF16).requires_grad_(), make(4, 72, 96, seed=2, dtype=BF16).requires_grad_()
    gy = make(400, 72, seed=3, dtype=BF16)
    a, b = (f(x, w, offsets, tokens, slots) for f in (sk.sinkhorn_expert_product_kept, sk.sinkhorn_expert_product))
    assert torch.equal(a, b)
    assert torch.equal(torch.autograd.grad(a, x, gy, retain_graph=True)[0], torch.autograd.grad(b, x, gy)[0])
    exact = sk.sinkhorn_unpack(sk.sinkhorn_pack(x, 128), BF16).requires_grad_()
    again = sk.sinkhorn_expert_product(exact, w, offsets, tokens, slots)
    assert torch.equal(torch.autograd.grad(a, w, gy)[0], torch.autograd.grad(again, w, gy)[0])


def test_refused_derivatives():
    x, w = make(8, 32, seed=1, dtype=BF16).requires_grad_(), make(1, 16, 32, seed=2, dtype=BF16).requires_grad_()
    offsets = torch.tensor([0, 8], dtype=torch.int32).cuda()
    for call in (lambda v: sk.sinkhorn_expert_product_kept(v, w, offsets, activation="silu"),
                 lambda v: sk.sinkhorn_activation(v, "silu")):
        g, = torch.autograd.grad(call(x).float().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(g.float().sum(), x)
        import torch.autograd.forward_ad as fwad
        with fwad.dual_level():
            with pytest.raises(RuntimeError, match="forward mode AD"):
                call(fwad.make_dual(x.detach(), torch.ones_like(x)))
    with pytest.raises(ValueError):
        sk.sinkhorn_expert_product_kept(x, w, offsets, activation="silu", gated=True)
    with pytest.raises(TypeError):
        sk.sinkhorn_expert_product_kept(x.float(), w.float(), offsets)


def test_on_another_stream():
    x = rows(500, 300, 1, BF16)
    w8 = sk.sinkhorn_pack(make(40, 300, seed=2, dtype=BF16))
    want = sk.sinkhorn_expert_product_packed(x, w8), sk.sinkhorn_unpack(sk.sinkhorn_pack(x, 128))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = (sk.sinkhorn_expert_product_packed(x, w8, stream=side),
           sk.sinkhorn_unpack(sk.sinkhorn_pack(x, 128, stream=side), stream=side))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
