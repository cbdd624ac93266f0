"""The norms around a block against their formulas in 64 bits: forward, gradients, odd sizes, every gate, and the ways in
which a program calls them."""
import pytest
import torch

import norm_util as ref
import paper_1907_01729_amd as sk

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def gen(seed):
    return torch.Generator().manual_seed(seed)


def make(*shape, seed, dtype=F32, by=1.0, plus=0.0):
    return (by * torch.randn(*shape, generator=gen(seed)) + plus).to(dtype).cuda()


def rows(T, N, seed, dtype):
    """Columns of different sizes."""
    return (make(T, N, seed=seed) * torch.exp(0.7 * make(N, seed=seed + 1))).to(dtype)


def norm_of(N, wdtype, center, eps, seed, bias=True):
    return sk.Norm(make(N, seed=seed, by=0.3, plus=1.0, dtype=wdtype),
                   make(N, seed=seed + 1, by=0.3, dtype=wdtype) if bias else None, eps, center)


def check_norm(T, N, dtype, wdtype, center, eps=1e-5, bias=True, x=None):
    x = rows(T, N, 3, dtype) if x is None else x
    norm = norm_of(N, wdtype, center, eps, 5, bias)
    gy = make(T, N, seed=7, dtype=dtype)
    leaves = [t.requires_grad_() for t in (x, norm.weight, norm.bias) if t is not None]
    y = sk.sinkhorn_norm(x, norm)
    grads = torch.autograd.grad(y, leaves, gy)
    X, w, b = ref.double(x), ref.double(norm.weight), ref.double(norm.bias)
    want, off = ref.forward(X, w, b, eps, center, dtype)
    ref.close(y, want, off)
    back = ref.backward(X, w, eps, center, ref.double(gy))
    for g, n in zip(grads, "xwb"):
        ref.close(g, *back[n])
    with torch.no_grad():
        assert torch.equal(sk.sinkhorn_norm(x, norm), y)


@pytest.mark.parametrize("T,N", [(1, 1), (3, 1), (1, 7), (5, 8), (65, 9), (33, 64), (7, 65), (100, 100), (3, 127), (19, 129),
                                 (2, 511), (9, 513), (4, 1000), (17, 1001), (3, 2048), (2, 4096), (3, 4104), (5, 8191),
                                 (3, 8192)])
@pytest.mark.parametrize("dtype,wdtype,center", [(BF16, BF16, False), (F16, F32, True), (F32, F32, True)])
def test_norm(T, N, dtype, wdtype, center):
    check_norm(T, N, dtype, wdtype, center)


@pytest.mark.parametrize("T,N", [(3, 8193), (2, 8200), (5, 20003), (1, 65536)])
@pytest.mark.parametrize("dtype,center", [(BF16, False), (F32, True)])
def test_rows_wider_than_a_work_group(T, N, dtype, center):
    check_norm(T, N, dtype, dtype, center)


@pytest.mark.parametrize("T,N,dtype", [(3000, 24, BF16), (700, 520, F32), (2500, 1024, F16), (1100, 4100, BF16)])
@pytest.mark.parametrize("bias", [True, False])
def test_many_rows(T, N, dtype, bias):
    """More rows than groups, so that each goes through several."""
    check_norm(T, N, dtype, dtype, bias, bias=bias)


def test_without_weight_and_bias():
    x = rows(6, 33, 3, F32).requires_grad_()
    y = sk.sinkhorn_norm(x)
    want, off = ref.forward(ref.double(x), None, None, 1e-6, False, F32)
    ref.close(y, want, off)
    gy = make(6, 33, seed=1)
    gx, = torch.autograd.grad(y, x, gy)
    ref.close(gx, *ref.backward(ref.double(x), None, 1e-6, False, ref.double(gy))["x"])


@pytest.mark.parametrize("center", [False, True])
def test_far_means_and_constant_rows(center):
    """A mean far from zero does not eat the variance; a row of one value has r = 1 / sqrt(eps)."""
    x = make(8, 300, seed=2, plus=1000.0)
    x[3] = 5.0
    x[4] = 0.0
    check_norm(8, 300, F32, F32, center, x=x)


def test_what_is_not_finite_stays_in_its_row():
    x = rows(40, 200, 3, BF16)
    norm = norm_of(200, BF16, True, 1e-5, 5)
    want = sk.sinkhorn_norm(x, norm)
    x[7, 3], x[9, 199], x[39, 0] = float("nan"), float("inf"), -float("inf")
    got = sk.sinkhorn_norm(x, norm)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[7, 9, 39]] = True
    assert torch.equal(got[~bad], want[~bad])
    assert got[bad].isnan().any(1).all()


def formula(h, residual, gate, scale, after, before, dtype):
    """The sum before its rounding, and its bound."""
    off = torch.zeros_like(h)
    n = h
    if after is not None:
        n, off = ref.forward(h, ref.double(after.weight), ref.double(after.bias), after.eps, after.center, F32)
    g = 1.0 if gate is None else gate
    size = (scale * residual).abs() + (g * n).abs()
    return scale * residual + g * n, n, off * (g if gate is None else g.abs()) + 4 * ref.U * size


def check_block(T, N, dtype, wdtype, gate, gdtype, after, before, scale=0.7, use_out=True, use_next=True, bias=True):
    h, residual = rows(T, N, 3, dtype).requires_grad_(), rows(T, N, 11, dtype).requires_grad_()
    shape = {"none": None, "token": (T, 1), "channel": (1, N), "full": (T, N)}[gate]
    gate = None if shape is None else make(*shape, seed=13, dtype=gdtype).requires_grad_()
    after = norm_of(N, wdtype, after == "centred", 1e-5, 15, bias) if after else None
    before = norm_of(N, wdtype, before == "centred", 1e-3, 17, bias) if before else None
    parameters = [t.requires_grad_() for n in (after, before) if n is not None for t in (n.weight, n.bias)
                  if t is not None]
    got = sk.sinkhorn_residual_norm(h, residual, gate, scale, after, before)
    out, normed = (got, None) if before is None else got
    H, R, G = ref.double(h), ref.double(residual), ref.double(gate)
    total, n, off = formula(H, R, G, scale, after, before, dtype)
    ref.close(out, total, off)
    g_out = make(T, N, seed=19, dtype=dtype) if use_out else None
    g_next = make(T, N, seed=21, dtype=dtype) if use_next and before is not None else None
    outputs = [(o, g) for o, g in ((out, g_out), (normed, g_next)) if g is not None]
    leaves = [t for t in (h, residual, gate, *parameters) if t is not None]
    grads = torch.autograd.grad([o for o, _ in outputs], leaves, [g for _, g in outputs], allow_unused=True)
    O = ref.double(out)  # the next norm is of the rounded sum
    g = torch.zeros_like(H) if g_out is None else ref.double(g_out)
    g_off = torch.zeros_like(H)
    want = {}
    if before is not None:
        w, b = ref.double(before.weight), ref.double(before.bias)
        y, y_off = ref.forward(O, w, b, before.eps, before.center, dtype)
        ref.close(normed, y, y_off)
        gn = torch.zeros_like(H) if g_next is None else ref.double(g_next)
        back = ref.backward(O, w, before.eps, before.center, gn)
        g, g_off = g + back["x"][0], back["x"][1] + 2 * ref.U * (g.abs() + back["x"][0].abs())
        want.update(before_w=back["w"], before_b=back["b"])
    want["residual"] = scale * g, abs(scale) * g_off + ref.U * (scale * g).abs()
    gate_of = torch.ones_like(H[:1]) if G is None else G
    dn, dn_off = gate_of * g, gate_of.abs() * g_off + ref.U * (gate_of * g).abs()
    if G is not None:
        n_off = off / gate_of.abs().clamp(min=1e-300)  # of n, and more
        d, d_off = g * n, g_off * n.abs() + g.abs() * n_off + ref.U * (g * n).abs()
        dims = [i for i in (0, 1) if G.shape[i] != H.shape[i]]
        if dims:
            d_off = (d_off + (ref.D + T) * ref.U * d.abs()).sum(dims, keepdim=True)
            d = d.sum(dims, keepdim=True)
        want["gate"] = d, d_off
    if after is not None:
        back = ref.backward(H, ref.double(after.weight), after.eps, after.center, dn, dn_off)
        want.update(h=back["x"], after_w=back["w"], after_b=back["b"])
    else:
        want["h"] = dn, dn_off
    names = ["h", "residual"] + ["gate"] * (G is not None)
    for name, norm in (("after", after), ("before", before)):
        if norm is not None:
            names += [name + "_w"] + [name + "_b"] * (norm.bias is not None)
    assert len(names) == len(grads)
    for name, got in zip(names, grads):
        ref.close(got, *want[name])
    with torch.no_grad():
        again = sk.sinkhorn_residual_norm(h, residual, gate, scale, after, before)
    assert torch.equal(again if before is None else again[0], out)
    assert before is None or torch.equal(again[1], normed)


@pytest.mark.parametrize("gate,gdtype", [("none", F32), ("token", F32), ("token", BF16), ("channel", BF16),
                                         ("channel", F32), ("full", BF16), ("full", F32)])
@pytest.mark.parametrize("after,before", [("rms", "rms"), ("centred", ""), ("", "centred"), ("", "")])
def test_block_gates(gate, gdtype, after, before):
    check_block(37, 100, BF16, BF16, gate, gdtype, after, before)


@pytest.mark.parametrize("T,N", [(1, 1), (2, 1), (1, 9), (1, 64), (67, 17), (130, 65), (9, 520), (600, 1001), (4, 4096),
                                 (3, 8192), (2, 8193), (3, 10000)])
@pytest.mark.parametrize("dtype,wdtype,gate,kinds", [(BF16, F32, "token", ("rms", "rms")),
                                                     (F16, F16, "full", ("centred", "rms")),
                                                     (F32, F32, "channel", ("rms", "centred"))])
def test_block_sizes(T, N, dtype, wdtype, gate, kinds):
    check_block(T, N, dtype, wdtype, gate, F32 if gate == "token" else dtype, *kinds)


@pytest.mark.parametrize("T,N", [(3000, 48), (1500, 1000), (800, 4096), (300, 8000)])
@pytest.mark.parametrize("gate,bias", [("none", False), ("token", False), ("channel", True)])
def test_block_many_rows(T, N, gate, bias):
    check_block(T, N, BF16, BF16, gate, F32, "rms", "rms", bias=bias)


@pytest.mark.parametrize("N", [60, 9000])
@pytest.mark.parametrize("use_out,use_next", [(True, False), (False, True)])
def test_a_gradient_from_one_side_only(N, use_out, use_next):
    check_block(20, N, F32, F32, "channel", F32, "rms", "centred", use_out=use_out, use_next=use_next)


def test_against_differences():
    """The gradients by central differences of a sum of the outputs in 32 bits.  A step of 2^-6 leaves an error of the
    third derivative, below 2^-12 times the size of terms that are about one, and one of 2^-24 2^6 times the sum's size,
    about a hundred: 2e-3 of gradients of about one holds both."""
    T, N = 3, 20
    t = {"h": make(T, N, seed=1), "residual": make(T, N, seed=2), "gate": make(T, 1, seed=3),
         "aw": make(N, seed=4, plus=1.0), "ab": make(N, seed=5), "bw": make(N, seed=6, plus=1.0), "bb": make(N, seed=7)}
    weigh = make(T, N, seed=8), make(T, N, seed=9)

    def total(v):
        o, n = sk.sinkhorn_residual_norm(v["h"], v["residual"], v["gate"], 0.8, sk.Norm(v["aw"], v["ab"], 1e-3, True),
                                         sk.Norm(v["bw"], v["bb"], 1e-3))
        return (o.double() * weigh[0]).sum() + (n.double() * weigh[1]).sum()
    leaves = {n: v.clone().requires_grad_() for n, v in t.items()}
    grads = dict(zip(leaves, torch.autograd.grad(total(leaves), list(leaves.values()))))
    for n, v in t.items():
        for i in range(0, v.numel(), max(1, v.numel() // 5)):
            step = torch.zeros_like(v).view(-1)
            step[i] = 2.0 ** -6
            step = step.view_as(v)
            up, down = total({**t, n: v + step}), total({**t, n: v - step})
            slope, got = float(up - down) * 2.0 ** 5, float(grads[n].view(-1)[i])
            assert abs(slope - got) <= 4e-3 * max(1.0, abs(got)), (n, i, slope, got)


def test_strided_inputs_and_gradients():
    N = 96
    wide = make(10, 2 * N, seed=1, dtype=BF16)
    h, residual = wide[:, ::2], wide.t()[:N].t()[:10]
    assert not h.is_contiguous()
    w = make(2 * N, seed=2, dtype=BF16)[::2]
    norm = sk.Norm(w, None, 1e-5)
    want = sk.sinkhorn_residual_norm(h.contiguous(), residual.contiguous(), after=sk.Norm(w.contiguous(), None, 1e-5))
    assert torch.equal(sk.sinkhorn_residual_norm(h, residual, after=norm), want)
    x = h.clone().requires_grad_()
    y = sk.sinkhorn_norm(x, norm)
    g1, = torch.autograd.grad(y.sum(), x)  # an expanded gradient
    g2, = torch.autograd.grad(sk.sinkhorn_norm(x, norm), x, torch.ones_like(y))
    assert torch.equal(g1, g2)


@pytest.mark.parametrize("shift", [1, 3, 8])
def test_unaligned_rows(shift):
    """Rows that begin at any element."""
    T, N = 5, 264
    store = make(T * N + shift, seed=1, dtype=BF16)
    x = store[shift:].view(T, N)
    norm = norm_of(N, BF16, False, 1e-5, 5)
    assert torch.equal(sk.sinkhorn_norm(x, norm), sk.sinkhorn_norm(x.clone(), norm))


def test_no_rows():
    w = make(8, seed=1).requires_grad_()
    x = torch.zeros(0, 8, device="cuda", requires_grad=True)
    gate = torch.ones(1, 8, device="cuda", requires_grad=True)
    o, n = sk.sinkhorn_residual_norm(x, x, gate, after=sk.Norm(w), before=sk.Norm(w))
    gx, gg, gw = torch.autograd.grad((o, n), (x, gate, w), (o, n))
    assert gx.shape == (0, 8) and not gg.any() and not gw.any()
    assert sk.sinkhorn_norm(x, sk.Norm(w)).shape == (0, 8)


def test_raw_calls_and_workspace():
    T, N = 300, 200
    x, gy = rows(T, N, 1, BF16), make(T, N, seed=2, dtype=BF16)
    norm = norm_of(N, BF16, True, 1e-5, 3)
    y, stats = sk.sinkhorn_norm_forward(x, norm)
    assert torch.equal(y, sk.sinkhorn_norm(x, norm))
    first = sk.sinkhorn_norm_backward(x, norm, stats, gy)
    space = torch.full((1 << 22,), 0xFF, dtype=torch.uint8, device="cuda")
    for a, b in zip(first, sk.sinkhorn_norm_backward(x, norm, stats, gy, workspace=space)):
        assert torch.equal(a, b)
    gate = make(1, N, seed=4)
    out, nxt, stats = sk.sinkhorn_residual_norm_forward(x, gy, gate, 0.5, norm, norm)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = sk.sinkhorn_residual_norm_backward(x, out, stats, gy, gy, gate, 0.5, norm, norm)
    b = sk.sinkhorn_residual_norm_backward(x, out, stats, gy, gy, gate, 0.5, norm, norm, workspace=space, stream=side)
    torch.cuda.synchronize()
    for u, v in zip(a, b):
        assert torch.equal(u, v)


def test_forward_and_backward_in_a_graph():
    T, N = 700, 520
    t = [rows(T, N, 1, BF16), rows(T, N, 2, BF16), make(T, 1, seed=3), make(N, seed=4, plus=1.0, dtype=BF16),
         make(N, seed=5, plus=1.0, dtype=BF16)]
    for v in t:
        v.requires_grad_()
    g = make(T, N, seed=6, dtype=BF16)

    def step():
        y = sk.sinkhorn_residual_norm(*t[:3], 0.9, sk.Norm(t[3]), sk.Norm(t[4]))
        return [*y, *torch.autograd.grad(y, t, (g, g))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in range(4):
        with torch.no_grad():
            for v in t:
                v.copy_(v.flip(0) * 1.25)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_only_what_is_wanted():
    """Each input's gradient alone is the same as among all."""
    T, N = 90, 130
    t = [rows(T, N, 1, F32), rows(T, N, 2, F32), make(1, N, seed=3), *(make(N, seed=4 + i) for i in range(4))]

    def run(v):
        return sk.sinkhorn_residual_norm(*v[:3], 0.9, sk.Norm(v[3], v[4]), sk.Norm(v[5], v[6], center=True))
    g = make(T, N, seed=9), make(T, N, seed=10)
    every = torch.autograd.grad(run([v.requires_grad_() for v in t]), t, g)
    for i in range(len(t)):
        for j, v in enumerate(t):
            v.requires_grad_(j == i)
        one, = torch.autograd.grad(run(t), t[i:i + 1], g)
        assert torch.equal(one, every[i])


def test_second_derivatives_and_tangents_are_refused():
    x = make(4, 16, seed=1).requires_grad_()
    w = make(16, seed=2).requires_grad_()
    for call in (lambda: sk.sinkhorn_norm(x, sk.Norm(w)),
                 lambda: sk.sinkhorn_residual_norm(x, x * 2, after=sk.Norm(w))):
        g, = torch.autograd.grad(call().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(g.sum(), x)
    import torch.autograd.forward_ad as fwad
    with fwad.dual_level():
        dual = fwad.make_dual(x.detach(), torch.ones_like(x))
        with pytest.raises(RuntimeError, match="forward mode AD"):
            sk.sinkhorn_norm(dual)
        with pytest.raises(RuntimeError, match="forward mode AD"):
            sk.sinkhorn_residual_norm(x.detach(), dual)


def test_wrong_arguments():
    x, w = make(4, 16, seed=1), make(16, seed=2)
    for call, error in ((lambda: sk.sinkhorn_norm(x[0]), ValueError), (lambda: sk.sinkhorn_norm(x, sk.Norm(w[:8])), ValueError),
                        (lambda: sk.sinkhorn_norm(x, sk.Norm(w.half())), TypeError),
                        (lambda: sk.sinkhorn_norm(x.half(), sk.Norm(w, w.half())), TypeError),
                        (lambda: sk.sinkhorn_norm(x.double()), TypeError),
                        (lambda: sk.sinkhorn_norm(x, sk.Norm(w, eps=-1.0)), sk.SinkhornError),
                        (lambda: sk.sinkhorn_norm(x, sk.Norm(w, eps=float("nan"))), sk.SinkhornError),
                        (lambda: sk.sinkhorn_residual_norm(x, x[:2]), ValueError),
                        (lambda: sk.sinkhorn_residual_norm(x, x.half()), TypeError),
                        (lambda: sk.sinkhorn_residual_norm(x, x, gate=w), ValueError),
                        (lambda: sk.sinkhorn_residual_norm(x, x, gate=x.half()), TypeError),
                        (lambda: sk.sinkhorn_residual_norm(x, x, scale=float("inf")), sk.SinkhornError),
                        (lambda: sk.sinkhorn_residual_norm(x, x, after=sk.Norm(w.cpu())), TypeError)):
        with pytest.raises(error):
            call()


def test_a_plain_sum_has_one_gradient_for_both():
    """out = residual + h: the gradients are equal, whichever are asked for; with a scale they are not."""
    T, N = 70, 96
    h, residual, w = rows(T, N, 1, BF16), rows(T, N, 2, BF16), make(N, seed=3, plus=1.0, dtype=BF16).requires_grad_()
    g = make(T, N, seed=4, dtype=BF16)

    def grads(need, scale=1.0):
        a, b = h.clone().requires_grad_(need[0]), residual.clone().requires_grad_(need[1])
        y = sk.sinkhorn_residual_norm(a, b, scale=scale, before=sk.Norm(w))
        return torch.autograd.grad(y, [t for t in (a, b) if t.requires_grad], (g, g))
    both = grads((True, True))
    assert torch.equal(*both)
    assert torch.equal(grads((True, False))[0], both[0]) and torch.equal(grads((False, True))[0], both[0])
    a, b = grads((True, True), 0.5)
    assert torch.equal((0.5 * a.float()).to(BF16), b)
    x = h.clone().requires_grad_()  # accumulated in place, the two do not disturb each other
    y = residual.clone().requires_grad_()
    for _ in range(2):
        o, n = sk.sinkhorn_residual_norm(x, y, before=sk.Norm(w.detach()))
        torch.autograd.backward((o, n), (g, g))
    want = (2 * both[0].float()).to(BF16)
    assert torch.equal(x.grad, want) and torch.equal(y.grad, want)


def test_more_than_2_to_the_32_bytes():
    """Rows whose bytes 32 bits do not count: those at the end are their own, forward and backward."""
    T, N = 540000, 4096
    h, w = torch.zeros(T, N, device="cuda", dtype=BF16), make(N, seed=1, plus=1.0, dtype=BF16)
    h[:4], h[-4:] = rows(4, N, 3, BF16), rows(4, N, 5, BF16)
    few = torch.cat((h[:4], h[-4:])).requires_grad_()
    norm = sk.Norm(w, None, 1e-3)
    small = sk.sinkhorn_residual_norm(few, few.detach(), None, 0.5, norm, norm)
    g = torch.zeros_like(h)
    g[:4], g[-4:] = rows(4, N, 7, BF16), rows(4, N, 9, BF16)
    want, = torch.autograd.grad(small, few, [torch.cat((g[:4], g[-4:]))] * 2)
    h.requires_grad_()
    large = sk.sinkhorn_residual_norm(h, h.detach(), None, 0.5, norm, norm)
    for a, b in zip(large, small):
        assert torch.equal(torch.cat((a[:4], a[-4:])), b)
        assert not a[4:-4].any()
    got, = torch.autograd.grad(large, h, [g] * 2)
    assert torch.equal(torch.cat((got[:4], got[-4:])), want) and not got[4:-4].any()


@pytest.mark.parametrize("T,N", [(2, 16392), (1, 33000), (3, 40001)])
@pytest.mark.parametrize("dtype,kinds", [(BF16, ("rms", "rms")), (F32, ("centred", "centred")), (F16, ("", "rms"))])
def test_block_ends_of_very_wide_rows(T, N, dtype, kinds):
    """More columns than the lanes hold: the sum is read again from where it has been written."""
    check_block(T, N, dtype, dtype, "none", F32, *kinds)


def test_many_wide_rows():
    """Several rows to a work-group whose sums lie in memory."""
    check_block(600, 8200, BF16, BF16, "channel", BF16, "centred", "rms")
    check_norm(530, 9001, F32, F32, True)
