"""The norms, the routed layer's products with kept rows, and the same layer served in 8 bits, as a block uses them."""
import os
import sys

import pytest
import torch

import paper_1907_01729_amd as sk

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def block(dim=64, hidden=96, experts=8):
    from routed_layer import RoutedBlock
    torch.manual_seed(3)
    b = RoutedBlock(dim, hidden, experts)
    with torch.no_grad():
        for p in (b.first, b.after, b.before, b.open):
            p.add_(0.2 * torch.randn_like(p))
    return b.eval()


def rows(T, dim=64, seed=0):
    return torch.randn(T, dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16()


def test_the_example_runs_as_a_block(capsys):
    from routed_layer import main
    losses, spread = main(steps=4, tokens=256, dim=64, experts=8, block=True)
    assert len(losses) == len(spread) == 4 and all(l == l and abs(l) < float("inf") for l in losses)
    assert "served in 8 bits" in capsys.readouterr().out


@pytest.mark.parametrize("T", [1, 7, 300])
def test_the_fused_block_against_its_parts(T):
    """The same block of separate calls: norms one by one, products that keep 16 bits, the activation in torch.  The
    gradients differ by the rows' 8 bits (half of 1/127 of the largest of 128 numbers, about 3 of them: 1 % of a number
    of about one) and by 16-bit roundings (2^-9 each, a dozen of them, 2 %): 6 % of a gradient's norm holds both."""
    b, x = block(), rows(T, seed=T)
    g = torch.randn_like(x)

    def parts(x):
        f = lambda t: t.float()  # noqa: E731

        def norm(v, w):
            return (f(v) * torch.rsqrt(f(v).square().mean(1, keepdim=True) + 1e-6) * f(w)).bfloat16()
        n = norm(x, b.first)
        r = b.route(n, True)
        h = sk.sinkhorn_expert_product(n, b.w1, r.offsets, r.tokens, r.slots)
        v, u = f(h).chunk(2, 1)
        z = sk.sinkhorn_expert_product((torch.nn.functional.silu(v) * u).bfloat16(), b.w2, r.offsets)
        z = sk.sinkhorn_expert_combine(z, r.weights, r.slots, r.offsets)
        out = (b.scale * f(x) + b.open * f(norm(z, b.after))).bfloat16()
        return norm(out, b.before)
    names = ["x"] + [n for n, p in b.named_parameters()]
    a1, a2 = x.clone().requires_grad_(), x.clone().requires_grad_()
    y1, y2 = b(a1, 0)[0], parts(a2)
    assert float((y1.float() - y2.float()).norm() / y2.float().norm()) < 0.02
    g1 = torch.autograd.grad(y1, [a1, *b.parameters()], g)
    g2 = torch.autograd.grad(y2, [a2, *b.parameters()], g)
    for name, u, v in zip(names, g1, g2):
        assert u.dtype == v.dtype and float((u.float() - v.float()).norm()) <= 0.06 * float(v.float().norm()), name


@pytest.mark.parametrize("T", [1, 5, 64, 900])
def test_served_in_8_bits(T):
    """Rows and weights rounded to 127 steps of their largest number, of about three times the rest: each factor is off by
    about 0.7 % (a uniform half step, 3 / 127 / sqrt 12), the result of two products by the root of four such terms
    and the gated activation's product: 3 % holds it."""
    b, x = block(), rows(T, seed=T)
    with torch.no_grad():
        want = b(x, 0)[0].float()
    got = b.serve(x, b.packed())
    assert got.dtype == torch.bfloat16 and float((got.float() - want).norm() / want.norm()) < 0.03


@pytest.mark.parametrize("T", [4, 500])
def test_serving_in_a_graph(T):
    """Captured once, replayed on new tokens with the program's own work between."""
    b, x = block(), rows(T)
    packed = b.packed()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            b.serve(x, packed, False)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = b.serve(x, packed, False)
    for seed in range(4):
        x.copy_(rows(T, seed=50 + seed))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, b.serve(x, packed, False))


def test_training_in_a_graph():
    """Forward and backward of the block captured together, replayed on new inputs."""
    b = block()
    x = rows(200).requires_grad_()
    g = torch.randn_like(x)
    leaves = [x, *b.parameters()]

    def step():
        y = b(x, 0, False)[0]
        return [y, *torch.autograd.grad(y, leaves, g)]
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
            x.copy_(rows(200, seed=70 + seed))
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(got, step()):
            assert torch.equal(u, v)


def test_two_backward_passes_and_a_released_graph():
    b, x = block(), rows(40).requires_grad_()
    y = b(x, 0)[0]
    g = torch.ones_like(y)
    first = torch.autograd.grad(y, x, g, retain_graph=True)[0]
    assert torch.equal(torch.autograd.grad(y, x, g)[0], first)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y, x, g)
    for call in (lambda v: sk.sinkhorn_norm(v), lambda v: sk.sinkhorn_residual_norm(v, v), lambda v: sk.sinkhorn_activation(v, "silu"),
                 lambda v: sk.sinkhorn_residual_norm(v, v, before=sk.Norm())[1]):
        y = call(x)
        torch.autograd.grad(y, x, g)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(y, x, g)


def test_one_tensor_as_both_inputs():
    """h and residual the same leaf: the gradient is the sum of both."""
    x = rows(30).float().requires_grad_()
    g = torch.randn_like(x)
    got, = torch.autograd.grad(sk.sinkhorn_residual_norm(x, x), x, g)
    assert torch.equal(got, 2 * g)
    got, = torch.autograd.grad(sk.sinkhorn_residual_norm(x, x, scale=0.5), x, g)
    assert torch.equal(got, 1.5 * g)


def test_a_changed_sum_is_noticed():
    """The next norm's gradient needs the sum as it was."""
    x, w = rows(20).requires_grad_(), torch.ones(64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    out, n = sk.sinkhorn_residual_norm(x, x.detach(), before=sk.Norm(w))
    with torch.no_grad():
        out.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        n.float().sum().backward()


def test_calls_under_inference_mode_and_many_threads():
    import threading
    b, x = block(), rows(64)
    packed = b.packed()
    want = b.serve(x, packed)
    with torch.inference_mode():
        assert torch.equal(b.serve(x.clone(), packed), want)
    got = [None] * 4

    def work(i):
        for _ in range(10):
            got[i] = b.serve(x, packed)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    for v in got:
        assert torch.equal(v, want)


def test_on_another_stream():
    """Forward and backward on a side stream, what they leave behind used there again at once."""
    b, x = block(), rows(300).requires_grad_()
    g = torch.randn_like(x)
    leaves = [x, *b.parameters()]
    want = torch.autograd.grad(b(x, 0)[0], leaves, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(5):
            got = torch.autograd.grad(b(x, 0)[0], leaves, g)
            torch.full((1 << 20,), float("nan"), device="cuda")  # takes what was freed
    torch.cuda.synchronize()
    for u, v in zip(got, want):
        assert torch.equal(u, v)


def test_what_is_kept_goes_through_hooks_on_saved_tensors():
    """Saved on the host and brought back: the same gradients, and nothing of the rows' size left on the GPU."""
    b, x = block(), rows(4000).requires_grad_()
    g = torch.randn_like(x)
    leaves = [x, *b.parameters()]
    want = torch.autograd.grad(b(x, 0)[0], leaves, g)
    seen = []

    def pack(t):
        seen.append(t.dtype)
        return t.to("cpu")
    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.to("cuda")):
        y = b(x, 0)[0]
    got = torch.autograd.grad(y, leaves, g)
    assert torch.int8 in seen
    for u, v in zip(got, want):
        assert torch.equal(u, v)
    for call in (lambda: sk.sinkhorn_norm(x), lambda: sk.sinkhorn_residual_norm(x, x, before=sk.Norm())[1],
                 lambda: sk.sinkhorn_activation(x, "silu")):
        want, = torch.autograd.grad(call(), x, g)
        call()
        before = torch.cuda.memory_allocated()
        with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.to("cuda")):
            y = call()
        assert torch.cuda.memory_allocated() - before <= 2 * y.numel() * y.element_size()  # y, and what it is the norm of
        assert torch.equal(torch.autograd.grad(y, x, g)[0], want)


def test_under_a_checkpoint():
    from torch.utils.checkpoint import checkpoint
    b, x = block(), rows(4000).requires_grad_()
    g = torch.randn_like(x)
    leaves = [x, *b.parameters()]
    y = b(x, 0)[0]
    want = torch.autograd.grad(y, leaves, g)
    before = torch.cuda.memory_allocated()
    again = checkpoint(lambda v: b(v, 0)[0], x, use_reentrant=False)
    # The result alone is left, up to what the allocator rounds.
    assert torch.cuda.memory_allocated() - before <= y.numel() * y.element_size() + 4096
    assert torch.equal(again, y)
    for u, v in zip(torch.autograd.grad(again, leaves, g), want):
        assert torch.equal(u, v)


def test_a_captured_backward_pass_beside_an_eager_graph_is_refused():
    """The default stream cannot wait for a captured one; once the eager graph is gone the capture goes through."""
    x = rows(40).requires_grad_()
    w = torch.ones(1, 64, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    offsets = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    g = torch.randn_like(x)
    for call in (lambda: sk.sinkhorn_norm(x), lambda: sk.sinkhorn_residual_norm(x, x), lambda: sk.sinkhorn_activation(x, "silu"),
                 lambda: sk.sinkhorn_expert_product_kept(x, w, offsets)):
        eager = call()
        want, = torch.autograd.grad(eager, x, g, retain_graph=True)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(RuntimeError, match="cannot be captured"):
            with torch.cuda.graph(graph):
                torch.autograd.grad(call(), x, g)
        del eager, graph
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got, = torch.autograd.grad(call(), x, g)
        for _ in range(3):
            got.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want)
