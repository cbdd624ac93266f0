"""The bounds of the router's gradient tests, on the CPU: the formula against differentiation, and what they can see."""
import pytest
import torch

import routed_terms

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("T,E,k", routed_terms.SIZES[:5])
def test_formula_against_differentiation(T, E, k):
    logits, mask, renormalize, want, gw, gb, gz = routed_terms.case(T, E, k, F32)
    got = routed_terms.terms(logits, k, want, mask, renormalize, gw, gb, gz)
    for name, incoming in (("weights", gw.double()), ("balance", torch.tensor(gb).double()),
                           ("z_loss", torch.tensor(gz).double())):
        grad, = torch.autograd.grad(want[name], (want["logits"],), incoming, retain_graph=True)
        # in 64 bits both, and the scalars of the incoming gradients in 32
        assert ((grad - got[name][0]).abs() <= 1e-6 * got[name][0].abs() + 1e-12).all(), name


@pytest.mark.parametrize("T,E,k", routed_terms.SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_wrong_term_is_seen(T, E, k, dtype):
    """A term left out, taken twice, with another expert's count or another number of tokens leaves its bound."""
    logits, mask, renormalize, want, gw, gb, gz = routed_terms.case(T, E, k, dtype)
    right = routed_terms.terms(logits, k, want, mask, renormalize, gw, gb, gz)
    n = int(mask.sum())
    more = routed_terms.terms(logits, k, want, mask, renormalize, gw, gb, gz, tokens=n + max(1, n // 30))
    rolled = routed_terms.terms(logits, k, want, mask, renormalize, gw, gb, gz,
                                count_of=want["counts"].double().roll(1))

    def seen(name, planted):
        value, bound = right[name]
        off = ((planted - value).abs() > bound) & (value != 0)
        return float(off.sum()) / float((value != 0).sum())

    for name in ("weights", "balance", "z_loss"):
        value = right[name][0]
        assert seen(name, torch.zeros_like(value)) > 0.9 and seen(name, 2 * value) > 0.9, name
    assert seen("z_loss", more["z_loss"][0]) > 0.9
    assert seen("balance", more["balance"][0]) > 0.5
    assert seen("balance", rolled["balance"][0]) > 0.5
