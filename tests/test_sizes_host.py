"""Sizes that the C ABI's fields of 32 bits do not hold: refused, not cut off to what they would hold (no GPU needed)."""
import pytest

import paper_1907_01729_amd as sk
from paper_1907_01729_amd import _binding, routed

TOO_LARGE = [1 << 31, (1 << 32) + 4, (1 << 64) + 4, -(1 << 31) - 1, -(1 << 32) + 4]


def replaced(sizes, i, n):
    return (*sizes[:i], n, *sizes[i + 1:])


@pytest.mark.parametrize("n", TOO_LARGE)
@pytest.mark.parametrize("make,sizes,rest", [
    (routed._router, (4, 8, 2), (1, 1)), (routed._experts, (4, 2, 8, 16, 16), (1,)), (routed._combine, (4, 8, 2), (1,)),
    (_binding.problem, (4, 8, 8, 0), (0.1, 5)), (sk.sinkhorn_workspace_bytes, (4, 8, 8, 0), (0.1, 5)),
    (sk.sinkhorn_describe, (4, 8, 8, 0), (0.1, 5)), (sk.sinkhorn_points_workspace_bytes, (4, 8, 8, 0, 3), (0.1, 5))])
def test_sizes_are_not_cut_off(make, sizes, rest, n):
    make(*sizes, *rest)
    for i in range(len(sizes)):
        with pytest.raises(sk.SinkhornError) as refused:
            make(*replaced(sizes, i, n), *rest)
        assert refused.value.status == -2


@pytest.mark.parametrize("n", TOO_LARGE)
def test_iterations_are_not_cut_off(n):
    with pytest.raises(sk.SinkhornError) as refused:
        _binding.problem(4, 8, 8, 0, 0.1, n)
    assert refused.value.status == -4


def test_the_largest_that_fit():
    p = _binding.problem((1 << 31) - 1, 1, -(1 << 31), 1, 0.1, (1 << 31) - 1)
    assert (p.B, p.d2, p.n_iter) == ((1 << 31) - 1, -(1 << 31), (1 << 31) - 1)
    with pytest.raises(sk.SinkhornError):
        sk.sinkhorn_describe((1 << 31) - 1, 1, -(1 << 31), 1, 0.1, 5)
