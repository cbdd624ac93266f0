"""Weight gradients of few small matrices over many rows are summed in parts at any width (no GPU needed)."""
import pytest

from paper_1907_01729_amd.routed import _experts


@pytest.mark.parametrize("E,K,N", [(2, 127, 128), (2, 128, 127), (1, 1, 1), (8, 512, 511), (4, 767, 768)])
def test_odd_widths_have_parts(E, K, N):
    T = 8192 * E
    even = _experts(T, 1, E, K + -K % 8, N + -N % 8, 1)[2]
    odd = _experts(T, 1, E, K, N, 1)[2]
    assert odd // (E * K * N * 4) == even // (E * (K + -K % 8) * (N + -N % 8) * 4) > 1 and odd % (E * K * N * 4) == 0
