"""None in the place of a tensor is refused by name (no GPU needed)."""
import pytest
import torch

import paper_1907_01729_amd as sk

X = torch.zeros(4, 8)
EIGHT = sk.Packed(torch.zeros(2, 8, 16, dtype=torch.int8), torch.zeros(2, 8), 8)
OFFSETS = torch.zeros(3, dtype=torch.int32)


def test_no_rows_for_a_packed_product():
    """Nothing stood in their place; with a GPU's weight they were read all the same."""
    with pytest.raises(TypeError, match="x must be"):
        sk.sinkhorn_expert_product_packed(None, EIGHT, OFFSETS)


@pytest.mark.parametrize("call", [
    lambda: sk.sinkhorn_norm(None), lambda: sk.sinkhorn_norm(X, None), lambda: sk.sinkhorn_residual_norm(None, X),
    lambda: sk.sinkhorn_residual_norm(X, None), lambda: sk.sinkhorn_pack(None), lambda: sk.sinkhorn_unpack(None),
    lambda: sk.sinkhorn_unpack(EIGHT._replace(values=None)), lambda: sk.sinkhorn_unpack(EIGHT._replace(scales=None)),
    lambda: sk.sinkhorn_expert_product_packed(X, None, OFFSETS), lambda: sk.sinkhorn_activation(None, "silu"),
    lambda: sk.sinkhorn_expert_product_kept(None, X, OFFSETS), lambda: sk.sinkhorn_expert_product_kept(X, None, OFFSETS),
    lambda: sk.sinkhorn_expert_product_kept(X, X, None)])
def test_none_is_no_tensor(call):
    with pytest.raises(TypeError):
        call()
