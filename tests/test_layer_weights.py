"""The router's weights of the layer of experts lie as its choices do, [tokens x slots]: as many numbers in another order are refused."""
import pytest
import torch

from test_abi_b128 import on_host  # noqa: F401

TOKENS, SLOTS = 4, 2


def _arguments(mx, device):
    u8 = dict(dtype=torch.uint8, device=device)
    return dict(x=torch.ones((TOKENS, 64), dtype=torch.bfloat16, device=device), experts=torch.zeros((TOKENS, SLOTS), dtype=torch.int32, device=device),
                format=mx.WEIGHTS_MXFP8, up_q=torch.zeros((3, 64, 64), **u8), up_s=torch.zeros((3, 64, 2), **u8), down_q=torch.zeros((3, 64, 32), **u8),
                down_s=torch.zeros((3, 64, 1), **u8), out=torch.full((TOKENS, 64), 7.0, device=device),
                workspace=torch.zeros((mx.mxfp8_expert_layer_workspace(TOKENS, SLOTS, 32),), **u8))


def _refuses(mx, device):
    given = _arguments(mx, device)
    for shape in ((SLOTS, TOKENS), (TOKENS * SLOTS,), (TOKENS, SLOTS, 1), (1, TOKENS * SLOTS)):
        with pytest.raises(ValueError, match="weights"):
            mx.mxfp8_expert_layer(weights=torch.ones(shape, device=device), **given)
    assert (given["out"] == 7).all()
    return given


def test_weights_of_another_shape_are_refused_on_the_host(on_host):  # noqa: F811
    _refuses(on_host, "cpu")


@pytest.mark.gpu
def test_weights_of_another_shape_are_refused():
    import paper_2506_08027_amd as mx
    given = _refuses(mx, "cuda")
    mx.mxfp8_expert_layer(weights=torch.ones((TOKENS, SLOTS), device="cuda"), **given)
    assert (given["out"] == 0).all()
