"""The LayerNorm across all heads with a gamma and a beta that both have to be copied to lie contiguous."""
import pytest
import torch

import paper_2407_12077_b200 as gf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [1, 4, 32])
def test_both_copies_live_until_the_call(dtype, H):
    g = torch.Generator(device=DEV).manual_seed(H)
    y = torch.randn(50, H, 64, generator=g, device=DEV).to(dtype)
    gamma, beta = (torch.randn(H, 128, generator=g, device=DEV)[:, ::2] for _ in range(2))
    want = gf.layernorm_heads(y, gamma.contiguous(), beta.contiguous())
    for _ in range(3):
        assert torch.equal(gf.layernorm_heads(y, gamma, beta), want)


@pytest.mark.parametrize("H", [1, 4, 32])
def test_gradient_takes_the_same_gammas(H):
    g = torch.Generator(device=DEV).manual_seed(H)
    y, dout = (torch.randn(50, H, 64, generator=g, device=DEV) for _ in range(2))
    wide = torch.randn(H, 128, generator=g, device=DEV)
    for gamma in (wide[:, ::2], wide[:, :64]):
        want = gf.layernorm_heads_backward(y, dout, gamma.contiguous())
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(gf.layernorm_heads_backward(y, dout, gamma), want))
        assert torch.equal(gf.layernorm_heads(y, gamma, wide[:, 64:]), gf.layernorm_heads(y, gamma.contiguous(), wide[:, 64:].contiguous()))
