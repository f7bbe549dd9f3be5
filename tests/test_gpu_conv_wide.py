"""Gradients of the convolution at the most channels that its header allows: the sums of dw and
dbias are more columns than one dimension of a launch has threads for."""
import pytest
import torch

from paper_2606_01294_amd import ccq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C,W", [(1 << 24, 4), ((1 << 24) - 8, 2), (13_421_776, 4)])
def test_gradients_of_one_token(C, W):
    """One token, no activation: every gradient is one product of two bf16 values, exact in fp32."""
    g = torch.Generator(device="cuda").manual_seed(C)
    x, dy = (torch.randn(1, 1, C, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    w, bias = torch.randn(C, W, generator=g, device="cuda"), torch.zeros(C, device="cuda")
    got = ccq.ccq_conv_bwd(x, w, dy, bias=bias, act=ccq.CCQ_ACT_NONE)
    xf, df = x.float().view(C), dy.float().view(C)
    assert torch.equal(got["dw"][:, W - 1], xf * df)
    assert bool((got["dw"][:, :W - 1] == 0).all())
    assert torch.equal(got["dbias"], df)
    assert torch.equal(got["dx"].view(C), (w[:, W - 1] * df).to(torch.bfloat16))
