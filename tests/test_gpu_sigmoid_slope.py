"""The derivative of the sigmoid far from zero, s (1 - s), on a scale that a derivative of 0 fails.

s is held to a few 2^-24 with fp32 io and to 2^-20 (the hardware's exponential and reciprocal) with
bf16 io, relative to itself, and so is 1 - s to that much of 1: the product is off by at most that
share of s (8 2^-24, 2^-19 with its own roundings), and the stored value by half a step more.  For
z < 0 this is relative to the derivative itself; for z > 0 the scale is s = 1, where a derivative of
0 passes from 2^-19 down (z = 13) and from 2^-21 down (z = 14.5) only."""
import pytest
import torch

from paper_2606_01294_amd import ccq

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dt", [F32, BF], ids=["fp32", "bf16"])
def test_sigmoid_slope(dt):
    z = torch.cat([torch.linspace(-80, 80, 641), torch.linspace(-16, 16, 513)]).to(dt)
    n, C = len(z), 8
    x = z[:, None, None].expand(n, 1, C).contiguous().cuda()  # one token a sequence
    w = torch.zeros(C, 2, device="cuda")
    w[:, 1] = 1
    s = torch.sigmoid(z.double())
    ref = s * torch.sigmoid(-z.double())
    half, work = {F32: (2.0 ** -24, 8 * 2.0 ** -24), BF: (2.0 ** -8, 2.0 ** -19)}[dt]
    tol = half * ref + work * s + 2.0 ** -126
    conv = ccq.ccq_conv_bwd(x, w, torch.ones_like(x), act=ccq.CCQ_ACT_SIGMOID)["dx"][:, 0]
    # and as the gate of a norm whose n is 1 in every channel: dgate = dy n act'(gate)
    one = torch.ones(n, 1, C, device="cuda", dtype=dt)
    norm = ccq.ccq_norm_bwd(one, one, gate=x, kind=ccq.CCQ_NORM_RMS, act=ccq.CCQ_ACT_SIGMOID, eps=0.0)["dgate"][:, 0]
    for name, got in (("conv", conv), ("norm", norm)):
        off = (got.double().cpu() - ref[:, None]).abs()
        print(name, float((off / tol[:, None]).max()), flush=True)
        assert bool((off <= tol[:, None]).all()), name
