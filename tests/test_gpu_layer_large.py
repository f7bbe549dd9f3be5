"""The operators around the contraction where element offsets pass 32 bits: the last rows of a
call on more than 2^31 elements against a call on those rows alone.  The convolution, the norm
and the recurrent step treat tokens alike wherever they lie: the same bits.  The chunked rule
may group its chunks differently: its bar, 2e-2 of the largest value."""
import pytest
import torch

from paper_2606_01294_amd import ccq

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
BIG = (1 << 31) + (1 << 20)


def rand(*shape):
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    return torch.randn(*shape, generator=g, device="cuda", dtype=BF)


def test_norm():
    G, D = 8, 256
    rows = BIG // (G * D) + 3
    x = rand(rows, G, D)
    w = 1 + 0.1 * torch.randn(D, device="cuda")
    y = ccq.ccq_norm_fwd(x, weight=w, gate=x)
    tail = x[-5:].clone()
    assert torch.equal(y[-5:], ccq.ccq_norm_fwd(tail, weight=w, gate=tail))
    got = ccq.ccq_norm_bwd(x, y, weight=w, gate=x)
    one = ccq.ccq_norm_bwd(tail, y[-5:].clone(), weight=w, gate=tail)
    assert torch.equal(got["dx"][-5:], one["dx"]) and torch.equal(got["dgate"][-5:], one["dgate"])


def test_conv():
    C, W = 4096, 4
    T = BIG // C + 5
    x = rand(1, T, C)
    w = torch.randn(C, W, device="cuda") * 0.5
    out = ccq.ccq_conv_fwd(x, w, want_state=True)
    n = 40
    s0 = x[:, T - n - W + 1:T - n].contiguous()
    tail = x[:, T - n:].contiguous()
    one = ccq.ccq_conv_fwd(tail, w, state0=s0, want_state=True)
    assert torch.equal(out["y"][:, T - n:], one["y"])
    assert torch.equal(out["stateT"], one["stateT"])
    got = ccq.ccq_conv_bwd(x, w, out["y"])
    last = ccq.ccq_conv_bwd(tail, w, one["y"], state0=s0)
    assert torch.equal(got["dx"][:, T - n:], last["dx"])


def test_delta_packed():
    H, D, n = 8, 64, 2048
    B = BIG // (H * D * n) + 2
    rows = B * n
    q, k, v = rand(rows, H, D), rand(rows + 1, H, D)[:rows], rand(rows + 2, H, D)[:rows]
    q, k = (ccq.ccq_norm_fwd(t, kind=ccq.CCQ_NORM_L2, act=ccq.CCQ_ACT_NONE) for t in (q, k))
    la = -0.1 * torch.rand(rows, H, device="cuda")
    be = torch.rand(rows, H, device="cuda")
    cu = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
    got = ccq.ccq_delta_fwd_varlen(q, k, v, la, be, cu, n)
    end = slice(rows - n, rows)
    one = ccq.ccq_delta_fwd(*[t[end].unsqueeze(0).contiguous() for t in (q, k, v, la, be)])
    o = one["o"][0].float()
    assert float((got["o"][end].float() - o).abs().max()) <= 2e-2 * float(o.abs().max())
    # the state pass splits the features over waves by the number of heads: fp32 sums in
    # another order, and the operands' tails (2^-17)
    s = one["ST"][0]
    assert float((got["ST"][-1] - s).abs().max()) <= 2e-5 * float(s.abs().max())


def test_delta_step():
    HV, dk, dv = 16, 256, 256
    B = BIG // (HV * dk * dv) + 2
    S = torch.zeros(B, HV, dv, dk, device="cuda")
    q, k, v = rand(B, 1, HV, dk) * 0.06, rand(B, 1, HV, dk) * 0.06, rand(B, 1, HV, dv)
    la, be = -0.1 * torch.rand(B, 1, HV, device="cuda"), torch.rand(B, 1, HV, device="cuda")
    for _ in range(2):
        o = ccq.ccq_delta_step(q, k, v, la, be, S)
    S1 = torch.zeros(1, HV, dv, dk, device="cuda")
    for _ in range(2):
        o1 = ccq.ccq_delta_step(*[t[-1:].contiguous() for t in (q, k, v, la, be)], S1)
    assert torch.equal(o[-1:], o1) and torch.equal(S[-1:], S1)
