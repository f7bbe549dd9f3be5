"""The plain gated delta rule behind many resets and steep gates of one chunk, fp32 io.

A reset adds -104 to the chunk's running sum of log alpha, so behind dozens of them the sum is
thousands, where a step of fp32 is up to 4.9e-4; the decays between the tokens behind them are
e^(differences) and must not feel it.

Tolerance, of a tensor's largest value: a decay is good to a few 2^-24; an output passes three
products of at most 128 terms (scores, transform, values), 128 roundings of 2^-24 each, 3 2^-17; a
gradient as many again on the way back, 6 2^-17."""
import pytest
import torch

from paper_2606_01294_amd import ccq
from test_gpu_delta import check, dev, make, solve

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16
FWD_TOL, GRAD_TOL = 3 * 2.0 ** -17, 6 * 2.0 ** -17


def gates(d, lens, kind):
    """Overwrites log alpha: resets in every chunk's first 48 tokens, in half or nine tenths of
    all tokens, or no reset but steep gates."""
    g = torch.Generator().manual_seed(7)
    la = d["la"]
    if kind == "front":
        at = torch.cat([torch.arange(n) % 64 for n in lens])
        la[at < 48] = -float("inf")
    elif kind == "steep":
        la.copy_(-5 - 2 * torch.rand(la.shape, generator=g))
    else:
        la[torch.rand(la.shape, generator=g) < {"half": 0.5, "most": 0.9}[kind]] = -float("inf")
    # what follows a reset reads much of it: keys that resemble their neighbours, queries their keys
    d["k"] = torch.nn.functional.normalize(0.5 * d["k"].float() + d["k"].float().mean((0, 1)), dim=-1).to(d["k"].dtype)
    d["q"] = d["k"].clone()


@pytest.mark.parametrize("kind", ["front", "half", "most", "steep"])
@pytest.mark.parametrize("lens,HK,HV,dk,dv", [([64, 64], 1, 2, 64, 64), ([200], 2, 4, 128, 128)])
def test_forward(lens, HK, HV, dk, dv, kind):
    d = make(lens, HK, HV, dk, dv, F32, True)
    gates(d, lens, kind)
    ref = solve(d, lens, 0.7, False)
    got = ccq.ccq_delta_fwd(*dev(d, (len(lens), lens[0])), S0=d["S"].cuda(), scale=0.7)
    check(got, ref, FWD_TOL)


@pytest.mark.parametrize("kind", ["front", "half", "most", "steep"])
@pytest.mark.parametrize("lens,HK,HV,dv", [([130, 130], 2, 2, 64), ([64, 3, 0, 100], 1, 3, 128)])
def test_training_step(lens, HK, HV, dv, kind):
    d = make(lens, HK, HV, 64, dv, F32, True)
    gates(d, lens, kind)
    ref = solve(d, lens, 0.7, True)
    cu = torch.tensor([0] + [sum(lens[:i + 1]) for i in range(len(lens))], dtype=torch.int32).cuda()
    got = ccq.ccq_delta_fwd_bwd_varlen(*dev(d), d["dO"].cuda(), cu, max(lens), S0=d["S"].cuda(),
                                       scale=0.7, want_states=True)
    check(got, ref, FWD_TOL, ("o", "ST"))
    check(got, ref, GRAD_TOL, ("dq", "dk", "dv", "dlogalpha", "dbeta"))


@pytest.mark.parametrize("kind", ["front", "most"])
@pytest.mark.parametrize("HK,HV,dk,dv", [(2, 4, 128, 128), (1, 1, 256, 256), (1, 2, 64, 64)])
def test_bf16(HK, HV, dk, dv, kind):
    """bf16 io takes the same decays; its bar is the framework's, 2e-2."""
    lens = [130, 130]
    d = make(lens, HK, HV, dk, dv, BF, True)
    gates(d, lens, kind)
    ref = solve(d, lens, 0.7, True)
    got = ccq.ccq_delta_fwd_bwd(*dev(d, (2, 130)), d["dO"].cuda().view(2, 130, HV, dv),
                                S0=d["S"].cuda(), scale=0.7, want_states=True)
    check(got, ref, 2e-2)
