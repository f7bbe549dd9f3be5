"""Refusals of the operators around the contraction (plain delta rule, short convolution, head
norm): bad arguments are answered by a status before anything is launched, so these run on the
CPU with addresses that are never read."""
import ctypes

import pytest
import torch

from paper_2606_01294_amd import ccq

FAKE = 1 << 20
BF, F32 = torch.bfloat16, torch.float32
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def ptrs(*p):
    return [ctypes.c_void_p(x) if x else None for x in p]


def delta(shape, cu=None, S0=0, o=FAKE, ST=0, ws=FAKE, size=1 << 40, q=FAKE):
    args = ptrs(q, FAKE, FAKE, FAKE, FAKE, S0, o, ST, ws) + [size, None]
    if cu is None:
        return ccq.lib().ccq_delta_fwd(shape, *args)
    return ccq.lib().ccq_delta_fwd_varlen(shape, *(ptrs(cu) + args))


def delta_train(shape, o=0, dO=FAKE, dbeta=FAKE, size=1 << 40):
    return ccq.lib().ccq_delta_fwd_bwd(shape, *ptrs(FAKE, FAKE, FAKE, FAKE, FAKE, 0, dO, o, 0, FAKE,
                                                    FAKE, FAKE, FAKE, dbeta, FAKE), size, None)


def dshape(B=2, T=100, HK=2, HV=4, dk=128, dv=128, dt=BF):
    return ccq.make_delta_shape(B, T, HK, HV, dk, dv, dt)


def test_delta_refusals():
    assert delta(None) == INVALID
    assert delta(dshape(T=-1)) == INVALID
    assert delta(dshape(HK=3, HV=4)) == INVALID      # heads that do not divide
    assert delta(dshape(HK=0, HV=4)) == INVALID
    assert delta(dshape(dk=96)) == UNSUPPORTED
    assert delta(dshape(dv=96)) == UNSUPPORTED
    assert delta(dshape(dk=256, dt=F32)) == UNSUPPORTED
    assert delta(dshape(), q=0) == INVALID
    assert delta(dshape(), q=FAKE + 8) == INVALID    # misaligned
    assert delta(dshape(), o=0) == INVALID           # the forward needs o
    assert delta(dshape(), S0=FAKE + 4) == INVALID
    assert delta(dshape(), S0=FAKE, ST=FAKE + 64) == INVALID  # partly over each other
    assert delta(dshape(), size=64) == WORKSPACE
    assert delta(dshape(), ws=0) == WORKSPACE
    assert delta(dshape(), cu=FAKE + 2) == INVALID
    assert delta(dshape(B=70000, T=4), cu=FAKE) == UNSUPPORTED
    bad = dshape()
    bad.io_dtype = 7
    assert delta(bad) == INVALID
    # nothing to do
    assert delta(dshape(B=0), q=0, o=0, ws=0) == 0
    assert delta(dshape(HK=0, HV=0), q=0, o=0, ws=0) == 0
    assert delta(dshape(T=0), q=0, o=0, ws=0) == 0


def test_delta_train_refusals():
    assert delta_train(dshape(), dO=0) == INVALID
    assert delta_train(dshape(), dbeta=0) == INVALID
    assert delta_train(dshape(), o=FAKE + 8) == INVALID
    assert delta_train(dshape(dk=128, dt=F32)) == UNSUPPORTED   # fp32 training has dk = 64
    assert delta_train(dshape(), size=ccq.ccq_delta_workspace_size(dshape())) == WORKSPACE
    assert ccq.ccq_delta_workspace_size(dshape(), True) > ccq.ccq_delta_workspace_size(dshape())
    assert ccq.ccq_delta_workspace_size(dshape(dk=96)) == 0
    # shared heads need their value heads' gradients apart
    one = ccq.ccq_delta_workspace_size(dshape(HK=4, HV=4), True)
    assert ccq.ccq_delta_workspace_size(dshape(HK=2, HV=4), True) > one


def test_delta_step_refusals():
    def step(s, S=FAKE, q=FAKE):
        return ccq.lib().ccq_delta_step(s, *ptrs(q, FAKE, FAKE, FAKE, FAKE, S, FAKE), None)
    assert step(None) == INVALID
    assert step(dshape(), S=0) == INVALID
    assert step(dshape(), q=FAKE + 2) == INVALID
    assert step(dshape(HK=3)) == INVALID
    assert step(dshape(dk=32)) == UNSUPPORTED
    assert step(dshape(T=0), S=0) == 0


def cshape(B=2, T=9, C=64, W=4, dt=BF, act=1, ldx=64):
    return ccq.ConvShape(B, T, C, W, ccq._dt(dt), act, ldx)


def test_conv_refusals():
    def fwd(s, x=FAKE, w=FAKE, s0=0, sT=0, y=FAKE):
        return ccq.lib().ccq_conv_fwd(s, *ptrs(x, w, 0, s0, y, sT), None)

    def bwd(s, bias=0, dbias=0, dw=FAKE, ws=FAKE, size=1 << 40, dy=FAKE):
        return ccq.lib().ccq_conv_bwd(s, *ptrs(FAKE, FAKE, bias, 0, dy, 0, FAKE, dw, dbias, 0, ws),
                                      size, None)
    assert fwd(None) == INVALID
    assert fwd(cshape(W=1)) == UNSUPPORTED
    assert fwd(cshape(W=5)) == UNSUPPORTED
    assert fwd(cshape(C=60, ldx=64)) == UNSUPPORTED
    assert fwd(cshape(C=0)) == UNSUPPORTED
    assert fwd(cshape(act=3)) == INVALID
    assert fwd(cshape(ldx=56)) == INVALID            # tokens over each other
    assert fwd(cshape(ldx=68)) == INVALID            # rows off 16 bytes
    assert fwd(cshape(dt=F32, ldx=66)) == INVALID
    assert fwd(cshape(), x=0) == INVALID
    assert fwd(cshape(), w=FAKE + 4) == INVALID
    assert fwd(cshape(), s0=FAKE, sT=FAKE) == INVALID  # the state is read while it is written
    assert fwd(cshape(B=1 << 30, T=1 << 20)) == UNSUPPORTED
    assert fwd(cshape(B=0), x=0, w=0, y=0) == 0
    assert fwd(cshape(T=0), x=0, y=0) == 0
    assert bwd(cshape(), bias=FAKE) == INVALID       # a bias without its gradient
    assert bwd(cshape(), dbias=FAKE) == INVALID
    assert bwd(cshape(), dw=0) == INVALID
    assert bwd(cshape(), dy=0) == INVALID
    assert bwd(cshape(), size=8) == WORKSPACE
    assert bwd(cshape(), ws=0) == WORKSPACE
    assert ccq.lib().ccq_conv_workspace_size(cshape(W=6)) == 0

    def step(s, st=FAKE):
        return ccq.lib().ccq_conv_step(s, *ptrs(FAKE, FAKE, 0, st, FAKE), None)
    assert step(cshape()) == INVALID                 # one token
    assert step(cshape(T=1), st=0) == INVALID
    assert step(cshape(T=1, B=0)) == 0


def nshape(rows=3, G=2, D=64, dt=BF, kind=1, act=1, shared=0, eps=1e-5, ldx=128, ldg=128):
    return ccq.NormShape(rows, G, D, ccq._dt(dt), kind, act, shared, eps, ldx, ldg)


def test_norm_refusals():
    def fwd(s, x=FAKE, w=FAKE, b=0, g=0, y=FAKE):
        return ccq.lib().ccq_norm_fwd(s, *ptrs(x, w, b, g, y), None)

    def bwd(s, w=FAKE, dw=FAKE, g=0, dg=0, b=0, db=0, ws=FAKE, size=1 << 40):
        return ccq.lib().ccq_norm_bwd(s, *ptrs(FAKE, w, b, g, FAKE, FAKE, dw, db, dg, ws), size, None)
    assert fwd(None) == INVALID
    assert fwd(nshape(D=60, ldx=120)) == UNSUPPORTED
    assert fwd(nshape(D=8200, G=1, ldx=8200)) == UNSUPPORTED
    assert fwd(nshape(G=1 << 20, ldx=1 << 26)) == UNSUPPORTED
    assert fwd(nshape(kind=3)) == INVALID
    assert fwd(nshape(act=-1)) == INVALID
    assert fwd(nshape(shared=2)) == INVALID
    for eps in (-1e-6, float("nan"), float("inf")):
        assert fwd(nshape(eps=eps)) == INVALID
    assert fwd(nshape(ldx=120)) == INVALID
    assert fwd(nshape(ldx=132)) == INVALID
    assert fwd(nshape(ldg=64), g=FAKE) == INVALID
    assert fwd(nshape(), w=0, b=FAKE) == INVALID     # a bias without a weight
    assert fwd(nshape(), x=FAKE + 2) == INVALID
    assert fwd(nshape(rows=0), x=0, y=0) == 0
    assert bwd(nshape(), dw=0) == INVALID
    assert bwd(nshape(), g=FAKE) == INVALID          # a gate without its gradient
    assert bwd(nshape(), dg=FAKE) == INVALID
    assert bwd(nshape(), b=FAKE) == INVALID
    assert bwd(nshape(), size=16) == WORKSPACE
    assert ccq.lib().ccq_norm_workspace_size(nshape(D=4)) == 0


def test_the_binding_refuses_tensors_off_the_gpu():
    """A host pointer must never reach a kernel."""
    x = torch.zeros(2, 5, 64, dtype=BF)
    w = torch.zeros(64, 4)
    q = torch.zeros(1, 3, 2, 64, dtype=BF)
    g = torch.zeros(1, 3, 2)
    with pytest.raises(ValueError):
        ccq.ccq_conv_fwd(x, w)
    with pytest.raises(ValueError):
        ccq.ccq_conv_step(x[:, 0], w, torch.zeros(2, 3, 64, dtype=BF))
    with pytest.raises(ValueError):
        ccq.ccq_norm_fwd(x.view(2, 5, 1, 64))
    with pytest.raises(ValueError):
        ccq.ccq_delta_fwd(q, q, q, g, g)
    with pytest.raises(ValueError):
        ccq.ccq_delta_step(q, q, q, g, g, torch.zeros(1, 2, 64, 64))


def test_row_pitch_of_slices():
    """The pitch of a slice of a wider tensor, and what has none."""
    t = torch.zeros(3, 5, 4, 32)
    assert ccq._pitch(t, 2, "t") == 128
    assert ccq._pitch(torch.zeros(3, 5, 200)[..., 8:72], 1, "t") == 200
    assert ccq._pitch(torch.zeros(15, 6, 32)[:, 2:5], 2, "t") == 192
    assert ccq._pitch(torch.zeros(1, 1, 200)[..., :64], 1, "t") == 64  # one row: any pitch
    with pytest.raises(ValueError):
        ccq._pitch(t.transpose(2, 3), 2, "t")          # channels apart
    with pytest.raises(ValueError):
        ccq._pitch(torch.zeros(3, 8, 64)[:, :5], 1, "t")  # unevenly spaced tokens
    with pytest.raises(ValueError):
        ccq._pitch(torch.zeros(1, 64).expand(5, 64), 1, "t")  # one row over itself
