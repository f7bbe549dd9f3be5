"""The convolution's step on column slices: which states lie apart from its tokens.  Tensors are
carved out of one buffer, so that where they lie does not depend on the allocator."""
import pytest
import torch

from paper_2606_01294_amd import ccq

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
B, C, W, LD = 8, 64, 4, 192


def step(buf, at, state, C0):
    """The step on columns C0 .. of the [B, LD] tensor at buf[at], its state at buf[state]; against
    the same step on copies."""
    x = buf[at:at + B * LD].view(B, LD)[:, C0:C0 + C]
    st = buf[state:state + B * (W - 1) * C].view(B, W - 1, C)
    w = torch.randn(C, W, generator=torch.Generator().manual_seed(1)).cuda()
    other = st.clone()
    want = ccq.ccq_conv_step(x.contiguous(), w, other)
    assert torch.equal(ccq.ccq_conv_step(x, w, st), want) and torch.equal(st, other)


def buffer(n):
    return torch.randn(n, generator=torch.Generator().manual_seed(2)).to(BF).cuda()


@pytest.mark.parametrize("C0", [0, 64, 128])
def test_a_state_right_behind_or_ahead_of_the_projection(C0):
    n = B * LD + B * (W - 1) * C
    step(buffer(n), 0, B * LD, C0)
    step(buffer(n), B * (W - 1) * C, 0, C0)


def test_one_token_of_a_sequence():
    """x[:, t] of [B,T,C], the state right behind x."""
    T = 5
    buf = buffer(B * T * C + B * (W - 1) * C)
    x = buf[:B * T * C].view(B, T, C)
    st = buf[B * T * C:].view(B, W - 1, C)
    w = torch.randn(C, W, device="cuda")
    for t in range(T):
        other = st.clone()
        want = ccq.ccq_conv_step(x[:, t].contiguous(), w, other)
        assert torch.equal(ccq.ccq_conv_step(x[:, t], w, st), want) and torch.equal(st, other)


def test_a_state_between_two_tokens():
    """One projection row is wider than the whole state."""
    wide = B * (W - 1) * C + 2 * C
    buf = buffer(2 * wide)
    x, w = buf.view(2, wide)[:, :C], torch.randn(C, W, device="cuda")
    st = buf[C:C + 2 * (W - 1) * C].view(2, W - 1, C)
    other = st.clone()
    want = ccq.ccq_conv_step(x.contiguous(), w, other)
    assert torch.equal(ccq.ccq_conv_step(x, w, st), want) and torch.equal(st, other)


@pytest.mark.parametrize("state", [B * LD - 8, 8, 128 + 8])
def test_overlap_is_refused(state):
    """One vector of the state within a token's columns (here the last ones of a row)."""
    buf = buffer(2 * B * LD + B * (W - 1) * C)
    x = buf[:B * LD].view(B, LD)[:, 128:]
    st = buf[state:state + B * (W - 1) * C].view(B, W - 1, C)
    with pytest.raises(ValueError):
        ccq.ccq_conv_step(x, torch.randn(C, W, device="cuda"), st)


def test_no_sequences():
    x = torch.empty(0, C, device="cuda", dtype=BF)
    assert ccq.ccq_conv_step(x, torch.randn(C, W, device="cuda"), x.new_empty(0, W - 1, C)).shape == (0, C)
