"""Outputs of the convolution that lie over its inputs: runs of tokens read what an earlier run would
have overwritten, so the call is refused.  CPU: refused before anything is launched, the addresses
are never read."""
import pytest

from paper_2606_01294_amd import ccq
from test_layer_abi import FAKE, INVALID, cshape, ptrs

B, T, C, W, LD = 2, 100, 64, 4, 192
ROW, Y, ST = 2 * LD, 2 * B * T * C, 2 * B * (W - 1) * C  # bytes


def fwd(x, s0, y, sT, ld=LD):
    return ccq.lib().ccq_conv_fwd(cshape(B=B, T=T, C=C, W=W, ldx=ld), *ptrs(x, FAKE, 0, s0, y, sT), None)


@pytest.mark.parametrize("y", [FAKE, FAKE + 16, FAKE - Y + 16, FAKE + (B * T - 1) * ROW + 2 * C - 16,
                               FAKE + 2 * C])
def test_y_over_x(y):
    assert fwd(FAKE, 0, y, 0) == INVALID


def test_in_place():
    assert fwd(FAKE, 0, FAKE, 0, ld=C) == INVALID


@pytest.mark.parametrize("off", [0, 16, Y - 16, 16 - ST])
def test_y_over_the_states(off):
    assert fwd(1 << 30, FAKE + off, FAKE, 0) == INVALID
    assert fwd(1 << 30, 0, FAKE, FAKE + off) == INVALID


@pytest.mark.parametrize("sT", [FAKE, FAKE + ROW, FAKE + (B * T - 1) * ROW, FAKE + 2 * C])
def test_the_final_state_over_x(sT):
    assert fwd(FAKE, 0, 1 << 30, sT) == INVALID
