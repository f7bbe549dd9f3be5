"""Sizes of the plain delta rule that a launch cannot count, or whose offsets within a chunk pass 32
bits: refused before anything is launched.  CPU: the addresses are never read, and the largest
sizes that pass are asked for with a workspace that is too small, or none."""
import pytest
import torch

from paper_2606_01294_amd import ccq
from test_layer_abi import FAKE, UNSUPPORTED, WORKSPACE, delta, delta_train, dshape, ptrs

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("call", [delta, delta_train])
@pytest.mark.parametrize("dk,dv,dt", [(64, 64, BF), (128, 512, BF), (256, 256, BF), (64, 64, F32)])
def test_chunked_forms(call, dk, dv, dt):
    def ask(B, T, HV):
        shape = dshape(B=B, T=T, HK=1, HV=HV, dk=dk, dv=dv, dt=dt)
        rc = call(shape, size=64)
        assert (rc == UNSUPPORTED) == (ccq.ccq_delta_workspace_size(shape, call is delta_train) == 0)
        return rc
    # 2^23 chunks of up to 512 threads
    assert ask(1 << 10, 64 << 10, 8) == UNSUPPORTED
    assert ask((1 << 10) - 1, 64 << 10, 8) == WORKSPACE
    # tiles of 16 value channels, up to 256 threads each
    tiles = 28 if dk == 256 else 29
    assert ask(1 << 10, 1, (1 << tiles) // dv >> 10) == UNSUPPORTED
    assert ask((1 << 10) - 1, 1, (1 << tiles) // dv >> 10) == WORKSPACE
    # rows of a chunk
    heads = (1 << 24) // max(dk, dv)
    assert ask(1, 64, heads) == WORKSPACE
    assert ask(1, 64, heads + 1) == UNSUPPORTED


def test_step():
    def step(B, HV, dk, dv):  # (without a state, so that what passes the sizes stops there)
        return ccq.lib().ccq_delta_step(dshape(B=B, T=1, HK=1, HV=HV, dk=dk, dv=dv),
                                        *ptrs(FAKE, FAKE, FAKE, FAKE, FAKE, 0, FAKE), None)
    assert step(1 << 16, 16, 64, 256) == UNSUPPORTED  # 2^32 threads
    assert step((1 << 16) - 1, 16, 64, 256) == 1
    assert step(1, (1 << 16) + 1, 256, 64) == UNSUPPORTED
    assert step(1, 1 << 16, 256, 64) == 1
