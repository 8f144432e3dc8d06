"""The largest calls of the gated delta rule: what the launches hold, and what is refused before any of them (without a GPU)."""
import ctypes

import pytest

import paper_2603_04127_amd as dk

A = 1 << 20   # aligned, never dereferenced


def _p(**kw):
    base = dict(B=1, H=1, L=64, dk=16, dv=8, io_dtype=dk.DARK_F32, layout=dk.BHLD, scale=0.0)
    base.update(kw)
    return ctypes.byref(dk.DeltaParams(*base.values()))


def _backward(p):
    far = [A + (i << 44) for i in range(15)]   # tensors of their real sizes, apart from each other
    return dk.lib().dark_delta_bwd(p, *far, None, 0, None)


@pytest.mark.parametrize("heads,L,wide,dtype", [(4129776, 65, 128, dk.DARK_F32), (4129776, 65, 256, dk.DARK_F32), (2767375, 97, 65, dk.DARK_F32), (1 << 22, 64, 128, dk.DARK_F32)])
def test_more_chunks_than_a_launch_holds(heads, L, wide, dtype):
    # the gradients' kernel has 512 threads for a chunk of 32 rows where keys are wider than 64: 2^32 threads from 2^23 chunks on
    assert heads * L <= 1 << 28 and heads * -(-L // 32) * 512 >= 1 << 32
    assert _backward(_p(B=heads, L=L, dk=wide, dv=1, io_dtype=dtype)) == dk.DARK_EUNSUPPORTED
    assert dk.lib().dark_delta_workspace_bytes(_p(B=heads, L=L, dk=wide, dv=1, io_dtype=dtype), 1) == 0


@pytest.mark.parametrize("heads,L,wide,dtype", [(4129776, 65, 64, dk.DARK_F32), (4129776, 65, 128, dk.DARK_BF16), ((1 << 22) - 1, 64, 128, dk.DARK_F32), (1 << 22, 32, 128, dk.DARK_F32)])
def test_as_many_chunks_as_a_launch_holds(heads, L, wide, dtype):
    p = _p(B=heads, L=L, dk=wide, dv=1, io_dtype=dtype)
    assert dk.lib().dark_delta_workspace_bytes(p, 1) > dk.lib().dark_delta_workspace_bytes(p, 0) > 0
    assert _backward(p) == dk.DARK_EWORKSPACE   # the next thing that is looked at


def test_what_a_forward_call_holds():
    # 256 threads for a chunk's triangles: the most chunks that 2^28 rows make are 12.4 million
    p = _p(B=4129776, L=65, dk=128, dv=1)
    assert 4129776 * 3 * 256 < 1 << 32 and dk.lib().dark_delta_workspace_bytes(p, 0) > 0
    assert dk.lib().dark_delta_workspace_bytes(_p(B=(1 << 22) + 1, L=1), 0) == 0                       # heads
    assert dk.lib().dark_delta_workspace_bytes(_p(layout=dk.BLHD, H=(1 << 18) + 1, dk=16), 0) == 0      # elements of a row of all heads
    assert dk.lib().dark_delta_workspace_bytes(_p(layout=dk.BLHD, H=1 << 18, dk=16), 0) > 0
