"""Attention's largest calls, at the C boundary and without a GPU: more workgroups than a launch counts are refused."""
import ctypes

import pytest

from paper_2202_00774_amd import binding

P, E_SHAPE = ctypes.c_void_p(16), -3                                             # never dereferenced


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("S, T, H, Hk", [(1 << 24, 1 << 24, 1, 1), (1 << 22, 1 << 22, 8, 8), (1 << 21, 0x1FF000, 512, 8)])
def test_more_workgroups_than_a_launch_counts(S, T, H, Hk, dt):
    lib, st = binding.load(), (ctypes.c_int64 * 6)(H * 64, 64, Hk * 64, 64, Hk * 64, 64)
    assert Hk * (S + 2) >= 1 << 24
    ws, size = P, 1 << 62
    assert lib.sdgp_attention(P, P, P, st, P, P, None, S, P, P, T, T, H, Hk, 64, dt, 1, 0.1, ws, size, None) == E_SHAPE
    assert lib.sdgp_attention_bwd(P, P, P, P, P, P, st, P, P, S, P, P, P, T, T, H, Hk, 64, dt, 1, 0.1, ws, size, None) == E_SHAPE
