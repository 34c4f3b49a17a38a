"""Sizes of scratch memory that go with the sizes that weight gradients take."""
import ctypes

import pytest

from paper_2607_24953_b200 import binding as b

P = 0x100000


@pytest.mark.parametrize("T,N,K,groups", [(1 << 24, 1 << 30, 1 << 30, 1), (1 << 30, 1 << 24, 1 << 24, 1), (1 << 30, 1 << 30, 256, 2047), (1 << 30, 1 << 19, 1 << 19, 1),
                                          (2000, 1 << 30, 1 << 30, 3)])
def test_what_the_call_refuses_needs_none(T, N, K, groups):
    g = ctypes.byref(b._CGroups(groups, 0, P))
    assert b.lib().fp4q_ragged_gemm_wgrad(P, T, N, N, P, K, K, P, K, 1, 0, g, None, 0, P, 256, None) == 4
    assert b.lib().fp4q_ragged_gemm_wgrad_scratch_bytes(T, N, K, groups) == 0


def test_updates_of_more_tiles_and_parts_than_are_counted_are_refused():
    f = b.lib().fp4q_newton_schulz_scratch_bytes
    assert f(1, 1 << 20, 1 << 20) == 0 and f(1, 4096, 1 << 20) > 0 and f(130, 16, 1 << 20) > 0
