"""Projections of so many tiles that a launch could not count their work items (2^32) take larger tiles."""
import ctypes

import pytest

from paper_2601_20655_amd import binding as B


def form_of(name, M, N, K):
    f = getattr(B.lib(), name)
    f.restype = ctypes.c_int
    return f(M, N, K, 256)


@pytest.mark.parametrize("name", ["_ZN3dit21choose_linear_form_i8Eiiii", "_ZN3dit18choose_linear_formEiiii"])
@pytest.mark.parametrize("M,N", [(1 << 30, 8), (1 << 30, 5), (540000011, 5), (540000011, 64), (1 << 24, 5120), (5, 1 << 30),
                                 (268435456, 8), (268435457, 8), (40000000, 520)])
@pytest.mark.parametrize("K", [64, 128, 5120])
def test_tiles_fit_a_launch(name, M, N, K):
    form = form_of(name, M, N, K)
    if form in (0, 64):  # (workgroups that walk over their tiles)
        assert N >= 8 or "i8" not in name
        return
    tb, fb = form // 10, form % 10
    assert -(-M // (32 * tb)) * -(-N // (64 * fb)) * 512 < 1 << 32
