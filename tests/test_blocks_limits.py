"""Sizes that the block-scaled operators hold, at the limits that include/srq.h names (no GPU here: every call is rejected before a launch)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2511_00874_amd import build
    if build.stale():
        build.build()
    from paper_2511_00874_amd import lib as L
    return L


NULL, SHAPE = -1, -2


def test_gated_backward_fits_one_launch(lib):
    q = C.byref(lib.srq_quant(3, 1, 0.0, 0, None, 0, 0))

    def f(M, F):  # without its operands: NULL where the size is taken
        return lib.raw.sr_gated_bwd(None, None, None, 0, None, None, 0, None, None, M, F, 0, q, None)

    most = 2**22 - 8  # tiles, two workgroups of 512 threads each
    assert f(most * 128, 128) == f(most // 8 * 128, 8 * 128) == NULL
    assert f(most * 128 + 1, 128) == f(most // 8 * 128 + 1, 8 * 128) == SHAPE
