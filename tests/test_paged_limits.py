"""Sizes up to which calls on trees of drafted tokens go: host arithmetic, nothing is launched."""
import ctypes as C
import os

import pytest

from paper_2605_23163_amd import binding as bd
from paper_2605_23163_amd import paged as pg


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(bd.library_path()):
        from paper_2605_23163_amd import build
        build.build()
    return bd.load_library()


@pytest.mark.parametrize("N,V,fits", [(1, 1 << 30, True), (33, 1 << 30, True), (300, 1 << 28, True), ((1 << 14) - 1, 1 << 30, True), (1 << 14, 1 << 30, False), (1 << 20, 32768, False),
                                      ((1 << 20) - 1, 32768, True)])
def test_verification_of_wide_rows(lib, N, V, fits):
    """A row is drawn from in 1024 pieces at most, a workgroup each: N times that is what a launch limits, not N * V."""
    p = pg.TreeVerifyParams(N=N, B=1, V=V, dtype=1, temperature=1.0, draft_temperature=1.0)
    assert (lib.fdd_tree_verify_workspace(C.byref(p)) > 0) == fits
