"""Scalars of the layers of include/lccrf_layers.h at the ends of what their header allows, without a GPU: what is refused."""
import ctypes
import os

import pytest

from paper_2308_03291_amd import binding
from paper_2308_03291_amd.encoder import _Rows

EINVAL, EALIGN = -1, -4
FAKE = 4096  # an aligned "pointer" that is never dereferenced on these paths
ODD = FAKE + 2  # scalars are looked at first: a call that they let through ends here


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2308_03291_amd import build_ext
        build_ext.build()
    return binding.load_library()


def test_temperatures(lib):
    def both(t):
        return (lib.lccrf_distill(ODD, 10, 0, FAKE, FAKE, 4, 10, 3, t, FAKE, FAKE, None),
                lib.lccrf_distill_grad(FAKE, ODD, 10, 0, FAKE, FAKE, 4, 10, 3, t, None, None, FAKE, None))

    for t in (2.0 ** -126, 1e-6, 1.0, 1e9, 3e38):
        assert both(t) == (EALIGN, EALIGN), t
    for t in (1e-45, 1e-39, 2.0 ** -127, 0.0, -1.0, float("inf"), float("nan")):
        assert both(t) == (EINVAL, EINVAL), t


def test_eps(lib):
    """What is added to the variance: its root's inverse is taken in float, where nothing below the least normal float has one."""
    rows = ctypes.byref(_Rows(ODD, 8, 8))

    def both(eps, alone):
        return (lib.lccrf_group_norm(rows, 0, FAKE, FAKE, None, 2, 4, 8, 2, alone, eps, 1, FAKE, None, None, 0, None),
                lib.lccrf_group_norm_grad(rows, rows, 0, FAKE, FAKE, None, 2, 4, 8, 2, alone, eps, 1, None, FAKE, FAKE, FAKE, FAKE, 1 << 20, None))

    for alone in (0, 1):
        for eps in (2.0 ** -126, 1e-12, 1e-5, 1.0, 3e38):
            assert both(eps, alone) == (EALIGN, EALIGN), eps
        for eps in (1e-45, 1e-39, 0.0, -1e-5, float("inf"), float("nan")):
            assert both(eps, alone) == (EINVAL, EINVAL), eps
