"""Scalars of the layers of include/lccrf_layers.h at the ends of what their header allows, without a GPU: what is refused."""
import os

import pytest

from paper_2308_03291_amd import binding

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
