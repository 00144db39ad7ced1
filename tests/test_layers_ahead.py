"""Which positions the layers' kernels ask for ahead of those that they work on (csrc/lccrf_ahead.h), compiled for the host."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2308_03291_amd", "csrc")
MOST = 2 ** 31 - 1024  # positions of a call
BATCH = 4              # positions in flight of a thread

SOURCE = '''
#include "lccrf_ahead.h"
extern "C" int before(int l, int more, int stop) { return lccrf::enc::before(l, more, stop); }
extern "C" int or_last(int l, int more, int stop) { return lccrf::enc::or_last(l, more, stop); }
'''


@pytest.fixture(scope="module")
def ahead(tmp_path_factory):
    folder = tmp_path_factory.mktemp("ahead")
    (folder / "ahead.cpp").write_text(SOURCE)
    lib = str(folder / "libahead.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-ftrapv", "-shared", "-fPIC", "-I", CSRC, "-o", lib, str(folder / "ahead.cpp")], check=True)
    return ctypes.CDLL(lib)


@pytest.mark.parametrize("N", (1, 3, 1000, 5000, MOST - 1500, MOST - 769, MOST - 1, MOST))
@pytest.mark.parametrize("high", (1, 2, 64, 256))
def test_positions_ahead_stay_inside(ahead, N, high):
    """As the norm's passes over a sequence go: a thread's turns of four positions, `high` apart, the next turn asked for in each; the last turns of every thread."""
    for ty in {0, 1, high // 2, high - 1}:
        turn = BATCH * high
        l = ty + max(0, (N - 1 - ty) // turn - 2) * turn
        while True:
            for u in range(BATCH):
                at = ahead.or_last(l, u * high, N)
                assert at == min(l + u * high, N - 1), (N, high, l, u, at)
                assert bool(ahead.before(l, u * high, N)) == (l + u * high < N), (N, high, l, u)
            if l >= N:
                break
            l += turn
            assert l < 2 ** 31
