"""What the encoder's entry points launch, without a GPU: a stand-in for the HIP runtime (launch_recorder.cpp) writes launches down and
lets the one fail that a test names.  Pointers are made up; the host code looks at none of them."""
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2308_03291_amd", "liblccrf.so")
OK, EINVAL, ELAUNCH = 0, -1, -5

# Run in a process of its own, where no other copy of the runtime is: [call, fail_launch, fail_attribute] a line in, [status, launches] out.
PROGRAM = r'''
import ctypes, json, sys
recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
i, i64, f, vp, sz = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
P, BIG = 4096, 1 << 62
Rows, Inputs, Grads = i64 * 3, i64 * 20, i64 * 9
rows = Rows(P, 8, 8)
def inputs(z):
    return Inputs(*[v for p in (P, P, P, P, z) for v in (p, 8, 8)], 8, 8, P, P, P)
def byref(v):
    return ctypes.byref(v)
def embed(n, V, D, dt=0):
    return lib.lccrf_embed(vp(P), i(dt), i(V), i(D), i64(D), vp(P), i64(n), f(1.0), vp(P), None)
def embed_grad(B, N, V, D, dt=0):
    return lib.lccrf_embed_grad(byref(rows), i(dt), vp(P), i(B), i(N), i(V), i(D), f(1.0), vp(P), vp(P), sz(BIG), None)
def conv(B, N, D, K, dt=0):
    return lib.lccrf_conv(byref(rows), i(dt), vp(P), vp(P), None, None, i(B), i(N), i(D), i(K), vp(P), vp(P), None)
def conv_grad(B, N, D, K, dt=0):
    return lib.lccrf_conv_grad(byref(rows), byref(rows), i(dt), vp(P), vp(P), None, None, i(B), i(N), i(D), i(K), vp(P), vp(P), vp(P), None, vp(P), sz(BIG), None)
def conv_step(B, D, K, dt=0):
    return lib.lccrf_conv_step(vp(P), i64(D), i(dt), vp(P), vp(P), vp(P), i(B), i(D), i(K), vp(P), None)
def scan(B, N, D, S, G, saved=0, dt=0):
    return lib.lccrf_state_scan(byref(inputs(0)), i(dt), None, i(B), i(N), i(D), i(S), i(G), None, vp(P), vp(P), vp(saved or None), vp(P), sz(BIG), None)
def scan_grad(B, N, D, S, G, saved=0, dt=0):
    g = Grads(P, P, P, P, 0, P, P, P, 0)
    return lib.lccrf_state_scan_grad(byref(rows), byref(inputs(0)), i(dt), None, i(B), i(N), i(D), i(S), i(G), None, vp(saved or None), byref(g), vp(P), sz(BIG), None)
def state_step(B, D, S, G, dt=0):
    return lib.lccrf_state_step(byref(inputs(0)), i(dt), i(B), i(D), i(S), i(G), vp(P), vp(P), None)
def size(name, *a):
    fn = getattr(lib, name)
    fn.restype = sz
    return fn(*[i(v) for v in a])
answers = []
for call, launch, attribute in json.load(sys.stdin):
    recorder.recorder_reset(launch, attribute)
    rc = globals()[call[0]](*call[1:])
    made = []
    for k in range(recorder.recorder_count()):
        six = (ctypes.c_uint32 * 6)()
        recorder.recorder_get(k, six)
        made.append(list(six))
    answers.append([rc, made])
print(json.dumps(answers))
'''


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask([(call, arguments ...), ...], ...): (status, launches) of every call."""
    if not os.path.exists(LIB):
        from paper_2308_03291_amd import build_ext
        build_ext.build()
    recorder = str(tmp_path_factory.mktemp("recorder") / "librecorder.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", recorder, os.path.join(HERE, "launch_recorder.cpp")], check=True)

    def run(calls, launch=-1, attribute=0):
        lines = [[list(c), launch, attribute] for c in calls]
        out = subprocess.run([sys.executable, "-c", PROGRAM, recorder, LIB], input=json.dumps(lines), capture_output=True, text=True, timeout=60)
        assert out.returncode == 0, out.stderr
        return [(rc, made) for rc, made in json.loads(out.stdout)]

    return run


# Calls of several launches: segments and their join, partial sums, the forward pass inside the gradient.
SEVERAL = [("embed_grad", 4, 20, 100, 8), ("embed_grad", 4, 20, 200000, 65), ("conv_grad", 2, 40, 24, 4),
           ("scan", 2, 5000, 8, 4, 2), ("scan", 2, 5000, 8, 40, 2), ("scan", 2, 5000, 130, 16, 1, 4096),
           ("scan_grad", 2, 5000, 8, 4, 2, 4096), ("scan_grad", 2, 5000, 130, 16, 1), ("scan_grad", 2, 5000, 1000, 40, 1), ("scan_grad", 300, 20, 260, 8, 1)]


def test_a_launch_that_fails_is_reported(ask):
    """Whichever it is; and nothing goes out behind it."""
    for call in SEVERAL:
        (rc, made), = ask([call])
        assert rc == OK and len(made) > 1, (call, rc, made)
        for k in range(len(made)):
            (rc, got), = ask([call], launch=k)
            assert rc == ELAUNCH, f"{call}: launch {k} of {len(made)} failed, status {rc}"
            assert len(got) == k + 1, f"{call}: {len(got) - k - 1} launches behind the one that failed"
    (rc, _), = ask([("embed", 10, 9, 8)], launch=0)
    assert rc == ELAUNCH


def test_shared_memory_is_asked_for_before_anything_goes_out(ask):
    """8 states, groups of four tiles: more LDS than a kernel may have unasked; two segments and the forward pass come before it."""
    for call in (("scan_grad", 2, 5000, 250, 8, 1), ("scan_grad", 2, 5000, 250, 8, 1, 4096)):
        (rc, made), = ask([call], attribute=1)
        assert rc == ELAUNCH and made == [], f"{call}: status {rc}, {len(made)} launches"


# ---- sizes at their limits ------------------------------------------------------------------------------------

MOST = 2 ** 31 - 1024  # positions of a call


def up256(n):
    return -(-n // 256) * 256


def test_sizes_of_the_longest_sequences(ask):
    """Rounded up past 2^31 on the way: sizes of workspaces and numbers of workgroups at the limit, refusals past it."""
    def sizes(*calls):
        return [rc for rc, _ in ask([("size", *c) for c in calls])]
    for B, N in ((1, MOST), (1, MOST - 63), (MOST, 1), (3, MOST // 3)):
        blocks = -(-N // 8)
        assert sizes(("lccrf_state_scan_saved_bytes", B, N, 1, 1), ("lccrf_state_scan_saved_bytes", B, N, 3, 13)) == [up256(B * blocks * 16), up256(B * blocks * 4 * 3 * 16)]
        assert sizes(("lccrf_conv_grad_workspace_bytes", B, N, 1, 4)) == [2048 * 5 * 4]  # as many partial sums as workgroups
        need, grad, more = sizes(("lccrf_state_scan_workspace_bytes", B, N, 1, 1, 1), ("lccrf_state_scan_grad_workspace_bytes", B, N, 1, 1, 1, 1),
                                 ("lccrf_state_scan_grad_workspace_bytes", B, N, 1, 1, 1, 0))
        if B == 1:  # one wave by itself: two segments a SIMD, three in the gradient, but for what rounding their length up takes off
            assert 2000 * 20 <= need <= 2 * 1024 * 20 and 3000 * 32 <= grad <= 3 * 1024 * 32 + 1024
        assert 0 < need and 0 < grad and more == grad + up256(B * blocks * 16) + need
    assert sizes(*[(name, 1, MOST + 1, *rest) for name, *rest in (("lccrf_state_scan_saved_bytes", 1, 1), ("lccrf_state_scan_workspace_bytes", 1, 1, 1),
                                                                  ("lccrf_state_scan_grad_workspace_bytes", 1, 1, 1, 1), ("lccrf_conv_grad_workspace_bytes", 1, 4))]) == [0] * 4


def test_launches_of_the_longest_sequences(ask):
    for (rc, made), runs in zip(ask([("conv", 1, MOST, 1, 4), ("conv", 1, MOST, 1, 5, 1), ("conv", 2, MOST // 2, 1, 3)]), (-(-MOST // 64), -(-MOST // 60), 2 * -(-(MOST // 2) // 60))):
        assert rc == OK and made == [[-(-runs // 256), 1, 1, 256, 1, 1]]
    for rc, made in ask([("conv_grad", 1, MOST, 1, 4), ("scan", 1, MOST, 1, 1, 1), ("scan_grad", 1, MOST, 1, 1, 1)]):
        assert rc == OK and all(v[0] <= 1 << 20 for v in made), made
    for call in (("conv", 1, MOST + 1, 1, 4), ("conv", MOST + 1, 1, 1, 4), ("conv_grad", 1, MOST + 1, 1, 4), ("scan", 1, MOST + 1, 1, 1, 1),
                 ("scan_grad", 1, MOST + 1, 1, 1, 1), ("scan_grad", 1 << 16, 1 << 15, 1, 1, 1)):
        (rc, made), = ask([call])
        assert rc == EINVAL and made == [], call


WIDEST = 2 ** 31 - 1


def test_launches_of_the_widest_rows(ask):
    """Up to the documented widths every launch has a grid that the runtime takes; the stand-in refuses the others."""
    for call in (("conv_grad", 1, 1, 1 << 28, 2), ("conv_grad", 1, 1, 1 << 28, 8), ("conv_grad", 1, 1, WIDEST, 8, 1), ("conv", 1, 1, WIDEST, 4), ("conv", 1, 1, WIDEST, 4, 1),
                 ("conv_step", 1, WIDEST, 4), ("scan", 1, 1, 1 << 22, 64, 1), ("scan_grad", 1, 1, 1 << 22, 64, 1), ("scan_grad", 1, 1, 1 << 22, 62, 1 << 20, 4096),
                 ("state_step", 1, 1 << 22, 64, 1), ("embed", 2, 5, WIDEST), ("embed", 2, 5, WIDEST, 1)):
        (rc, made), = ask([call])
        assert rc == OK and made, (call, rc, made)
        assert all(v[0] * v[3] < 2 ** 32 for v in made), (call, made)


def test_what_no_grid_can_hold_is_refused_first(ask):
    for call in (("conv", 8, 64, WIDEST, 4), ("conv_step", 64, WIDEST - 3, 4), ("scan", 1 << 23, 64, 64, 4, 1), ("scan_grad", 1 << 23, 64, 64, 4, 1), ("scan_grad", 8192, 8192, 64, 64, 1),
                 ("state_step", 1 << 16, 1 << 16, 64, 1), ("embed_grad", 1 << 14, 1 << 14, 100, 1 << 13), ("embed_grad", 2, 5, 1 << 30, 1 << 6), ("embed", 1 << 25, 100, 1 << 20)):
        (rc, made), = ask([call])
        assert rc == EINVAL and made == [], (call, rc, made)
