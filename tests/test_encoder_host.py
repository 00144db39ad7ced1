"""The encoder without a GPU: what its entry points refuse, what they ask for, and the 64-bit reference of the GPU tests against
automatic differentiation and differences."""
import ctypes
import os

import pytest
import torch

import encoder_reference as ref
from paper_2308_03291_amd import binding, encoder

EINVAL, ENULL, EWS, EALIGN = -1, -2, -3, -4
FAKE = 4096  # an aligned "pointer" that is never dereferenced on these paths


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2308_03291_amd import build_ext
        build_ext.build()
    return binding.load_library()


def rows(data=FAKE):
    return encoder._Rows(data or 0, 8, 8)


def inputs(x=FAKE, dt=FAKE, Bm=FAKE, Cm=FAKE, z=None, A=FAKE, D=FAKE, dt_bias=FAKE):
    rows = [v for p in (x, dt, Bm, Cm, z) for v in (p or 0, 8, 8)]
    return encoder._ScanInputs(*rows, 8, 8, A or 0, D or 0, dt_bias or 0)


def test_embed_refuses(lib):
    f = lib.lccrf_embed
    assert f(FAKE, 0, 0, 8, 8, FAKE, 4, 1.0, FAKE, None) == EINVAL
    assert f(FAKE, 0, 9, 0, 8, FAKE, 4, 1.0, FAKE, None) == EINVAL
    assert f(FAKE, 2, 9, 8, 8, FAKE, 4, 1.0, FAKE, None) == EINVAL
    assert f(FAKE, 0, 9, 8, 8, FAKE, -1, 1.0, FAKE, None) == EINVAL
    for k in (0, 5, 8):
        args = [FAKE, 0, 9, 8, 8, FAKE, 4, 1.0, FAKE, None]
        args[k] = None
        assert f(*args) == ENULL
        args[k] = FAKE + 1
        assert f(*args) == EALIGN
    assert f(FAKE, 0, 9, 8, 8, FAKE, 0, 1.0, FAKE, None) == 0  # nothing to do, nothing enqueued
    assert f(FAKE, 0, 9, 8192, 8192, FAKE, 1 << 40, 1.0, FAKE, None) == EINVAL  # more threads than a launch has


def test_embed_grad_refuses(lib):
    need = lib.lccrf_embed_grad_workspace_bytes(32, 9, 8)
    assert need > 0 and need % 256 == 0
    f = lib.lccrf_embed_grad
    assert f(rows(), 0, FAKE, 4, 8, 0, 8, 1.0, FAKE, FAKE, need, None) == EINVAL
    assert f(rows(), 0, FAKE, -1, 8, 9, 8, 1.0, FAKE, FAKE, need, None) == EINVAL
    assert f(rows(), 0, FAKE, 1 << 16, 1 << 16, 9, 8, 1.0, FAKE, FAKE, need, None) == EINVAL
    assert f(None, 0, FAKE, 4, 8, 9, 8, 1.0, FAKE, FAKE, need, None) == ENULL
    assert f(rows(None), 0, FAKE, 4, 8, 9, 8, 1.0, FAKE, FAKE, need, None) == ENULL
    assert f(rows(), 0, None, 4, 8, 9, 8, 1.0, FAKE, FAKE, need, None) == ENULL
    assert f(rows(), 0, FAKE, 4, 8, 9, 8, 1.0, None, FAKE, need, None) == ENULL
    assert f(rows(), 0, FAKE, 4, 8, 9, 8, 1.0, FAKE, FAKE, need - 1, None) == EWS
    assert f(rows(), 0, FAKE, 4, 8, 9, 8, 1.0, FAKE, None, need, None) == EWS
    assert f(rows(), 0, FAKE, 4, 8, 9, 8, 1.0, FAKE, FAKE + 16, need, None) == EALIGN
    assert f(rows(FAKE + 2), 0, FAKE, 4, 8, 9, 8, 1.0, FAKE, FAKE, need, None) == EALIGN
    assert lib.lccrf_embed_grad_workspace_bytes(32, 0, 8) == 0 and lib.lccrf_embed_grad_workspace_bytes(-1, 9, 8) == 0


def test_conv_refuses(lib):
    f = lib.lccrf_conv

    def call(x=rows(), dt=0, w=FAKE, b=FAKE, st=FAKE, B=2, N=4, D=8, K=4, out=FAKE, fin=2 * FAKE):
        return f(x, dt, w, b, st, None, B, N, D, K, out, fin, None)

    assert [call(K=k) for k in (0, 1, 9)] == [EINVAL] * 3
    assert [call(B=0), call(N=0), call(D=0), call(dt=7), call(B=1 << 16, N=1 << 16)] == [EINVAL] * 5
    assert call(st=2 * FAKE) == EINVAL  # final over state
    assert [call(x=None), call(x=rows(None)), call(w=None), call(out=None)] == [ENULL] * 4
    assert [call(w=FAKE + 2), call(out=FAKE + 2), call(x=rows(FAKE + 1)), call(fin=FAKE + 1)] == [EALIGN] * 4
    need = lib.lccrf_conv_grad_workspace_bytes(2, 4, 8, 4)
    assert need > 0 and need % 256 == 0 and lib.lccrf_conv_grad_workspace_bytes(2, 4, 8, 9) == 0
    g = lib.lccrf_conv_grad

    def grad(dout=rows(), x=rows(), st=FAKE, dx=FAKE, dw=FAKE, dst=FAKE, ws=FAKE, n=need, K=4):
        return g(dout, x, 0, FAKE, FAKE, st, None, 2, 4, 8, K, dx, dw, FAKE, dst, ws, n, None)

    assert grad(K=1) == EINVAL and grad(st=None) == EINVAL
    assert [grad(dout=None), grad(x=None), grad(dx=None), grad(dw=None)] == [ENULL] * 4
    assert [grad(ws=None), grad(n=need - 1)] == [EWS] * 2
    assert [grad(ws=FAKE + 4), grad(dx=FAKE + 2)] == [EALIGN] * 2
    s = lib.lccrf_conv_step
    assert s(FAKE, 8, 0, FAKE, FAKE, FAKE, 2, 8, 1, FAKE, None) == EINVAL
    assert s(FAKE, 8, 0, FAKE, FAKE, None, 2, 8, 4, FAKE, None) == ENULL
    assert s(FAKE + 2, 8, 0, FAKE, FAKE, FAKE, 2, 8, 4, FAKE, None) == EALIGN


def test_scan_refuses(lib):
    need = lib.lccrf_state_scan_workspace_bytes(2, 4, 8, 16, 2)
    assert need > 0 and need % 256 == 0
    f = lib.lccrf_state_scan

    def call(block=None, dt=0, B=2, N=4, D=8, S=16, G=2, out=FAKE, ws=FAKE, n=need, saved=None):
        return f(ctypes.byref(block or inputs()), dt, None, B, N, D, S, G, FAKE, out, FAKE, saved, ws, n, None)

    assert [call(S=0), call(S=65), call(G=0), call(G=3), call(G=16), call(B=0), call(N=0), call(D=0), call(dt=3)] == [EINVAL] * 9
    assert [call(out=None), call(inputs(x=None)), call(inputs(dt=None)), call(inputs(Bm=None)), call(inputs(Cm=None)), call(inputs(A=None))] == [ENULL] * 6
    assert [call(ws=None), call(n=need - 1)] == [EWS] * 2
    assert [call(saved=FAKE + 16), call(ws=FAKE + 16), call(inputs(x=FAKE + 2)), call(inputs(z=FAKE + 2)), call(inputs(A=FAKE + 2))] == [EALIGN] * 5
    assert f(None, 0, None, 2, 4, 8, 16, 2, FAKE, FAKE, FAKE, None, FAKE, need, None) == ENULL
    # the state in front of every eighth position
    assert lib.lccrf_state_scan_saved_bytes(3, 17, 64, 16) == 3 * 3 * 64 * 16 * 4
    assert lib.lccrf_state_scan_saved_bytes(3, 17, 64, 13) == 3 * 3 * 64 * 16 * 4
    assert lib.lccrf_state_scan_saved_bytes(3, 17, 64, 65) == 0
    big = lib.lccrf_state_scan_grad_workspace_bytes(2, 4, 8, 16, 2, 0)
    small = lib.lccrf_state_scan_grad_workspace_bytes(2, 4, 8, 16, 2, 1)
    assert big > small > 0 and lib.lccrf_state_scan_grad_workspace_bytes(2, 4, 8, 16, 3, 1) == 0
    g = lib.lccrf_state_scan_grad

    def grad(block=None, dout=rows(), state=FAKE, saved=FAKE, n=small, S=16, **other):
        names = ("dx", "ddt", "dBm", "dCm", "dz", "dA", "dD", "ddt_bias", "dstate")
        values = {k: FAKE for k in names} | {"dz": None} | other
        return g(dout, ctypes.byref(block or inputs()), 0, None, 2, 4, 8, S, 2, state, saved, encoder._ScanGrads(*[v or 0 for v in values.values()]), FAKE, n, None)

    assert [grad(S=65), grad(dz=FAKE), grad(inputs(z=FAKE)), grad(state=None)] == [EINVAL] * 4
    assert [grad(dout=None), grad(dx=None), grad(ddt=None), grad(dBm=None), grad(dCm=None), grad(dA=None)] == [ENULL] * 6
    assert [grad(n=small - 1), grad(saved=None)] == [EWS] * 2
    assert [grad(dx=FAKE + 2), grad(dA=FAKE + 2), grad(saved=FAKE + 64)] == [EALIGN] * 3
    s = lib.lccrf_state_step
    assert s(ctypes.byref(inputs()), 0, 2, 8, 65, 2, FAKE, FAKE, None) == EINVAL
    assert s(ctypes.byref(inputs()), 0, 2, 8, 16, 2, None, FAKE, None) == ENULL
    assert s(ctypes.byref(inputs()), 0, 2, 8, 16, 2, FAKE + 2, FAKE, None) == EALIGN


def test_binding_refuses_cpu_tensors():
    t = torch.zeros
    with pytest.raises(ValueError):
        binding.lccrf_embed(t(4, 8), t(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        binding.lccrf_embed_grad(t(2, 3, 8), t(2, 3, dtype=torch.int32), 4)
    with pytest.raises(ValueError):
        binding.lccrf_conv(t(2, 3, 8), t(8, 4))
    with pytest.raises(ValueError):
        binding.lccrf_conv(t(2, 8), t(8, 4))
    with pytest.raises(ValueError):
        binding.lccrf_conv_step(t(2, 8), t(8, 4), None, None)
    with pytest.raises(ValueError):
        binding.lccrf_state_scan(t(2, 3, 8), t(2, 3, 8), t(8, 4), t(2, 3, 1, 4), t(2, 3, 1, 4))
    with pytest.raises(ValueError):
        binding.lccrf_state_step(t(2, 8), t(2, 8), t(8, 4), t(2, 1, 4), t(2, 1, 4), None, None, None, t(2, 8, 4))


def _leaf(*shape, g):
    return torch.randn(*shape, generator=g, dtype=torch.float64).requires_grad_(True)


def test_reference_of_the_convolution_is_its_own_derivative():
    g = torch.Generator().manual_seed(1)
    B, N, D, K = 3, 7, 5, 4
    x, w, b, st = _leaf(B, N, D, g=g), _leaf(D, K, g=g), _leaf(D, g=g), _leaf(B, K - 1, D, g=g)
    lens, dout = torch.tensor([7, 0, 4]), torch.randn(B, N, D, generator=g, dtype=torch.float64)
    on = (torch.arange(N)[None] < lens[:, None])[..., None]
    r = torch.cat([st, x * on], 1)
    loss = (torch.nn.functional.silu(sum(r[:, k:k + N] * w[:, k] for k in range(K)) + b) * on * dout).sum()
    want = torch.autograd.grad(loss, (x, w, b, st))
    got = ref.conv(x, w, b, lens, st, dout)
    for name, t in zip(("dx", "dweight", "dbias", "dstate"), want):
        assert torch.allclose(got[name], t, rtol=1e-12, atol=1e-12), name
    assert torch.allclose((got["out"] * dout).sum(), loss, rtol=1e-12)


def test_reference_of_the_scan_is_its_own_derivative():
    """By differences: the directional derivative of the loss along random directions, in 64 bits."""
    g = torch.Generator().manual_seed(2)
    B, N, W, S, G = 3, 6, 4, 3, 2
    def r(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)
    args = {"x": r(B, N, W), "dt": r(B, N, W), "A": -torch.exp(r(W, S)), "Bm": r(B, N, G, S), "Cm": r(B, N, G, S), "D": r(W), "z": r(B, N, W),
            "dt_bias": r(W), "lengths": torch.tensor([6, 0, 4]), "state": r(B, W, S)}
    dout = r(B, N, W)
    got = ref.scan(*args.values(), dout)
    names = {"x": "dx", "dt": "ddt", "A": "dA", "Bm": "dBm", "Cm": "dCm", "D": "dD", "z": "dz", "dt_bias": "ddt_bias", "state": "dstate"}
    eps = 1e-5
    for k, name in names.items():
        v = r(*args[k].shape)
        def loss(sign):
            moved = dict(args)
            moved[k] = args[k] + sign * eps * v
            return (ref.scan(*moved.values())["out"] * dout).sum()
        difference = float((loss(1) - loss(-1)) / (2 * eps))
        formula = float((got[name] * v).sum())
        assert abs(difference - formula) <= 1e-8 * (1 + abs(formula)) + 1e-7, name
        larger = ref.scan(*args.values(), dout, absolute=True)[name]
        assert (larger >= got[name].abs() - 1e-12).all(), f"{name}: its bound is below it"
