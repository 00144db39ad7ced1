"""The encoder's scan where inputs are infinite or far apart: what its formulas in 64 bits (tests/encoder_reference.py) make infinite is
infinite, what they make NaN is NaN, and all else is a number within the roundings of test_gpu_encoder.py."""
import pytest
import torch

import encoder_reference as ref
from test_gpu_encoder import DEV, TYPES, _dirty_memory, check, check_scan, crf, generator, normal, scan_inputs, scan_roundings  # noqa: F401

pytestmark = pytest.mark.gpu

INF = float("inf")
PER_CHANNEL = ("A", "D", "dt_bias")


def positive(g, t, B, N, D, S, G, *, gate=True):
    """Inputs above 0 but for A, so that sums of infinities have one sign; a state as well."""
    def above(*shape, dtype=t):
        return (torch.rand(shape, generator=g, device=DEV) + 0.25).to(dtype)
    inputs = {"x": above(B, N, D), "dt": normal(g, B, N, D, dtype=t) - 2, "A": -above(D, S, dtype=torch.float32) * 4, "Bm": above(B, N, G, S), "Cm": above(B, N, G, S),
              "D": above(D, dtype=torch.float32), "z": above(B, N, D) if gate else None, "dt_bias": normal(g, D, scale=0.1)}
    return inputs, above(B, D, S, dtype=torch.float32)


def same(got, want, bound, roundings, what):
    got64 = got.double().cpu()
    assert bool((torch.isnan(got64) == torch.isnan(want)).all()), f"{what}: NaN at {torch.isnan(got64).nonzero()[:3].tolist()}, not at {torch.isnan(want).nonzero()[:3].tolist()}"
    infinite = torch.isinf(want)
    assert bool((torch.isinf(got64) == infinite).all()) and bool((got64[infinite] == want[infinite]).all()), f"{what}: infinities"
    finite = torch.isfinite(want)
    assert torch.isfinite(bound[finite]).all()
    if finite.any():
        check(got.cpu()[finite], want[finite], bound[finite], roundings, what)


def rounds(inputs):
    B, N, D = inputs["x"].shape
    return scan_roundings(N, inputs["A"].shape[1], D, inputs["z"])


def forwards(crf, inputs, state, steps=True):
    """The scan and, position by position, its single-token form."""
    N = inputs["x"].shape[1]
    want, big = (ref.scan(*inputs.values(), None, state, absolute=a) for a in (False, True))
    R = rounds(inputs)
    out, final = crf.lccrf_state_scan(*inputs.values(), state=state)
    same(out, want["out"], big["out"], R, "out")
    same(final, want["final"], big["final"], R, "final")
    if steps:
        moving = state.clone()
        made = [crf.lccrf_state_step(*[v if k in PER_CHANNEL or v is None else v[:, l] for k, v in inputs.items()], moving) for l in range(N)]
        same(torch.stack(made, 1), want["out"], big["out"], R, "out by positions")
        same(moving, want["final"], big["final"], R, "final by positions")


def backwards(crf, inputs, state, dout):
    B, N, D = inputs["x"].shape
    want, big = (ref.scan(*inputs.values(), None, state, dout, absolute=a) for a in (False, True))
    R = rounds(inputs)
    for saved in (crf.state_scan_saved(inputs["x"], inputs["A"]), None):
        if saved is not None:
            crf.lccrf_state_scan(*inputs.values(), state=state, saved=saved)
        got = crf.lccrf_state_scan_grad(dout, *inputs.values(), state=state, saved=saved)
        for name in got._fields:
            if getattr(got, name) is not None:
                same(getattr(got, name), want[name], big[name], R + (B * N if name in ("dA", "dD", "ddt_bias") else 0), name)


STATES = (1, 2, 3, 4, 5, 7, 8, 9, 13, 16, 17, 24, 33, 50, 64)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("S", STATES)
@pytest.mark.parametrize("where", ("x", "dt", "state"))
def test_an_infinite_input(crf, t, S, where):
    """From where it is on, its channel is infinite, and no other: in a call for the prompt and in calls for single tokens."""
    g = generator(S)
    inputs, state = positive(g, t, 2, 19, 70, S, 2, gate=where != "dt")
    if where == "state":
        state[1, 40] = INF
    else:
        inputs[where][1, 6, 40] = INF
    forwards(crf, inputs, state)


@pytest.mark.parametrize("S", STATES)
@pytest.mark.parametrize("where", ("Bm", "Cm"))
def test_an_infinite_vector(crf, S, where):
    g = generator(S)
    inputs, state = positive(g, torch.float32, 2, 19, 70, S, 2)
    inputs[where][0, 6, 1, S - 1] = INF
    forwards(crf, inputs, state)


def an_infinite_gradient(crf, t, S, D, G):
    g = generator(S * D)
    inputs, state = positive(g, t, 2, 19, D, S, G, gate=D != 5)
    dout = (torch.rand(2, 19, D, generator=g, device=DEV) + 0.25).to(t)
    dout[1, 11, D - 1] = INF
    backwards(crf, inputs, state, dout)


def gradients_of_an_infinite_input(crf, S, D, G, where):
    g = generator(S * D)
    inputs, state = positive(g, torch.float32, 2, 19, D, S, G)
    inputs[where][(1, 11, D // 2) if where == "x" else (1, 11, G - 1, S - 1)] = INF
    backwards(crf, inputs, state, torch.rand(2, 19, D, generator=g, device=DEV) + 0.25)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("S", STATES)
def test_an_infinite_gradient(crf, t, S):
    an_infinite_gradient(crf, t, S, 64, 1)


@pytest.mark.parametrize("S", STATES)
@pytest.mark.parametrize("where", ("x", "Bm", "Cm"))
def test_gradients_of_an_infinite_input(crf, S, where):
    gradients_of_an_infinite_input(crf, S, 64, 1, where)


# Channels that fill one lane, a part of a tile, a tile and a part of another, tiles of several waves: lanes past them hold some again.
PARTS = [(1, 1), (5, 1), (3, 3), (70, 2), (130, 1), (250, 1)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("S", STATES)
@pytest.mark.parametrize("D,G", PARTS)
def test_an_infinite_gradient_in_part_of_a_tile(crf, t, S, D, G):
    an_infinite_gradient(crf, t, S, D, G)


@pytest.mark.parametrize("S", STATES)
@pytest.mark.parametrize("D,G", PARTS)
@pytest.mark.parametrize("where", ("x", "Bm", "Cm"))
def test_gradients_of_an_infinite_input_in_part_of_a_tile(crf, S, D, G, where):
    gradients_of_an_infinite_input(crf, S, D, G, where)


@pytest.mark.parametrize("width", range(1, 65))
def test_every_part_of_a_tile(crf, width):
    """The sums over the channels take every channel once, however many lanes hold it."""
    g = generator(width)
    inputs = scan_inputs(g, torch.float32, 2, 17, width, 8, 1)
    check_scan(crf, inputs, None, normal(g, 2, width, 8), normal(g, 2, 17, width))


@pytest.mark.parametrize("N", (1, 5, 8, 13, 16))
def test_an_infinite_input_at_the_last_position(crf, N):
    """No decay works on the state that it makes: the gradient by A is a number, wherever the last eight positions end."""
    g = generator(N)
    inputs, state = positive(g, torch.float32, 2, N, 70, 16, 1)
    inputs["x"][1, N - 1, 9] = INF
    backwards(crf, inputs, state, torch.rand(2, N, 70, generator=g, device=DEV) + 0.25)


@pytest.mark.parametrize("S", (4, 13, 24))
def test_infinities_in_a_sequence_that_is_cut(crf, S):
    """Every decay is above 0, so an infinite state stays what it is, though the decays of a segment together are below every float."""
    g = generator(S)
    inputs, state = positive(g, torch.float32, 1, 700, 6, S, 2)
    inputs["dt_bias"] += 4.0
    state[0, 1] = INF
    forwards(crf, inputs, state, steps=False)
    state[0, 1] = 1.0
    dout = torch.rand(1, 700, 6, generator=g, device=DEV) + 0.25
    dout[0, 690, 4] = INF
    backwards(crf, inputs, state, dout)


def test_gates_that_all_but_close(crf):
    """y silu(z) where y z is past the largest float and the result is not; the same of its gradient."""
    g = generator(3)
    inputs, state = positive(g, torch.float32, 2, 11, 70, 16, 1)
    inputs["z"] = torch.linspace(-80, -20, 70, device=DEV).repeat(2, 11, 1)
    inputs["x"][:, 3] = 5e36
    forwards(crf, inputs, state)
    inputs["x"][:, 3] = 1.0
    dout = torch.rand(2, 11, 70, generator=g, device=DEV) + 0.25
    dout[:, 3] = 1e37
    backwards(crf, inputs, state, dout)
