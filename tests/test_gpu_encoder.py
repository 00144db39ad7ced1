"""The encoder's operators on the GPU against their formulas in 64 bits (tests/encoder_reference.py).

Tolerances.  A result is off by half a step of its own type (rounded once), and by what float arithmetic loses before: u = 2^-24 for every
rounding, times the sum of the absolute values of what is added up (the reference with ``absolute``).  Roundings are counted
generously below, at most a factor of a few too many; a wrong term is off by 10^3 times that and more.
"""
import pytest
import torch

import encoder_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda"
TYPES = (torch.float32, torch.bfloat16)


@pytest.fixture(scope="module")
def crf():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2308_03291_amd import binding
    binding.load_library()
    return binding


@pytest.fixture(autouse=True)
def _dirty_memory(monkeypatch):
    """What the binding allocates starts as all-ones bytes (NaN, -1): nothing may rely on what memory held, or leave it."""
    from paper_2308_03291_amd import encoder
    empty, empty_like = torch.empty, torch.empty_like

    class Dirty:
        def __getattr__(self, name):
            return getattr(torch, name)

        @staticmethod
        def empty(*a, **k):
            t = empty(*a, **k)
            t.view(torch.uint8).fill_(0xFF) if t.numel() else None
            return t

        @staticmethod
        def empty_like(x):
            t = empty_like(x)
            t.view(torch.uint8).fill_(0xFF)
            return t

    monkeypatch.setattr(encoder, "torch", Dirty())
    yield


def generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def strided(g, *shape, dtype):
    """Dense rows inside wider ones, from an odd element on."""
    wide = normal(g, *shape[:-1], 2 * shape[-1] + 3, dtype=dtype)
    return wide[..., 1:1 + shape[-1]]


def check(got, want, bound, roundings, what):
    """bound: the sum of absolute values (or its largest possible value), of the result's shape or one number."""
    got, t = got.detach(), got.dtype
    half = torch.finfo(t).eps / 2
    got = got.double().cpu()
    assert got.shape == want.shape, f"{what}: {tuple(got.shape)} for {tuple(want.shape)}"
    tol = half * want.abs() + roundings * U * (1 + half) * bound + U * torch.as_tensor(bound).max() + 1e-37
    assert not torch.isnan(got).any(), f"{what}: NaN at {torch.isnan(got).nonzero()[:4].tolist()}"
    off = (got - want).abs()
    worst = (off - tol).flatten().argmax()
    assert (off <= tol).all(), f"{what}: {got.flatten()[worst]} for {want.flatten()[worst]} (allowed {tol.flatten()[worst] if tol.dim() else tol}), {int((off > tol).sum())} of {off.numel()}"


# ---- embedding ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("V,D,shape", [(1, 1, (1,)), (7, 3, (5,)), (100, 8, (3, 4)), (50, 33, (2, 9)), (4099, 301, (7, 11)), (300, 1024, (5, 130)), (9, 5000, (3,)), (5, 64, (0, 4))])
def test_embed(crf, t, V, D, shape):
    g = generator(V + D)
    ids = torch.randint(-2, V + 2, shape, generator=g, device=DEV).to(torch.int32)
    for table in (normal(g, V, D, dtype=t), strided(g, V, D, dtype=t)):
        for scale in (1.0, 3.25):
            check(crf.lccrf_embed(table, ids, scale=scale), w := ref.embed(table, ids, scale), w.abs(), 1 if w.numel() else 0, "embed") if ids.numel() else \
                crf.lccrf_embed(table, ids, scale=scale)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kind", ("spread", "one", "runs", "heavy", "padding", "none"))
@pytest.mark.parametrize("V,D,B,N", [(1, 8, 1, 33), (3, 5, 2, 32), (64, 3, 4, 50), (65, 40, 1, 1), (1000, 301, 8, 77), (70001, 16, 16, 257), (2100, 1024, 3, 300)])
def test_embed_grad(crf, t, kind, V, D, B, N):
    g = generator(V * 7 + D)
    n = B * N
    if kind == "spread":
        ids = torch.randint(0, V, (n,), generator=g, device=DEV)
    elif kind == "one":
        ids = torch.full((n,), V - 1, device=DEV)
    elif kind == "runs":  # 31, 32 and 33 of a token, in turn: around the length from which a row is cut
        sizes = torch.tensor([31, 32, 33, 64, 65] * (n // 31 + 1), device=DEV)
        ids = torch.repeat_interleave(torch.arange(len(sizes), device=DEV) % V, sizes)[:n][torch.randperm(n, generator=g, device=DEV)]
    elif kind == "heavy":  # as in text
        ids = (float(V) ** torch.rand(n, generator=g, device=DEV, dtype=torch.float64) - 1).long().clamp(0, V - 1)
    else:
        ids = torch.full((n,), -1 if kind == "none" else 0, device=DEV)
        if kind == "padding":
            ids = torch.randint(-V, 2 * V, (n,), generator=g, device=DEV)
    ids = ids.to(torch.int32).view(B, N)
    for dout in (normal(g, B, N, D, dtype=t), strided(g, B, N, D, dtype=t), normal(g, B, 1, D, dtype=t).expand(B, N, D)):
        got = crf.lccrf_embed_grad(dout, ids, V, scale=1.5)
        most = int(torch.bincount(ids.flatten().long().clamp(0, V - 1).cpu(), minlength=V).max())
        check(got, ref.embed_grad(dout, ids, V, 1.5), ref.embed_grad(dout, ids, V, 1.5, absolute=True), most + 2, f"embed_grad {kind}")
        assert torch.equal(got, crf.lccrf_embed_grad(dout, ids, V, scale=1.5)), "not the same again"


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("offset", (0, 1, 3))
@pytest.mark.parametrize("V,D,B,N", [(180001, 101, 3, 41), (9001, 2001, 2, 40), (300007, 60, 1, 1), (180001, 101, 0, 5)])
def test_embed_grad_of_few_positions(crf, t, offset, V, D, B, N):
    """Tables of which few rows hold anything, rows and the table itself beginning anywhere; one token holds half of the positions."""
    g = generator(V + D + B * N + offset)
    ids = torch.randint(0, V, (B, N), generator=g, device=DEV, dtype=torch.int32)
    if B:
        ids.view(-1)[::2] = V - 1
        ids.view(-1)[0] = 0
    dout = normal(g, B, N, D, dtype=t)
    memory = torch.full((V * D + 16,), float("nan"), dtype=t, device=DEV)
    out = memory[offset:offset + V * D].view(V, D)
    got = crf.lccrf_embed_grad(dout, ids, V, scale=0.7, out=out)
    assert got.data_ptr() == out.data_ptr()
    assert bool(memory[:offset].isnan().all()) and bool(memory[offset + V * D:].isnan().all())
    held = torch.unique(ids.flatten().long())
    if B:
        check(got[held], ref.embed_grad(dout, ids, V, 0.7)[held.cpu()], ref.embed_grad(dout, ids, V, 0.7, absolute=True)[held.cpu()], B * N + 2, "grad")
    empty = torch.ones(V, dtype=torch.bool, device=DEV)
    empty[held] = False
    assert not bool(got[empty].count_nonzero())


def test_embed_grad_of_nothing(crf):
    out = crf.lccrf_embed_grad(torch.empty(0, 5, 8, device=DEV), torch.empty(0, 5, dtype=torch.int32, device=DEV), 70)
    assert out.shape == (70, 8) and (out == 0).all()
    out = crf.lccrf_embed_grad(torch.ones(3, 8, device=DEV), torch.tensor([2, 2, -1], dtype=torch.int32, device=DEV), 4)
    assert out[:, 0].tolist() == [0, 0, 2, 0]


# ---- convolution ----------------------------------------------------------------------------------------------

def conv_lengths(B, N, g):
    lens = torch.randint(0, N + 1, (B,), generator=g, device=DEV).to(torch.int32)
    lens[0] = 0
    lens[-1] = N + 3  # clamped
    return lens


CONV = [(1, 1, 1), (2, 2, 3), (3, 5, 4), (2, 9, 7), (3, 33, 8), (2, 66, 20), (4, 130, 301), (2, 17, 1001)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("K", range(2, 9))
@pytest.mark.parametrize("B,N,D", CONV)
def test_conv_and_gradient(crf, t, K, B, N, D):
    g = generator(1000 * K + D)
    w, b = normal(g, D, K, scale=K ** -0.5), normal(g, D, scale=0.1)
    for variant in range(3):
        bias, lens = (None, None) if variant == 1 else (b, conv_lengths(B, N, g))
        state = None if variant == 0 else normal(g, B, K - 1, D, dtype=t)
        x = strided(g, B, N, D, dtype=t) if variant < 2 else normal(g, 1, N, D, dtype=t).expand(B, N, D)
        dout = normal(g, B, N, D, dtype=t) if variant < 2 else strided(g, B, N, D, dtype=t)
        want, big = ref.conv(x, w, bias, lens, state, dout), ref.conv(x, w, bias, lens, state, dout, absolute=True)
        out, final = crf.lccrf_conv(x, w, bias, lens, state=state)
        P = float(big["pre"].max())
        check(out, want["out"], big["pre"], 2 * K + 10 + 2 * P, "out")
        assert torch.equal(final.double().cpu(), want["final"]), "final"
        got = crf.lccrf_conv_grad(dout, x, w, bias, lens, state=state)
        E = (K + 14) * (1 + P)
        check(got.dx, want["dx"], big["dx"], E + K, "dx")
        check(got.dweight, want["dweight"], big["dweight"], E + B * N, "dweight")
        assert (got.dbias is None) == (bias is None) and (got.dstate is None) == (state is None)
        if bias is not None:
            check(got.dbias, want["dbias"], big["dbias"], E + B * N, "dbias")
        if state is not None:
            check(got.dstate, want["dstate"], big["dstate"], E + K, "dstate")
        again = crf.lccrf_conv_grad(dout, x, w, bias, lens, state=state)
        assert all(torch.equal(p, q) for p, q in zip(got, again) if p is not None), "not the same again"


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("K,D", [(2, 5), (3, 64), (4, 301), (8, 12)])
def test_conv_goes_on_where_it_stopped(crf, t, K, D):
    """One call, the same in two, and position by position: the same numbers."""
    g = generator(K * D)
    B, N, cut = 3, 21, 9
    x, w, b = normal(g, B, N, D, dtype=t), normal(g, D, K), normal(g, D)
    state = normal(g, B, K - 1, D, dtype=t)
    whole, last = crf.lccrf_conv(x, w, b, state=state)
    first, mid = crf.lccrf_conv(x[:, :cut], w, b, state=state)
    second, end = crf.lccrf_conv(x[:, cut:], w, b, state=mid)
    assert torch.equal(torch.cat([first, second], 1), whole) and torch.equal(end, last)
    moving = state.clone()
    for l in range(N):
        one = crf.lccrf_conv_step(x[:, l], w, b, moving)
        assert torch.equal(one, whole[:, l]), l
    assert torch.equal(moving, last)


# ---- scan -----------------------------------------------------------------------------------------------------

def scan_inputs(g, t, B, N, D, S, G, *, gate=True, rich=True, step=0.05, views=False):
    make = (lambda *s: strided(g, *s, dtype=t)) if views else (lambda *s: normal(g, *s, dtype=t))
    lead = (B,) if N is None else (B, N)
    bias = torch.log(torch.expm1(torch.rand(D, generator=g, device=DEV) * step * 2 + 1e-3))
    return {"x": make(*lead, D), "dt": make(*lead, D) * 0.5 if not views else make(*lead, D),
            "A": -torch.exp(normal(g, D, S, scale=0.5)) * (1 + torch.arange(S, device=DEV) % 7), "Bm": make(*lead, G, S), "Cm": make(*lead, G, S),
            "D": normal(g, D) if rich else None, "z": make(*lead, D) if gate else None, "dt_bias": bias if rich else None}


def scan_roundings(N, S, D, z):
    """A path through the recursion: per position the product's, the exponential's and the addition's roundings; the decays' own
    errors, 10 u |step A| each, weigh at most e^-20 of the whole beyond a sum of 20; then the states and channels summed."""
    return 2 * (232 + 4 * N + S + D + (0 if z is None else 2 * float(z.float().abs().max())))


def check_scan(crf, inputs, lens, state, dout, saved=True):
    x = inputs["x"]
    B, N, D = x.shape
    S = inputs["A"].shape[1]
    want = ref.scan(*inputs.values(), lens, state, dout)
    big = ref.scan(*inputs.values(), lens, state, dout, absolute=True)
    R = scan_roundings(N, S, D, inputs["z"])
    keep = crf.state_scan_saved(x, inputs["A"]) if saved else None
    out, final = crf.lccrf_state_scan(*inputs.values(), lens, state=state, saved=keep)
    check(out, want["out"], big["out"], R, "out")
    check(final, want["final"], big["final"], R, "final")
    if dout is None:
        return
    got = crf.lccrf_state_scan_grad(dout, *inputs.values(), lens, state=state, saved=keep)
    for name in got._fields:
        v = getattr(got, name)
        there = {"dz": inputs["z"], "dD": inputs["D"], "ddt_bias": inputs["dt_bias"], "dstate": state}.get(name, x)
        assert (v is None) == (there is None), name
        if v is not None:
            check(v, want[name], big[name], R + (B * N if name in ("dA", "dD", "ddt_bias") else 0), name)
    again = crf.lccrf_state_scan_grad(dout, *inputs.values(), lens, state=state, saved=keep)
    assert all(torch.equal(p, q) for p, q in zip(got, again) if p is not None), "not the same again"


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("S", (1, 3, 4, 5, 8, 13, 16, 17, 32, 33, 48, 50, 64))
@pytest.mark.parametrize("B,N,D,G", [(1, 1, 1, 1), (2, 8, 3, 3), (3, 23, 70, 2), (2, 40, 130, 1)])
def test_scan_states(crf, t, S, B, N, D, G):
    g = generator(S * 31 + D)
    inputs = scan_inputs(g, t, B, N, D, S, G, views=D == 70)
    check_scan(crf, inputs, None, normal(g, B, D, S), normal(g, B, N, D, dtype=t))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("gate,rich,carry,ragged", [(False, True, False, True), (True, False, True, True), (False, False, True, False), (True, True, True, True)])
@pytest.mark.parametrize("B,N,D,S,G", [(5, 37, 24, 16, 1), (4, 64, 300, 16, 1), (3, 130, 257, 13, 1), (2, 200, 514, 16, 2), (3, 90, 96, 24, 4), (2, 300, 20, 4, 20)])
def test_scan_shapes(crf, t, gate, rich, carry, ragged, B, N, D, S, G):
    """Ragged and full lengths, zero among them; one workgroup and several a group; one segment and several."""
    g = generator(B * N + D)
    inputs = scan_inputs(g, t, B, N, D, S, G, gate=gate, rich=rich, views=True)
    lens = None
    if ragged:
        lens = conv_lengths(B, N, g)
    state = normal(g, B, D, S) if carry else None
    check_scan(crf, inputs, lens, state, strided(g, B, N, D, dtype=t), saved=gate)


@pytest.mark.parametrize("S", (3, 8, 16, 24))
@pytest.mark.parametrize("D,G", [(201, 3), (130, 2), (260, 4), (1001, 7), (258, 2)])
def test_groups_that_fill_no_tile(crf, S, D, G):
    """Waves that reach from a group into the next."""
    g = generator(S * D)
    inputs = scan_inputs(g, torch.float32, 3, 83, D, S, G, gate=D != 130)
    check_scan(crf, inputs, conv_lengths(3, 83, g), normal(g, 3, D, S), normal(g, 3, 83, D))


def test_what_is_not_a_number_stays_in_its_channel(crf):
    g = generator(44)
    inputs = scan_inputs(g, torch.float32, 2, 40, 70, 16, 1)
    want, _ = crf.lccrf_state_scan(*inputs.values())
    inputs["dt"] = inputs["dt"].clone()
    inputs["dt"][1, 11, 5] = float("nan")
    out, final = crf.lccrf_state_scan(*inputs.values())
    assert torch.isnan(out[1, 11:, 5]).all() and torch.isnan(final[1, 5]).all()
    out[1, 11:, 5] = want[1, 11:, 5]
    assert torch.equal(out, want)
    ids = torch.tensor([0, 2], dtype=torch.int32, device=DEV)
    assert torch.isnan(crf.lccrf_embed(inputs["dt"][1, 9:12], ids)).nonzero().tolist() == [[1, 5]]


@pytest.mark.parametrize("t", TYPES)
def test_scan_of_a_long_sequence(crf, t):
    """Cut into segments, every one of them needed: slow decays carry the first positions to the end."""
    g = generator(77)
    inputs = scan_inputs(g, t, 2, 2500, 8, 4, 2, step=0.0005)
    lens = torch.tensor([2500, 1111], dtype=torch.int32, device=DEV)
    check_scan(crf, inputs, lens, normal(g, 2, 8, 4), normal(g, 2, 2500, 8, dtype=t))


def test_scan_of_a_full_chip(crf):
    """So many sequences that none is cut."""
    g = generator(78)
    inputs = scan_inputs(g, torch.bfloat16, 300, 70, 260, 8, 1)
    check_scan(crf, inputs, conv_lengths(300, 70, g), None, normal(g, 300, 70, 260, dtype=torch.bfloat16))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("S,G,D", [(1, 1, 5), (4, 2, 6), (8, 1, 33), (13, 3, 9), (16, 2, 514), (32, 1, 40), (50, 1, 7), (64, 4, 64)])
def test_scan_goes_on_where_it_stopped(crf, t, S, G, D):
    """In two calls, the second over its own state, and position by position, against the formula of the whole."""
    g = generator(S * D)
    B, N, cut = 3, 19, 7
    inputs = scan_inputs(g, t, B, N, D, S, G)
    state = normal(g, B, D, S)
    want, big = ref.scan(*inputs.values(), None, state), ref.scan(*inputs.values(), None, state, absolute=True)
    R = scan_roundings(N, S, D, inputs["z"])
    def part(a, b):
        return [v if k in ("A", "D", "dt_bias") or v is None else v[:, a:b] for k, v in inputs.items()]
    first, mid = crf.lccrf_state_scan(*part(0, cut), state=state)
    second, end = crf.lccrf_state_scan(*part(cut, N), state=mid, final=mid)
    assert end is mid
    check(torch.cat([first, second], 1), want["out"], big["out"], R, "out in two")
    check(end, want["final"], big["final"], R, "final in two")
    moving = state.clone()
    steps = [crf.lccrf_state_step(*[v if k in ("A", "D", "dt_bias") or v is None else v[:, l] for k, v in inputs.items()], moving) for l in range(N)]
    check(torch.stack(steps, 1), want["out"], big["out"], R, "out by positions")
    check(moving, want["final"], big["final"], R, "final by positions")


@pytest.mark.parametrize("gate,rich", [(True, True), (False, False)])
@pytest.mark.parametrize("B", (1, 2, 3, 64, 513))
def test_step_of_many_streams(crf, B, gate, rich):
    """Batches of one to several streams a thread, rows of wider tensors."""
    g = generator(B)
    D, S, G = (2048, 16, 1) if B > 100 else (96, 16, 2)
    inputs = scan_inputs(g, torch.bfloat16, B, None, D, S, G, gate=gate, rich=rich, views=True)
    state = normal(g, B, D, S)
    one = {k: v if k in ("A", "D", "dt_bias") or v is None else v[:, None] for k, v in inputs.items()}
    want, big = ref.scan(*one.values(), None, state), ref.scan(*one.values(), None, state, absolute=True)
    out = crf.lccrf_state_step(*inputs.values(), state)
    R = scan_roundings(1, S, D, inputs["z"])
    check(out, want["out"][:, 0], big["out"][:, 0], R, "out")
    check(state, want["final"], big["final"], R, "state")


# ---- what must not be read, values at the ends, places and streams --------------------------------------------

@pytest.mark.parametrize("bad", (float("nan"), float("inf"), -float("inf")))
def test_positions_past_the_end_are_not_looked_at(crf, bad):
    g = generator(5)
    B, N, D, S, K = 3, 45, 70, 16, 4
    t = torch.bfloat16
    lens = torch.tensor([45, 0, 19], dtype=torch.int32, device=DEV)
    past = torch.arange(N, device=DEV)[None] >= lens[:, None]
    inputs = scan_inputs(g, t, B, N, D, S, 1)
    dout = normal(g, B, N, D, dtype=t)
    spoiled = {k: v.clone() if k not in ("A", "D", "dt_bias") else v for k, v in inputs.items()}
    for k in ("x", "dt", "Bm", "Cm", "z"):
        spoiled[k][past] = bad
    dout2 = dout.clone()
    dout2[past] = bad
    w, b = normal(g, D, K), normal(g, D)
    clean = [*crf.lccrf_state_scan(*inputs.values(), lens), *crf.lccrf_state_scan_grad(dout, *inputs.values(), lens),
             *crf.lccrf_conv(inputs["x"], w, b, lens), *crf.lccrf_conv_grad(dout, inputs["x"], w, b, lens)]
    dirty = [*crf.lccrf_state_scan(*spoiled.values(), lens), *crf.lccrf_state_scan_grad(dout2, *spoiled.values(), lens),
             *crf.lccrf_conv(spoiled["x"], w, b, lens), *crf.lccrf_conv_grad(dout2, spoiled["x"], w, b, lens)]
    for p, q in zip(clean, dirty):
        if p is not None:
            assert torch.equal(p, q)
            if p.dim() >= 3 and p.shape[:2] == (B, N):
                assert (p[past] == 0).all()


def test_values_at_the_ends(crf):
    """Steps from vanishing to very large, states that are forgotten at once (A = -inf) or kept for good (A = 0), closed and open gates."""
    g = generator(6)
    B, N, D, S = 2, 21, 64, 4
    inputs = scan_inputs(g, torch.float32, B, N, D, S, 1)
    inputs["dt"] = torch.linspace(-80, 40, D, device=DEV).expand(B, N, D)
    inputs["dt_bias"] = None
    inputs["z"] = torch.linspace(-100, 100, D, device=DEV).flip(0).expand(B, N, D)
    inputs["A"][:, 0] = 0.0
    inputs["A"][:, 1] = -1e30
    state = normal(g, B, D, S)
    check_scan(crf, inputs, None, state, None)
    inputs["A"][:, 1] = -float("inf")
    lens = torch.tensor([21, 5], dtype=torch.int32, device=DEV)
    check_scan(crf, inputs, lens, state, None)


def test_small_steps_keep_their_precision(crf):
    """log(1 + exp(v)) near 0: the state after one position is step x Bm, step as small as 1e-20."""
    D = 256
    v = torch.linspace(-46, 20, D, device=DEV)
    one = torch.ones(1, 1, D, device=DEV)
    _, final = crf.lccrf_state_scan(one, v.expand(1, 1, D), torch.zeros(D, 1, device=DEV), torch.ones(1, 1, 1, 1, device=DEV), torch.ones(1, 1, 1, 1, device=DEV))
    want = torch.logaddexp(v.double(), torch.zeros_like(v.double()))
    assert float(((final[0, :, 0].double() - want) / want).abs().max()) <= 8 * U


def test_offsets_past_32_bits(crf):
    """Sequences 2^31 elements and more apart, and a table of more than 2^32 bytes."""
    far, N, D = 2 ** 31 + 64, 9, 40
    g = generator(7)
    t = torch.bfloat16
    big = torch.empty(far + N * 2 * D, dtype=t, device=DEV)
    def place(v):
        view = big.as_strided((2, *v.shape[1:]), (far, *v.stride()[1:]))
        view.copy_(v)
        return view
    inputs = scan_inputs(g, t, 2, N, D, 4, 1)
    want = crf.lccrf_state_scan(*inputs.values())
    grads = crf.lccrf_state_scan_grad(inputs["z"], *inputs.values())
    w = normal(g, D, 4)
    conv = [*crf.lccrf_conv(inputs["x"], w), *crf.lccrf_conv_grad(inputs["z"], inputs["x"], w)[:2]]
    for k in ("x", "dt", "Bm", "Cm", "z"):
        moved = dict(inputs)
        moved[k] = place(inputs[k])
        got = crf.lccrf_state_scan(*moved.values())
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), k
        got = crf.lccrf_state_scan_grad(inputs["z"], *moved.values())
        assert all(torch.equal(p, q) for p, q in zip(got, grads) if p is not None), k
    x = place(inputs["x"])
    got = [*crf.lccrf_conv(x, w), *crf.lccrf_conv_grad(inputs["z"], x, w)[:2]]
    assert all(torch.equal(p, q) for p, q in zip(got, conv))
    dout = place(inputs["z"])
    ids = torch.arange(2 * N, device=DEV).view(2, N).to(torch.int32)
    assert torch.equal(crf.lccrf_embed_grad(dout, ids, 2 * N).view(2, N, D), inputs["z"])
    del big, x, dout, moved
    V = 2 ** 32 // (D * 2) + 5
    table = torch.empty(V, D, dtype=t, device=DEV)
    ids = torch.tensor([V - 1, 0, V // 2], dtype=torch.int32, device=DEV)
    table[ids.long()] = rows = normal(g, 3, D, dtype=t)
    assert torch.equal(crf.lccrf_embed(table, ids), rows)
    got = crf.lccrf_embed_grad(rows, ids, V)
    assert torch.equal(got[ids.long()], rows) and int((got != 0).any(1).sum()) == 3


def calls(crf, s):
    """All operators once, into buffers that are given."""
    crf.lccrf_embed(s["table"], s["ids"], scale=2.0, out=s["e"])
    crf.lccrf_conv(s["e"], s["w"], s["b"], s["lens"], out=s["c"], final=s["cf"])
    crf.lccrf_state_scan(s["c"], s["dt"], s["A"], s["Bm"], s["Cm"], s["D"], s["z"], s["dt_bias"], s["lens"], saved=s["saved"], out=s["o"], final=s["sf"])
    g = crf.lccrf_state_scan_grad(s["dout"], s["c"], s["dt"], s["A"], s["Bm"], s["Cm"], s["D"], s["z"], s["dt_bias"], s["lens"], saved=s["saved"])
    k = crf.lccrf_conv_grad(g.dx, s["e"], s["w"], s["b"], s["lens"])
    table = crf.lccrf_embed_grad(k.dx, s["ids"], s["table"].shape[0], scale=2.0)
    one = crf.lccrf_conv_step(s["c"][:, 0], s["w"], s["b"], s["cf"])
    step = crf.lccrf_state_step(one, s["dt"][:, 0], s["A"], s["Bm"][:, 0], s["Cm"][:, 0], s["D"], s["z"][:, 0], s["dt_bias"], s["sf"])
    return [s["o"], s["cf"], s["sf"], *(v for v in g if v is not None), *(v for v in k if v is not None), table, step]


def state_of_calls(crf, seed, t=torch.bfloat16, B=3, N=150, D=72, S=16, V=50):
    g = generator(seed)
    i = scan_inputs(g, t, B, N, D, S, 1)
    s = {**i, "table": normal(g, V, D, dtype=t), "ids": torch.randint(-1, V, (B, N), generator=g, device=DEV).to(torch.int32), "w": normal(g, D, 4), "b": normal(g, D),
         "lens": torch.tensor([N, 77, 1], dtype=torch.int32, device=DEV), "dout": normal(g, B, N, D, dtype=t)}
    s |= {"e": torch.empty_like(i["x"]), "c": torch.empty_like(i["x"]), "o": torch.empty_like(i["x"]), "cf": torch.empty(B, 3, D, dtype=t, device=DEV),
          "sf": torch.empty(B, D, S, device=DEV), "saved": crf.state_scan_saved(i["x"], i["A"])}
    return s


def test_another_stream(crf):
    """Work goes to the current stream, behind what that stream still has to do."""
    s = state_of_calls(crf, 11)
    want = [v.clone() for v in calls(crf, s)]
    side = torch.cuda.Stream()
    table = s["table"].clone()
    s["table"].zero_()
    big = torch.randn(4096, 4096, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            big = big @ big * 1e-2
        s["table"].copy_(table)
        got = calls(crf, s)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_captured_in_a_graph(crf):
    s = state_of_calls(crf, 12)
    other = state_of_calls(crf, 13)
    calls(crf, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = calls(crf, s)
    for rep in range(4):
        for k in ("table", "ids", "dt", "Bm", "Cm", "z", "dout"):
            s[k].copy_(state_of_calls(crf, 20 + rep)[k])
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in inside]
        eager = calls(crf, s)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, eager)), f"replay {rep}"
        calls(crf, other)


def test_refusals(crf):
    f32, bf16 = torch.float32, torch.bfloat16
    def t(*s, dtype=f32):
        return torch.zeros(s, dtype=dtype, device=DEV)
    x, A, Bm, ids = t(2, 3, 8), t(8, 4), t(2, 3, 2, 4), t(2, 3, dtype=torch.int32)
    bad = [
        lambda: crf.lccrf_embed(t(4, 8), ids.long()),
        lambda: crf.lccrf_embed(t(4, 8, dtype=torch.float16), ids),
        lambda: crf.lccrf_embed(t(8, 4).t(), ids),
        lambda: crf.lccrf_embed(t(4, 8), ids, out=t(2, 3, 7)),
        lambda: crf.lccrf_embed_grad(x, ids[:1], 4),
        lambda: crf.lccrf_embed_grad(x, ids, 0),
        lambda: crf.lccrf_conv(x, t(8, 1)),
        lambda: crf.lccrf_conv(x, t(8, 9)),
        lambda: crf.lccrf_conv(x, t(8, 4, dtype=bf16)),
        lambda: crf.lccrf_conv(x, t(7, 4)),
        lambda: crf.lccrf_conv(x, t(8, 4), t(7)),
        lambda: crf.lccrf_conv(x, t(8, 4), state=t(2, 3, 8, dtype=bf16)),
        lambda: crf.lccrf_conv(x, t(8, 4), lengths=t(3, dtype=torch.int32)),
        lambda: crf.lccrf_conv(x.transpose(1, 2).contiguous().transpose(1, 2), t(8, 4)),
        lambda: crf.lccrf_conv_grad(t(2, 3, 7), x, t(8, 4)),
        lambda: crf.lccrf_conv_grad(x, x, t(8, 4), workspace=t(8)),
        lambda: crf.lccrf_conv_step(x, t(8, 4), None, t(2, 3, 8)),
        lambda: crf.lccrf_conv_step(x[:, 0], t(8, 4), None, t(2, 4, 8)),
        lambda: crf.lccrf_state_scan(x, x, A, t(2, 3, 3, 4), t(2, 3, 3, 4)),
        lambda: crf.lccrf_state_scan(x, x, t(8, 65), t(2, 3, 2, 65), t(2, 3, 2, 65)),
        lambda: crf.lccrf_state_scan(x, x.to(bf16), A, Bm, Bm),
        lambda: crf.lccrf_state_scan(x, x, A, Bm, t(2, 3, 2, 5)),
        lambda: crf.lccrf_state_scan(x, x, A, Bm, Bm, t(7)),
        lambda: crf.lccrf_state_scan(x, x, A, Bm, Bm, state=t(2, 8, 4, dtype=bf16)),
        lambda: crf.lccrf_state_scan(x, x, A, Bm, Bm, saved=t(5, dtype=torch.uint8)),
        lambda: crf.lccrf_state_scan_grad(t(2, 3, 7), x, x, A, Bm, Bm),
        lambda: crf.lccrf_state_step(x, x, A, Bm, Bm, None, None, None, t(2, 8, 4)),
        lambda: crf.lccrf_state_step(x[:, 0], x[:, 0], A, Bm[:, 0], Bm[:, 0], None, None, None, t(2, 8, 5)),
        lambda: crf.lccrf_state_step(x[:, 0], x[:, 0], A, Bm[:, 0], Bm[:, 0], None, None, None, None),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    same = t(2, 3, 8)
    with pytest.raises(crf.LccrfError):
        crf.lccrf_conv(x, t(8, 4), state=same, final=same)
    with pytest.raises(crf.LccrfError):
        crf.lccrf_state_scan(x, x, A, Bm, Bm, workspace=t(16, dtype=torch.uint8))


@pytest.mark.parametrize("names", (("x",), ("dt",), ("A",), ("Bm", "Cm"), ("z",), ("D", "dt_bias"), ("state",)))
def test_scan_gradient_by_differences(crf, names):
    """The gradient along a random direction against the change of the loss, both sides in 64 bits but for the gradient itself."""
    g = generator(31)
    B, N, D, S, G = 2, 30, 20, 8, 2
    inputs = scan_inputs(g, torch.float32, B, N, D, S, G)
    state, dout = normal(g, B, D, S), normal(g, B, N, D)
    lens = torch.tensor([30, 17], dtype=torch.int32, device=DEV)
    got = crf.lccrf_state_scan_grad(dout, *inputs.values(), lens, state=state)
    of = {"x": got.dx, "dt": got.ddt, "A": got.dA, "Bm": got.dBm, "Cm": got.dCm, "z": got.dz, "D": got.dD, "dt_bias": got.ddt_bias, "state": got.dstate}
    exact = {k: ref.f64(v) for k, v in inputs.items()} | {"lengths": lens, "state": ref.f64(state)}
    eps, d64 = 1e-6, ref.f64(dout)
    direction = {k: torch.randn(exact[k].shape, generator=torch.Generator().manual_seed(9), dtype=torch.float64) for k in names}
    def loss(sign):
        moved = {k: v + sign * eps * direction[k] if k in direction else v for k, v in exact.items()}
        return float((ref.scan(*moved.values())["out"] * d64).sum())
    want = (loss(1) - loss(-1)) / (2 * eps)
    formula = sum(float((of[k].double().cpu() * direction[k]).sum()) for k in names)
    size = sum(float((of[k].double().cpu() * direction[k]).abs().sum()) for k in names)
    assert abs(want - formula) <= scan_roundings(N, S, D, inputs["z"]) * U * size + 1e-6 * size
