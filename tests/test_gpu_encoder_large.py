"""The encoder at sizes near its limits, and at those from which on it takes other kernels than test_gpu_encoder.py's cases do."""
import pytest
import torch

import encoder_reference as ref
from test_gpu_encoder import (DEV, TYPES, U, _dirty_memory, check, check_scan, conv_lengths, crf, generator, normal, scan_inputs,  # noqa: F401
                              scan_roundings)

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1024  # positions of a call


def alike(t, want, roundings):
    """One value everywhere: half a step of its type, and the roundings on the way."""
    half = torch.finfo(t.dtype).eps / 2
    worst = max(abs(float(v) - want) for v in (t.min(), t.max()))
    assert worst <= (half + roundings * U) * abs(want), f"{float(t.min())} .. {float(t.max())} for {want}"


def test_the_longest_sequence(crf):
    """One position repeated: what the operators settle at, and where they begin and end."""
    t = torch.bfloat16
    x = torch.full((1, 1, 1), 1.5, dtype=t, device=DEV).expand(1, MOST, 1)
    silu = lambda v: v * torch.sigmoid(v)  # noqa: E731
    w, pre = torch.tensor([[0.25, 0.5]], device=DEV), torch.tensor([0.75, 1.125], dtype=torch.float64)
    out, final = crf.lccrf_conv(x, w)
    alike(out[:, :1], float(silu(pre[0])), 20)
    alike(out[:, 1:], float(silu(pre[1])), 20)
    assert final.item() == 1.5
    dout = torch.full((1, 1, 1), -0.5, dtype=t, device=DEV).expand(1, MOST, 1)
    g = crf.lccrf_conv_grad(dout, x, w)
    gate = torch.sigmoid(pre)
    first, dpre = (-0.5 * gate * (1 + pre * (1 - gate))).tolist()
    alike(g.dx[:, :1], 0.5 * first + 0.25 * dpre, 30)
    alike(g.dx[:, 1:-1], 0.75 * dpre, 30)
    alike(g.dx[:, -1:], 0.5 * dpre, 30)
    alike(g.dweight, 1.5 * dpre * MOST, 2 ** 14)  # a thread adds 64 positions of 64 runs, a channel 16 x 128 workgroups of 256 threads
    del out, g


def test_the_longest_scan(crf):
    t = torch.bfloat16
    x, Bm, Cm, dout = (torch.full((1, 1, 1), v, dtype=t, device=DEV).expand(1, MOST, 1) for v in (1.5, 0.5, 2.0, -0.5))
    vectors = Bm[..., None], Cm[..., None]
    dt, A, D = torch.zeros(1, 1, 1, dtype=t, device=DEV).expand(1, MOST, 1), torch.full((1, 1), -0.5, device=DEV), torch.full((1,), 0.25, device=DEV)
    step = float(torch.log(torch.tensor(2.0, dtype=torch.float64)))
    a = 2.0 ** -0.5
    saved = crf.state_scan_saved(x, A)
    out, final = crf.lccrf_state_scan(x, dt, A, *vectors, D, saved=saved)
    h = step * 1.5 * 0.5 / (1 - a)
    alike(out[:, :1], 2.0 * step * 1.5 * 0.5 + 0.25 * 1.5, 40)
    alike(out[:, 400:], 2.0 * h + 0.25 * 1.5, 40)
    alike(final, h, 40)
    del out
    g = crf.lccrf_state_scan_grad(dout, x, dt, A, *vectors, D, saved=saved)
    dh = -0.5 * 2.0 / (1 - a)  # away from both ends
    dput, back = dh * 0.5, dh * a * h
    inner = slice(400, MOST - 400)
    alike(g.dx[:, inner], dput * step + 0.25 * -0.5, 80)
    alike(g.dx[:, -1:], -0.5 * 2.0 * 0.5 * step + 0.25 * -0.5, 80)
    alike(g.ddt[:, inner], (dput * 1.5 + back * -0.5) * 0.5, 1000)  # a difference twelve times smaller than what it is of
    alike(g.dBm[:, inner], dh * step * 1.5, 80)
    alike(g.dCm[:, inner], -0.5 * h, 80)
    alike(g.dD, -0.5 * 1.5 * MOST, 2 ** 20 + 400)  # a wave adds a segment's positions, three waves a SIMD are joined
    alike(g.dA, back * step * MOST, 2 ** 20 + 400)


def near(got, want, bound, roundings, what):
    """check() of test_gpu_encoder.py on the GPU, in pieces; want and bound: functions of a slice of the last dimension's entries."""
    half = torch.finfo(got.dtype).eps / 2
    for at in range(0, got.shape[-1], 1 << 25):
        part = slice(at, at + (1 << 25))
        w, b = want(part), bound(part)
        off = (got[..., part].double() - w).abs()
        assert bool((off <= half * w.abs() + roundings * U * b + 1e-30).all()), f"{what} from {at} on: off by {float(off.max())}"


def test_gradients_of_the_widest_rows(crf):
    """So wide that the sums over columns, a workgroup of 1024 threads for 64 of them, would take 2^32 threads."""
    g = generator(1)
    D = 2 ** 28 + 5
    x, dout, w = normal(g, 1, 2, D), normal(g, 1, 2, D), normal(g, D, 2)
    got = crf.lccrf_conv_grad(dout, x, w, torch.zeros(D, device=DEV))

    def slopes(p):
        x0, x1, w0, w1 = x[0, 0, p].double(), x[0, 1, p].double(), w[p, 0].double(), w[p, 1].double()
        pre = torch.stack([w1 * x0, w0 * x0 + w1 * x1])
        gate = torch.sigmoid(pre)
        return x0, x1, w0, w1, dout[0, :, p].double() * gate * (1 + pre * (1 - gate)), 1.1 * dout[0, :, p].double().abs()

    def of(k):  # (the gradient by what it says, the sum of absolute values)
        def values(p, absolute=False):
            x0, x1, w0, w1, d, most = slopes(p)
            if absolute:
                x0, x1, w0, w1, d = x0.abs(), x1.abs(), w0.abs(), w1.abs(), most
            return {"dx0": w1 * d[0] + w0 * d[1], "dx1": w1 * d[1], "dw0": d[1] * x0, "dw1": d[0] * x0 + d[1] * x1, "db": d[0] + d[1]}[k]
        return values, lambda p: values(p, True)

    # (K + 14) roundings times 1 + the largest input of a gate, about 6 * 6 * 2; and the sums
    for name, t in (("dx0", got.dx[0, 0]), ("dx1", got.dx[0, 1]), ("dw0", got.dweight[:, 0]), ("dw1", got.dweight[:, 1]), ("db", got.dbias)):
        near(t, *of(name), 16 * 73 + 4, name)


def test_gradient_of_the_widest_scan(crf):
    g = generator(2)
    D, S = 2 ** 22, 64
    x, dt, dout = (normal(g, 1, 1, D) for _ in range(3))
    A, Bm, Cm, state = -torch.rand(D, S, generator=g, device=DEV) - 0.1, normal(g, 1, 1, 1, S), normal(g, 1, 1, 1, S), normal(g, 1, D, S)
    got = crf.lccrf_state_scan_grad(dout, x, dt, A, Bm, Cm, state=state)
    v, d, x64 = dt[0, 0].double(), dout[0, 0].double(), x[0, 0].double()
    step = torch.logaddexp(v, torch.zeros_like(v))
    near(got.dx[0, 0], lambda p: d[p] * float((Bm.double() * Cm.double()).sum()) * step[p], lambda p: d[p].abs() * float((Bm.double() * Cm.double()).abs().sum()) * step[p], 200, "dx")
    dBm = Cm[0, 0, 0].double() * (d * step * x64).sum()
    assert bool(((got.dBm[0, 0, 0].double() - dBm).abs() <= (2 ** 16 + 200) * U * Cm[0, 0, 0].double().abs() * (d * step * x64).abs().sum()).all())
    for s in (0, 1, 31, 62, 63):
        a, h0, c, b = torch.exp(step * A[:, s].double()), state[0, :, s].double(), float(Cm[0, 0, 0, s]), float(Bm[0, 0, 0, s])
        near(got.dA[:, s], lambda p: (d * c * a * h0 * step)[p], lambda p: (d * c * a * h0 * step)[p].abs(), 200, f"dA {s}")
        near(got.dstate[0, :, s], lambda p: (d * c * a)[p], lambda p: (d * c * a)[p].abs(), 200, f"dstate {s}")
        h = a * h0 + step * x64 * b
        big = (d * a * h0).abs().sum() + (d * step * x64 * b).abs().sum()
        assert float((got.dCm[0, 0, 0, s].double() - (d * h).sum()).abs()) <= (2 ** 16 + 200) * U * float(big)


def test_sizes_past_32_bits_are_refused(crf):
    """Views can be that large without memory; a size cut to 32 bits would pass for a small one."""
    def t(*s, dtype=torch.float32):
        return torch.zeros(s, dtype=dtype, device=DEV)
    many = 2 ** 32 + 5
    ids = t(2, 3, dtype=torch.int32)
    x, v, A = t(1, 1, 1).expand(many, 1, 1), t(1, 1, 1, 1).expand(many, 1, 1, 1), -torch.ones(1, 1, device=DEV)
    wide, vectors = t(1, 1, 1).expand(1, many, 1), t(1, 1, 1, 1).expand(1, many, 1, 1)
    bad = [
        lambda: crf.lccrf_embed(t(1, 1).expand(many, 1), ids),
        lambda: crf.lccrf_embed_grad(t(2, 3, 1), ids, many),
        lambda: crf.lccrf_conv(x, t(1, 2)),
        lambda: crf.lccrf_conv(wide, t(1, 2)),
        lambda: crf.lccrf_conv_grad(x, x, t(1, 2)),
        lambda: crf.lccrf_conv_grad(wide, wide, t(1, 2)),
        lambda: crf.state_scan_saved(x, A),
        lambda: crf.lccrf_state_scan(x, x, A, v, v),
        lambda: crf.lccrf_state_scan(wide, wide, A, vectors, vectors),
        lambda: crf.lccrf_state_scan_grad(x, x, x, A, v, v),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")


# ---- kernels that only large calls take -----------------------------------------------------------------------

def ids_of(kind, n, V, g):
    if kind == "spread":
        ids = torch.randint(-5, V + 5, (n,), generator=g, device=DEV)
    elif kind == "heavy":  # as in text
        ids = (float(V) ** torch.rand(n, generator=g, device=DEV, dtype=torch.float64) - 1).long().clamp(0, V - 1)
    else:  # one token holds most positions, two others the rest: waves that keep no list of theirs, pieces without end
        ids = torch.full((n,), V // 2, device=DEV)
        ids[::97], ids[5::101] = V - 1, 0
    return ids.to(torch.int32)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kind", ("spread", "heavy", "most"))
@pytest.mark.parametrize("V,D,n", [(5000, 40, 40000), (300, 33, 40001), (70000, 5, 33000), (100000, 192, 3000), (50000, 100, 20000), (33000, 301, 16384), (4000000, 3, 2000)])
def test_embed_grad_of_many_positions(crf, t, kind, V, D, n):
    """More positions than a wave of the index reads or keeps at a time; tables written four rows a thread, past the caches and through them."""
    g = generator(V + n)
    ids, dout = ids_of(kind, n, V, g), normal(g, n, D, dtype=t)
    got = crf.lccrf_embed_grad(dout, ids, V, scale=0.75)
    most = int(torch.bincount(ids.long().clamp(0, V - 1)).max())
    # positions one by one in pieces of at most 128, those one by one; the scale
    check(got, ref.embed_grad(dout, ids, V, 0.75), ref.embed_grad(dout, ids, V, 0.75, absolute=True), min(most, 128 + most // 32) + 4, f"embed_grad {kind}")
    assert torch.equal(got, crf.lccrf_embed_grad(dout, ids, V, scale=0.75)), "not the same again"


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D", (1024, 1031, 3))
def test_embed_of_many_positions(crf, t, D):
    g = generator(D)
    n = (36 << 20) // (D * (4 if t == torch.float32 else 2))
    table, ids = normal(g, 999, D, dtype=t), torch.randint(-1, 1000, (n,), generator=g, device=DEV).to(torch.int32)
    want = ref.embed(table, ids, 1.5)
    check(crf.lccrf_embed(table, ids, scale=1.5), want, want.abs(), 1, "embed")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D,K", [(1024, 4), (1031, 3)])
def test_conv_of_many_positions(crf, t, D, K):
    """Results of more than 32 MB."""
    g = generator(D + K)
    B, N = 8, (36 << 20) // (8 * D * (4 if t == torch.float32 else 2))
    x, dout, state = normal(g, B, N, 2 * D, dtype=t)[..., :D], normal(g, B, N, D, dtype=t), normal(g, B, K - 1, D, dtype=t)
    w, bias, lens = normal(g, D, K, scale=K ** -0.5), normal(g, D, scale=0.1), conv_lengths(B, N, g)
    want, big = (ref.conv(x, w, bias, lens, state, dout, absolute=a) for a in (False, True))
    P = float(big["pre"].max())
    out, final = crf.lccrf_conv(x, w, bias, lens, state=state)
    check(out, want["out"], big["pre"], 2 * K + 10 + 2 * P, "out")
    assert torch.equal(final.double().cpu(), want["final"]), "final"
    got = crf.lccrf_conv_grad(dout, x, w, bias, lens, state=state)
    E = (K + 14) * (1 + P)
    for name, more in (("dx", K), ("dstate", K), ("dweight", B * N), ("dbias", B * N)):
        check(getattr(got, name), want[name], big[name], E + more, name)


@pytest.mark.parametrize("K", (2, 3, 5, 8))
def test_conv_in_long_runs(crf, K):
    """So many threads that a run is as long as it gets: every sequence as in a call of its own, where runs are short."""
    g = generator(K)
    t, B, N, D = torch.bfloat16, 64, 2100, 512
    x, dout, state = normal(g, B, N, D, dtype=t), normal(g, B, N, D, dtype=t), normal(g, B, K - 1, D, dtype=t)
    w, bias, lens = normal(g, D, K), normal(g, D), conv_lengths(B, N, g)
    out, final = crf.lccrf_conv(x, w, bias, lens, state=state)
    grad = crf.lccrf_conv_grad(dout, x, w, bias, lens, state=state)
    dweight, dbias = torch.zeros(D, K, dtype=torch.float64, device=DEV), torch.zeros(D, dtype=torch.float64, device=DEV)
    for b in range(B):
        at = slice(b, b + 1)
        one, last = crf.lccrf_conv(x[at], w, bias, lens[at], state=state[at])
        assert torch.equal(out[at], one) and torch.equal(final[at], last), b
        own = crf.lccrf_conv_grad(dout[at], x[at], w, bias, lens[at], state=state[at])
        assert torch.equal(grad.dx[at], own.dx) and torch.equal(grad.dstate[at], own.dstate), b
        dweight, dbias = dweight + own.dweight.double(), dbias + own.dbias.double()
    # sums of B N terms of about 1: either side's error stays below their number's root times their size
    assert float((grad.dweight.double() - dweight).abs().max()) <= B * N * U * 100 and float((grad.dbias.double() - dbias).abs().max()) <= B * N * U * 100


@pytest.mark.parametrize("S", (4, 8, 16))
@pytest.mark.parametrize("D,G", [(256, 1), (193, 1), (512, 2), (768, 3)])
def test_gradient_of_four_tiles_a_workgroup(crf, S, D, G):
    g = generator(S * D)
    inputs = scan_inputs(g, torch.float32, 3, 45, D, S, G, gate=G != 3)
    check_scan(crf, inputs, conv_lengths(3, 45, g), normal(g, 3, D, S), normal(g, 3, 45, D))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B", (65, 130, 256, 257))
@pytest.mark.parametrize("S", (4, 16, 24))
def test_scan_of_many_ragged_sequences(crf, t, B, S):
    """None is cut; up to 256 are worked on by length."""
    g = generator(B + S)
    inputs = scan_inputs(g, t, B, 40, 20, S, 1)
    check_scan(crf, inputs, conv_lengths(B, 40, g), normal(g, B, 20, S), normal(g, B, 40, 20, dtype=t))


@pytest.mark.parametrize("S", (3, 16, 24))
def test_roundings_of_wide_rows(crf, S):
    """Only the vectors' gradients add up over the channels: all other results are as near the formula as those of one channel."""
    g = generator(S)
    B, N, D = 2, 24, 2048
    inputs = scan_inputs(g, torch.float32, B, N, D, S, 1)
    state, dout = normal(g, B, D, S), normal(g, B, N, D)
    want, big = (ref.scan(*inputs.values(), None, state, dout, absolute=a) for a in (False, True))
    R = scan_roundings(N, S, 0, inputs["z"])
    out, final = crf.lccrf_state_scan(*inputs.values(), state=state)
    check(out, want["out"], big["out"], R, "out")
    check(final, want["final"], big["final"], R, "final")
    got = crf.lccrf_state_scan_grad(dout, *inputs.values(), state=state)
    for name in got._fields:
        more = 2 * D if name in ("dBm", "dCm") else B * N if name in ("dA", "dD", "ddt_bias") else 0
        check(getattr(got, name), want[name], big[name], R + more, name)
