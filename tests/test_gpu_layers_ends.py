"""The layers of include/lccrf_layers.h where memory ends and elsewhere: results between other memory, rows anywhere, offsets past 32 bits, streams, graphs."""
import math

import pytest
import torch

import layers_reference as ref
from test_gpu_layers import DEV, TYPES, check, clean, crf, generator, normal, recur_case, strided, top_of, U  # noqa: F401  (crf: fixture)

pytestmark = pytest.mark.gpu


class Between:
    """Memory filled with NaN, results laid into it from odd places on."""

    def __init__(self):
        self.all = []

    def __call__(self, *shape, dtype, offset=3):
        n = math.prod(shape)
        memory = torch.full((n + 64,), float("nan"), dtype=dtype, device=DEV)
        self.all.append((memory, offset, n))
        return memory[offset:offset + n].view(*shape)

    def untouched(self):
        for memory, offset, n in self.all:
            assert bool(memory[:offset].isnan().all()) and bool(memory[offset + n:].isnan().all()), "written outside"
            assert not bool(memory[offset:offset + n].isnan().any()), "not all written"


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,N,D", [(2, 9, 7), (3, 130, 33), (2, 2100, 131), (300, 5, 127), (1, 1, 1)])
def test_recurrence_between(crf, t, B, N, D):
    between = Between()
    c, lengths, state, dout = recur_case(1, B, N, D, t, "ragged" if B > 1 else "whole")
    out, final = between(B, N, D, dtype=t), between(B, D, dtype=torch.float32, offset=1)
    crf.lccrf_recurrence(**c, lengths=lengths, state=state, out=out, final=final)
    between.untouched()
    want = ref.recurrence(**clean(c), lengths=lengths, state=state)
    check(out, want["out"], "out")
    check(final, want["final"], "final")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("alone", (False, True))
@pytest.mark.parametrize("B,N,D,G", [(2, 9, 15, 3), (3, 130, 66, 2), (2, 2100, 131, 1), (40, 300, 260, 4), (2, 3, 9000, 2)])
def test_group_norm_between(crf, t, alone, B, N, D, G):
    between = Between()
    g = generator(2)
    x, lengths = strided(g, B, N, D, dtype=t), torch.randint(0, N + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    out, stats = between(B, N, D, dtype=t), between(*((B, N) if alone else (B,)), G, 2, dtype=torch.float32)
    crf.lccrf_group_norm(x, None, None, lengths, groups=G, per_position=alone, out=out, stats=stats)
    between.untouched()
    want = ref.group_norm(x, None, None, lengths, G, 1e-5, True, alone)
    check(out, want["out"], "out")
    check(stats, want["stats"], "stats")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,V,K", [(5, 3, 2), (9, 130, 9), (4, 1003, 70), (3, 5001, 16), (2, 40007, 3), (2, 140003, 3)])
def test_distill_between(crf, t, n, V, K):
    between = Between()
    g = generator(3)
    logits = normal(g, n, V, dtype=t)
    ids, teacher = top_of(g, logits, K, "any")
    ids[0, 0] = V - 1
    dloss = normal(g, n)
    want = ref.distill(logits, ids, teacher, 1.0, dloss)
    for lse in (None, crf.lccrf_distill(logits, ids, teacher)[1]):
        out, loss = between(n, V, dtype=t), between(n, dtype=torch.float32)
        crf.lccrf_distill_grad(dloss, logits, ids, teacher, lse=lse, out=out, loss=loss)
        between.untouched()
        if lse is None:
            check(out, want["dlogits"], "dlogits")


def test_rows_anywhere(crf):
    """Rows repeated (stride 0) and rows so far apart that 32-bit offsets do not reach from one to the next."""
    B, N, D, t = 3, 90, 70, torch.float32
    g = generator(4)
    c, _, state, dout = recur_case(5, B, N, D, t)
    c["x"], c["z"], dout = normal(g, B, 1, D).expand(B, N, D), normal(g, 1, N, D).expand(B, N, D), normal(g, 1, 1, D).expand(B, N, D)
    want = ref.recurrence(**c, state=state, dout=dout)
    check(crf.lccrf_recurrence(**c, state=state)[0], want["out"], "out")
    for name, got in crf.lccrf_recurrence_grad(dout, **c, state=state)._asdict().items():
        check(got, want[name], name)
    x = normal(g, 1, 1, D).expand(B, N, D)
    assert float(crf.lccrf_group_norm(x, groups=7, silu=False).mean().abs()) < 1e-5
    # a row every 2^24 + 8 elements, a few of them
    N = 20
    memory = torch.empty(N * ((1 << 24) + 8), dtype=torch.bfloat16, device=DEV)
    far = memory.as_strided((1, N, D), (memory.numel(), (1 << 24) + 8, 1))
    far.copy_(normal(g, 1, N, D))
    c, _, _, dout = recur_case(6, 1, N, D, torch.bfloat16, carry=False)
    near = dict(c, x=far.contiguous())
    c["x"] = far
    want = ref.recurrence(**near, dout=dout)
    check(crf.lccrf_recurrence(**c)[0], want["out"], "far out")
    for name, got in crf.lccrf_recurrence_grad(dout, **c)._asdict().items():
        if got is not None:
            check(got, want[name], f"far {name}")


def test_offsets_past_32_bits(crf):
    """Results of more than 2^31 elements; the inputs are one row repeated."""
    D = 2048
    B, N = 3, (1 << 31) // (2 * D)  # the last sequence begins past 2^31 - 1 elements
    g = generator(7)
    row = {k: normal(g, 1, 1, D, dtype=torch.bfloat16) for k in ("x", "f", "g")}
    decay = torch.full((D,), -6.0, device=DEV)
    lengths = torch.tensor([5, 7, 2000], dtype=torch.int32, device=DEV)
    out, final = crf.lccrf_recurrence(*[v.expand(B, N, D) for v in row.values()], decay, lengths=lengths)
    want = ref.recurrence(*[v.expand(1, 2000, D) for v in row.values()], decay)
    check(out[2, :2000], tuple(v[0] for v in want["out"]), "the last sequence")
    assert float(out[2, 2000:2100].abs().max()) == 0.0 and float(out[0, 5:60].abs().max()) == 0.0 and float(out[2, -1].abs().max()) == 0.0
    del out
    whole = crf.lccrf_group_norm(row["x"].expand(B, N, D), lengths=lengths, groups=4, per_position=True)
    few = crf.lccrf_group_norm(row["x"].expand(1, 1, D), groups=4, per_position=True)
    assert torch.equal(whole[2, 1999], few[0, 0]) and float(whole[2, 2000:].abs().max()) == 0.0
    del whole
    n, V = 70000, 40001
    logits = normal(g, 1, V, dtype=torch.bfloat16)
    ids = torch.full((n, 2), -1, dtype=torch.int32, device=DEV)
    ids[-1] = torch.tensor([7, V - 1], device=DEV)
    dlogits = crf.lccrf_distill_grad(torch.ones(n, device=DEV), logits.expand(n, V), ids, torch.zeros(n, 2, device=DEV))
    check(dlogits[-1:], ref.distill(logits, ids[-1:], torch.zeros(1, 2), 1.0, torch.ones(1))["dlogits"], "the last position")
    assert float(dlogits[-2].abs().max()) == 0.0


def train(crf, c, lengths, state, dout, w, b, top, weights):
    """One step through all of them, as a student runs it."""
    saved = crf.recurrence_saved(c["x"])
    h, final = crf.lccrf_recurrence(**c, lengths=lengths, state=state, saved=saved)
    stats = crf.group_norm_stats(h, 4)
    y = crf.lccrf_group_norm(h, w, b, lengths, groups=4, stats=stats)
    loss = torch.empty_like(weights)
    dy = crf.lccrf_distill_grad(weights, y, *top, temperature=2.0, loss=loss)
    n = crf.lccrf_group_norm_grad(dy + dout, h, w, b, lengths, groups=4, stats=stats)
    return [h, final, y, loss, *n, *crf.lccrf_recurrence_grad(n.dx, **c, lengths=lengths, state=state, saved=saved)]


@pytest.mark.parametrize("B,N,D", [(3, 50, 64), (40, 300, 256), (2, 1500, 68)])
def test_captured_and_replayed(crf, B, N, D):
    """A training step in a graph, replayed with eager work between, gives what the eager step gives; on two streams at once it does, too."""
    t = torch.bfloat16
    c, lengths, state, dout = recur_case(8, B, N, D, t, "ragged")
    c, dout = {k: None if v is None else v.to(t) if v.dim() == 3 else v for k, v in clean(c).items()}, torch.nan_to_num(dout)
    g = generator(9)
    w, b = 1 + normal(g, D, scale=0.1), normal(g, D)
    ids, teacher = top_of(g, normal(g, B, N, D), 5, "any")
    args = (c, lengths, state, dout, w, b, (ids, teacher), torch.full((B, N), 1.0 / N, device=DEV))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        train(crf, *args)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = train(crf, *args)
    for k in range(3):
        c["x"].copy_(normal(g, B, N, D, dtype=t))
        c["f"].copy_(normal(g, B, N, D, dtype=t))
        teacher.copy_(normal(g, *teacher.shape))
        eager = train(crf, *args)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(captured, eager):
            assert torch.equal(got, want), k
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = train(crf, *args)
    second = train(crf, *args)
    torch.cuda.synchronize()
    for one, two, want in zip(first, second, eager):
        assert torch.equal(one, want) and torch.equal(two, want)
