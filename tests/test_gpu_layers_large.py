"""The layers of include/lccrf_layers.h at the largest widths, batches and numbers of classes that fit the memory of one GPU."""
import math

import pytest
import torch

import layers_reference as ref
from test_gpu_layers import DEV, TYPES, U, _dirty_memory, check, check_norm, check_recurrence, crf, generator, normal, recur_case  # noqa: F401

pytestmark = pytest.mark.gpu

WIDEST = 1 << 22
MOST = 2 ** 31 - 1024  # positions of a call


def alike(t, want, roundings):
    """One value everywhere: half a step of its type, and the roundings on the way."""
    half = torch.finfo(t.dtype).eps / 2
    worst = max(abs(float(v) - want) for v in (t.min(), t.max()))
    assert worst <= (half + roundings * U) * abs(want), f"{float(t.min())} .. {float(t.max())} for {want}"


def test_recurrence_of_the_longest_sequence(crf):
    """One position repeated, a decay of a half: what the state settles at, and where it begins and ends."""
    t = torch.bfloat16
    x, gate, dout = (torch.full((1, 1, 1), v, dtype=t, device=DEV).expand(1, MOST, 1) for v in (1.5, 0.0, -0.5))
    decay, saved = torch.zeros(1, device=DEV), crf.recurrence_saved(x)
    out, final = crf.lccrf_recurrence(x, gate, gate, decay, rate=2.0, saved=saved)
    u, m = -math.log(2.0), math.sqrt(0.75)
    b = m * 0.5 * 1.5
    alike(out[:, :1], b, 40)
    alike(out[:, 60:], 2 * b, 60)
    alike(final, 2 * b, 60)
    del out, final
    g = crf.lccrf_recurrence_grad(dout, x, gate, gate, decay, rate=2.0, saved=saved)
    inner = slice(60, MOST - 60)
    dh = -0.5 / (1 - 0.5)
    alike(g.dx[:, inner], dh * m * 0.5, 80)
    alike(g.dx[:, -1:], -0.5 * m * 0.5, 80)
    alike(g.dg[:, inner], dh * m * 0.5 * 1.5 * 0.5, 100)
    parts = 0.5 * 2 * b * u, 0.5 * 1.5 * 0.25 * u / m  # of the state, of the input: their difference is a third of the larger
    dlog = dh * (parts[0] - parts[1])
    alike(g.df[:, inner], dlog * 0.5, 400)
    # a lane adds two positions of every block of eight of its segment, 2^20 positions
    alike(g.ddecay, dlog * MOST * 0.5 / math.log(2.0), 2 ** 18 + 2000)


@pytest.mark.parametrize("D", (WIDEST, WIDEST - 1))
def test_recurrence_of_the_widest_rows(crf, D):
    """Channels are independent: those of both ends and of the middle against the formula."""
    B, N, t = 2, 9, torch.bfloat16
    c, lengths, state, dout = recur_case(21, B, N, D, t, "ragged")
    saved = crf.recurrence_saved(c["x"])
    out, final = crf.lccrf_recurrence(**c, lengths=lengths, state=state, saved=saved)
    grads = crf.lccrf_recurrence_grad(dout, **c, lengths=lengths, state=state, saved=saved)._asdict()
    for part in (slice(0, 300), slice(D // 2 - 150, D // 2 + 150), slice(D - 300, D)):
        some = {k: torch.nan_to_num(v[..., part].float(), nan=0.0) for k, v in c.items()}
        want = ref.recurrence(**some, lengths=lengths, state=state[:, part], dout=torch.nan_to_num(dout[..., part].float(), nan=0.0))
        for name, got in ({"out": out, "final": final} | grads).items():
            check(got[..., part], want[name], f"{name} of channels {part}")


@pytest.mark.parametrize("B,N,D", [(200000, 1, 3), (70000, 3, 1), (30000, 9, 5)])
def test_recurrence_of_the_largest_batches(crf, B, N, D):
    check_recurrence(crf, *recur_case(B, B, N, D, torch.float32, "ends" if N > 1 else "whole"), 8.0, "batch")


@pytest.mark.parametrize("alone", (False, True))
@pytest.mark.parametrize("D,G", [(WIDEST, 1), (WIDEST, WIDEST), (WIDEST - 2, 2), (WIDEST - 1, 3)])
def test_group_norm_of_the_widest_rows(crf, alone, D, G):
    check_norm(crf, generator(G), 1, 2, D, G, torch.bfloat16, "whole", alone, True, True, normal, "wide")


@pytest.mark.parametrize("alone", (False, True))
@pytest.mark.parametrize("B,N,D,G", [(100000, 1, 6, 2), (50000, 4, 9, 3)])
def test_group_norm_of_the_largest_batches(crf, alone, B, N, D, G):
    check_norm(crf, generator(B), B, N, D, G, torch.float32, "ends" if N > 1 else "whole", alone, True, True, normal, "batch")


def test_distill_of_the_most_classes(crf):
    """Equal logits: every class has probability 2^-30."""
    V = 1 << 30
    logits = torch.zeros(2, V, dtype=torch.bfloat16, device=DEV)
    ids = torch.tensor([[0, V - 1], [V // 2 + 1, V]], dtype=torch.int32, device=DEV)  # (V: not there)
    teacher, dloss = torch.zeros(2, 2, device=DEV), torch.tensor([1.0, -2.0], device=DEV)
    loss, lse = crf.lccrf_distill(logits, ids, teacher)
    want = torch.tensor([29 * math.log(2.0), 30 * math.log(2.0)])
    assert float((loss.cpu() - want).abs().max()) <= 8 * U * 32 and float((lse.cpu() - 30 * math.log(2.0)).abs().max()) <= 8 * U * 32
    for given in (None, lse):
        over = logits.clone()
        assert crf.lccrf_distill_grad(dloss, over, ids, teacher, lse=given, out=over) is over
        named = [(0, 0), (0, V - 1), (1, V // 2 + 1)]
        for (row, v), value in zip(named, (-0.5, -0.5, 2.0)):
            assert float(over[row, v]) == value
            over[row, v] = 2.0 ** -30 * float(dloss[row])
        # exp of 30 log 2 rounded: off by 30 roundings; half a step of bfloat16
        for row, want in enumerate((2.0 ** -30, -2.0 ** -29)):
            low, high = float(over[row].min()), float(over[row].max())
            assert max(abs(low - want), abs(high - want)) <= (2.0 ** -8 + 64 * U) * abs(want)
        del over
