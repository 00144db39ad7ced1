"""The layers of include/lccrf_layers.h in the variants that ordinary large calls take, at the least sizes that take them: tiles of a recurrence that fill the chip,
over several blocks; groups of positions of every number of pieces a lane; rows of classes held by every number of pieces a thread."""
import pytest
import torch

import layers_reference as ref
from test_gpu_layers import (DEV, TYPES, _dirty_memory, check, check_norm, check_recurrence, crf, generator, normal, ragged, recur_case, strided,  # noqa: F401
                             top_of)

pytestmark = pytest.mark.gpu


# ---- gated linear recurrence: wide tiles in one segment --------------------------------------------------------
# Forwards from 256 tiles of 128 channels on, blocks of 32 positions; backwards from 768, blocks of eight.

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kind", ("whole", "ragged", "ends"))
@pytest.mark.parametrize("B,N,D,gate", [(260, 100, 130, True), (256, 33, 128, False)])
def test_recurrence_of_many_sequences(crf, t, kind, B, N, D, gate):
    c, lengths, state, dout = recur_case(B + N, B, N, D, t, kind, gate=gate)
    check_recurrence(crf, c, lengths, state, dout, 8.0, kind)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kind", ("whole", "ragged", "ends"))
@pytest.mark.parametrize("B,N,D,gate", [(400, 70, 130, True), (260, 75, 259, False), (384, 41, 256, True)])
def test_recurrence_of_many_sequences_both_ways(crf, t, kind, B, N, D, gate):
    c, lengths, state, dout = recur_case(B + N, B, N, D, t, kind, gate=gate, rows=strided if kind == "ragged" else normal)
    check_recurrence(crf, c, lengths, state, dout, 8.0, kind)


# ---- group norm, every position by itself ----------------------------------------------------------------------

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D,G", [
    (600, 1), (768, 1), (1000, 1), (1024, 1), (2000, 2),   # two pieces a lane of bfloat16, three and four of float
    (1536, 1), (2500, 1), (4000, 1), (4096, 1),            # whole workgroups: up to four pieces of float
    (6000, 1), (8000, 1), (8192, 1), (8200, 1), (8209, 1)  # the same of bfloat16; wider than registers
])
def test_group_norm_of_wide_positions(crf, t, D, G):
    g = generator(D + G)
    for kind, rows, silu, affine in (("ragged", normal, True, True), ("ends", strided, False, True), ("whole", normal, True, False)):
        check_norm(crf, g, 6, 7, D, G, t, kind, True, silu, affine, rows, f"{kind} {rows.__name__}")


# ---- distillation ----------------------------------------------------------------------------------------------

HELD = [(torch.bfloat16, V, K) for V, K in ((5003, 100), (12001, 65), (20011, 256), (50003, 90), (100003, 100), (102400, 3), (102408, 64), (128259, 64), (128259, 100), (131079, 70), (131080, 5))] + \
       [(torch.float32, V, K) for V, K in ((2050, 66), (6001, 100), (12001, 256), (30011, 90), (45001, 100), (51203, 9), (51204, 64), (65537, 16), (65537, 100), (65539, 65), (65540, 65))]


@pytest.mark.parametrize("t,V,K", HELD)
def test_distill_of_held_rows(crf, t, V, K):
    """Loss and gradient of a row in a workgroup's registers, apart and over the logits, and past the last size that is held."""
    g = generator(V + K)
    n, temperature = 5, 1.5
    for kind in ("top", "any"):
        logits = normal(g, n, V, dtype=t).mul_(2)
        ids, teacher = top_of(g, logits, K, kind)
        ids[0, 0], ids[2, -1], teacher[0, 0], teacher[2, -1] = V - 1, 0, 1.0, 1.0
        dloss = normal(g, n)
        want = ref.distill(logits, ids, teacher, temperature, dloss)
        loss, over_loss = torch.full((n,), float("nan"), device=DEV), torch.full((n,), float("nan"), device=DEV)
        dlogits = crf.lccrf_distill_grad(dloss, logits, ids, teacher, temperature=temperature, loss=loss)
        check(dlogits, want["dlogits"], f"{kind}: dlogits")
        check(loss, want["loss"], f"{kind}: loss")
        check(crf.lccrf_distill(logits, ids, teacher, temperature=temperature)[0], want["loss"], f"{kind}: loss by itself")
        over = logits.clone()
        assert torch.equal(crf.lccrf_distill_grad(dloss, over, ids, teacher, temperature=temperature, loss=over_loss, out=over), dlogits)
        assert torch.equal(over_loss, loss)
