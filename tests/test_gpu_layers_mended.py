"""Calls of the layers of include/lccrf_layers.h at the edges of what their header allows: the longest sequences, temperatures far from 1,
repeated entries over the logits themselves."""
import pytest
import torch

import layers_reference as ref
from test_gpu_layers import DEV, TYPES, U, _dirty_memory, check, crf, generator, normal  # noqa: F401

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1024  # positions of a call


# ---- group norm -----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("N", (MOST, MOST - 700))
def test_group_norm_of_the_longest_sequence(crf, N):
    """One channel, so that a workgroup's threads are 256 positions high and what they load ahead would reach past 2^31.  x is 1 and -1 in turn: the mean is 0 and
    the deviation 1 / sqrt(1 + eps), which is 1 in bfloat16."""
    x = torch.ones(1, N, 1, dtype=torch.bfloat16, device=DEV)
    x[:, 1::2] = -1.0
    stats = crf.group_norm_stats(x, 1)
    out = crf.lccrf_group_norm(x, groups=1, silu=False, stats=stats)
    assert torch.equal(out, x)
    del out
    # a thread joins 512 chunks one after another, some 60 additions and joinings besides
    off = (512 + 60) * U
    assert abs(float(stats[0, 0, 0])) <= 2 * off and abs(float(stats[0, 0, 1]) - (1 + 1e-5) ** -0.5) <= 2 * off
    w, bias = torch.full((1,), 2.0, device=DEV), torch.zeros(1, device=DEV)
    g = crf.lccrf_group_norm_grad(x, x, w, bias, groups=1, silu=False, stats=stats)
    # dx = rstd (2 x - hat mean(2 x hat)) = 2 x rstd (1 - rstd^2), 2e-5 of x; the mean of 2 is off by as many additions, rstd as above
    assert float(g.dx.abs().max()) <= 2e-5 + 8 * off
    # 8192 chunks' sums one after another
    assert abs(float(g.dweight) / N - (1 + 1e-5) ** -0.5) <= (8192 + 60) * U + 2 * off and abs(float(g.dbias)) <= (8192 + 60) * U * N


@pytest.mark.parametrize("alone", (False, True))
@pytest.mark.parametrize("N", (9, 3000))
def test_group_norm_of_equal_values_with_the_least_eps(crf, alone, N):
    """No spread and an eps of 2^-126: 0 times 2^63, and the bias."""
    bias = normal(generator(1), 8)
    out = crf.lccrf_group_norm(torch.full((2, N, 8), 3.0, device=DEV), None, bias, groups=2, eps=2.0 ** -126, silu=False, per_position=alone)
    assert torch.equal(out, bias.expand(2, N, 8))


# ---- distillation ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("V,K", [(5003, 100), (9001, 128), (20011, 200), (40009, 256)])
def test_distill_over_the_logits_with_entries_that_only_repeat(crf, t, V, K):
    """From the 65th entry on every class has been named before: the loss reads their logits, nothing else does, and other waves overwrite them."""
    g = generator(V + K)
    logits, dloss = normal(g, 40, V, dtype=t, scale=3.0), normal(g, 40)
    first = torch.stack([torch.randperm(V, generator=g, device=DEV)[:64] for _ in range(40)])
    ids = first[:, torch.arange(K, device=DEV) % 64].to(torch.int32).contiguous()
    teacher = normal(g, 40, K)
    want = ref.distill(logits, ids, teacher, 2.0, dloss)
    apart_loss, over_loss = torch.empty(40, device=DEV), torch.empty(40, device=DEV)
    apart = crf.lccrf_distill_grad(dloss, logits, ids, teacher, temperature=2.0, loss=apart_loss)
    check(apart, want["dlogits"], "dlogits")
    check(apart_loss, want["loss"], "loss")
    for _ in range(3):
        over = logits.clone()
        assert torch.equal(crf.lccrf_distill_grad(dloss, over, ids, teacher, temperature=2.0, loss=over_loss, out=over), apart)
        assert torch.equal(over_loss, apart_loss)


@pytest.mark.parametrize("t", (2.0 ** -120, 1e-30, 1e-10, 3e-3, 1e4, 2.0 ** 60))
@pytest.mark.parametrize("V,K", [(37, 9), (3001, 70), (9001, 64), (200003, 20)])
def test_distill_at_temperatures_far_from_one(crf, t, V, K):
    """Losses of the size of t differences of logits, and of t^2."""
    g = generator(V)
    logits, dloss = normal(g, 7, V, scale=2.0), normal(g, 7)
    teacher, ids = torch.topk(logits + normal(g, 7, V), K, -1)
    ids = ids.to(torch.int32)
    t = float(torch.tensor(t))
    want, given = (ref.distill(logits, ids, teacher, t, dloss, from_lse=k) for k in (False, True))
    loss, lse = crf.lccrf_distill(logits, ids, teacher, temperature=t)
    check(loss, want["loss"], "loss")
    check(lse, want["lse"], "lse")
    assert t > 1 or float(want["loss"][0].abs().max()) > 0.1 * t
    check(crf.lccrf_distill_grad(dloss, logits, ids, teacher, temperature=t, loss=loss), want["dlogits"], "dlogits")
    check(loss, want["loss"], "loss with the gradient")
    if t > 1e-3:
        check(crf.lccrf_distill_grad(dloss, logits, ids, teacher, temperature=t, lse=lse), given["dlogits"], "dlogits of lse")


@pytest.mark.parametrize("t", (2.0 ** -126, 1e30, 3e38))
@pytest.mark.parametrize("V,K", [(9, 9), (3001, 70), (30000, 5)])
def test_distill_at_the_ends_of_the_temperatures(crf, t, V, K):
    """Gradients of t (p - q) where t^2 or 1 / t is no normal float; the loss there is 0, or past every float, and no NaN."""
    g = generator(V)
    logits, dloss = normal(g, 5, V, scale=2.0), normal(g, 5, scale=1e-2)
    teacher, ids = torch.topk(logits + normal(g, 5, V), K, -1)
    ids, loss = ids.to(torch.int32), torch.empty(5, device=DEV)
    t = float(torch.tensor(t))
    check(crf.lccrf_distill_grad(dloss, logits, ids, teacher, temperature=t, loss=loss), ref.distill(logits, ids, teacher, t, dloss)["dlogits"], "dlogits")
    assert not bool(loss.isnan().any()) and (t < 1 or K == V or bool(torch.isposinf(loss).all())) and (t > 1 or bool((loss.abs() < 1e-36).all()))


@pytest.mark.parametrize("V", (40, 3001, 30000))
def test_distill_of_a_named_class_at_the_lowest_logit(crf, V):
    """t^2 times its distance by t passes no float where the distance divided by t does."""
    g = generator(V)
    logits = normal(g, 6, V)
    logits[:, 3] = torch.finfo(torch.float32).min
    ids = torch.tensor([[3, 7, 11, 20]], dtype=torch.int32, device=DEV).repeat(6, 1)
    teacher = normal(g, 6, 4)
    want = ref.distill(logits, ids, teacher, 0.25, torch.ones(6))
    assert 1e30 < float(want["loss"][0].min()) < float(want["loss"][0].max()) < 1e38
    loss = torch.empty(6, device=DEV)
    crf.lccrf_distill_grad(torch.ones(6, device=DEV), logits, ids, teacher, temperature=0.25, loss=loss)
    check(loss, want["loss"], "loss with the gradient")
    check(crf.lccrf_distill(logits, ids, teacher, temperature=0.25)[0], want["loss"], "loss")
