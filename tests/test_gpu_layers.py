"""The layers of include/lccrf_layers.h on the GPU against their formulas in 64 bits (tests/layers_reference.py, which also says how far
float arithmetic may be from them); a result is off by half a step of its own type more."""
import math

import pytest
import torch

import layers_reference as ref

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
    from paper_2308_03291_amd import encoder, layers
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
            t.view(torch.uint8).fill_(0xFF) if t.numel() else None
            return t

    monkeypatch.setattr(encoder, "torch", Dirty())
    monkeypatch.setattr(layers, "torch", Dirty())
    yield


def generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def strided(g, *shape, dtype):
    """Dense rows inside wider ones, from an odd element on."""
    wide = normal(g, *shape[:-1], 2 * shape[-1] + 3, dtype=dtype)
    return wide[..., 1:1 + shape[-1]]


def check(got, pair, what):
    want, error = pair
    half = torch.finfo(got.dtype).eps / 2
    got = got.detach().double().cpu()
    assert got.shape == want.shape, f"{what}: {tuple(got.shape)} for {tuple(want.shape)}"
    tol = half * want.abs() + U * error * (1 + half) + 1e-37
    off = (got - want).abs()
    bad = ~(off <= tol)
    if bad.any():
        worst = torch.where(torch.isnan(off), math.inf, off - tol).flatten().argmax()
        raise AssertionError(f"{what}: {float(got.flatten()[worst])} for {float(want.flatten()[worst])} (allowed {float(tol.flatten()[worst])}) at {int(worst)}, {int(bad.sum())} of {bad.numel()}")


def ragged(g, B, N, kind):
    """Lengths: none, from nothing to all, or out of range."""
    if kind == "whole":
        return None
    lengths = torch.randint(0, N + 1, (B,), generator=g, device=DEV)
    if kind == "ends":
        lengths = torch.tensor([(-3, 0, 1, N - 1, N, N + 9)[i % 6] for i in range(B)], device=DEV)
    return lengths.to(torch.int32)


def poison(t, lengths):
    """NaN at and past the lengths: never read."""
    if lengths is None or t is None:
        return t
    past = torch.arange(t.shape[1], device=DEV)[None] >= lengths[:, None]
    t[past] = float("nan")
    return t


# ---- gated linear recurrence ----------------------------------------------------------------------------------

def recur_case(seed, B, N, D, t, kind="whole", gate=True, bias=True, carry=True, rows=normal):
    g = generator(seed)
    lengths = ragged(g, B, N, kind)
    c = {k: poison(rows(g, B, N, D, dtype=t), lengths) for k in ("x", "f", "g")}
    c["decay"] = normal(g, D, scale=1.5) - 3.0
    c["z"] = poison(rows(g, B, N, D, dtype=t), lengths) if gate else None
    c["f_bias"], c["g_bias"] = (normal(g, D), normal(g, D)) if bias else (None, None)
    state = normal(g, B, D) if carry else None
    return c, lengths, state, poison(rows(g, B, N, D, dtype=t), lengths)


def clean(c):
    return {k: None if v is None else torch.nan_to_num(v.float(), nan=0.0) if v.dim() == 3 else v for k, v in c.items()}


def check_recurrence(crf, c, lengths, state, dout, rate, what):
    want = ref.recurrence(**clean(c), lengths=lengths, rate=rate, state=state, dout=torch.nan_to_num(dout.float(), nan=0.0))
    out, final = crf.lccrf_recurrence(**c, lengths=lengths, rate=rate, state=state)
    check(out, want["out"], f"{what}: out")
    check(final, want["final"], f"{what}: final")
    saved = crf.recurrence_saved(c["x"])
    again, final = crf.lccrf_recurrence(**c, lengths=lengths, rate=rate, state=state, saved=saved)
    assert torch.equal(out, again)
    grads = crf.lccrf_recurrence_grad(dout, **c, lengths=lengths, rate=rate, state=state, saved=saved)
    for name, got in grads._asdict().items():
        if got is None:
            assert name not in want or name in ("df_bias", "dg_bias")
        else:
            check(got, want[name], f"{what}: {name}")
    for got, same in zip(grads, crf.lccrf_recurrence_grad(dout, **c, lengths=lengths, rate=rate, state=state)):
        assert got is None or torch.equal(got, same), f"{what}: not the same without saved"


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kind", ("whole", "ragged", "ends"))
@pytest.mark.parametrize("B,N,D", [(1, 1, 1), (2, 3, 1), (3, 8, 2), (2, 9, 3), (5, 31, 5), (2, 33, 64), (6, 64, 127), (3, 65, 129), (2, 200, 130), (7, 100, 33), (150, 20, 6)])
def test_recurrence(crf, t, kind, B, N, D):
    for rows in (normal, strided):
        check_recurrence(crf, *recur_case(B * 100 + N, B, N, D, t, kind, rows=rows), 8.0, f"{rows.__name__} {kind}")


@pytest.mark.parametrize("gate,bias,carry", [(g, b, c) for g in (0, 1) for b in (0, 1) for c in (0, 1)])
def test_recurrence_without(crf, gate, bias, carry):
    check_recurrence(crf, *recur_case(5, 4, 70, 38, torch.float32, "ragged", gate, bias, carry), 3.0, "parts")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,N,D", [(1, 3000, 7), (2, 1500, 130), (3, 700, 64)])
def test_recurrence_in_segments(crf, t, B, N, D):
    """Long sequences in a small batch: their segments run side by side."""
    check_recurrence(crf, *recur_case(N, B, N, D, t, "ends" if B > 1 else "whole"), 8.0, "segments")
    c, lengths, state, dout = recur_case(N + 1, B, N, D, t, "ragged")
    check_recurrence(crf, c, lengths, state, dout, 0.3, "segments, slow decays")


def test_recurrence_goes_on_where_it_stopped(crf):
    """A prompt in pieces and single tokens give what one pass gives; final may be state."""
    B, N, D = 3, 90, 77
    c, _, state, _ = recur_case(11, B, N, D, torch.float32)
    want = ref.recurrence(**c, state=state)
    carry, outs = state.clone(), []
    for l0, l1 in ((0, 1), (1, 40), (40, 80)):
        piece = {k: v[:, l0:l1] if v is not None and v.dim() == 3 else v for k, v in c.items()}
        out, back = crf.lccrf_recurrence(**piece, state=carry, final=carry)
        assert back.data_ptr() == carry.data_ptr()
        outs.append(out)
    for l in range(80, N):
        outs.append(crf.lccrf_recurrence_step(*[c[k][:, l] if c[k].dim() == 3 else c[k] for k in ("x", "f", "g", "decay", "z", "f_bias", "g_bias")], carry)[:, None])
    check(torch.cat(outs, 1), want["out"], "out")
    check(carry, want["final"], "state")


@pytest.mark.parametrize("final_is_state", (False, True))
def test_recurrence_over_its_own_state(crf, final_is_state):
    """Segments and an odd width: what is read of the state before others write it."""
    B, N, D = 2, 2100, 259
    c, lengths, state, _ = recur_case(12, B, N, D, torch.bfloat16, "ragged")
    want = ref.recurrence(**clean(c), lengths=lengths, state=state)
    carry = state.clone()
    out, final = crf.lccrf_recurrence(**c, lengths=lengths, state=carry, final=carry if final_is_state else None)
    check(out, want["out"], "out")
    check(final, want["final"], "final")


@pytest.mark.parametrize("B,N,D", [(5, 9000, 40), (1, 20000, 130), (9, 700, 257), (3, 4000, 1)])
def test_recurrence_in_place_and_apart(crf, B, N, D):
    """The final state written over the call's by whichever segment ends a sequence: the same bits as into memory of its own."""
    c, lengths, state, _ = recur_case(13, B, N, D, torch.float32, "ragged")
    lengths[0] = 70  # (its last segment is among the first)
    apart = crf.lccrf_recurrence(**c, lengths=lengths, state=state)
    for _ in range(3):
        carry = state.clone()
        out, final = crf.lccrf_recurrence(**c, lengths=lengths, state=carry, final=carry)
        assert torch.equal(out, apart[0]) and torch.equal(final, apart[1])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,D", [(1, 1), (3, 5), (64, 256), (5, 1023), (700, 12)])
def test_recurrence_step(crf, t, B, D):
    for gate, bias in ((True, True), (False, False)):
        for rows in (normal, strided):
            c, _, state, _ = recur_case(B + D, B, 1, D, t, gate=gate, bias=bias, rows=rows)
            want = ref.recurrence(**c, rate=5.0, state=state)
            moved = state.clone()
            out = crf.lccrf_recurrence_step(*[v if v is None or v.dim() == 1 else v[:, 0] for v in c.values()], moved, rate=5.0)
            check(out[:, None], want["out"], "out")
            check(moved, want["final"], "state")


@pytest.mark.parametrize("N", (40, 3000))
def test_recurrence_of_closed_and_open_gates(crf, N):
    """Decays of exactly 1 (nothing is taken up, the gradient's 1 / sqrt(1 - a^2) has no value) and of almost 0, slow and fast channels."""
    B, D = 2, 12
    c, _, state, dout = recur_case(13, B, N, D, torch.float32, bias=False)
    c["f"][:, :, :3], c["f"][:, :, 3:6], c["f"][:, ::2, 6:9] = -200.0, 90.0, -30.0
    c["decay"][:] = torch.tensor([-40.0, -90.0, 0.0, 2.0, -100.0, 3.0, -16.5, -17.5, -1.0, -20.0, 6.0, -8.0], device=DEV)
    want = ref.recurrence(**c, state=state, dout=dout)
    out, final = crf.lccrf_recurrence(**c, state=state)
    check(out, want["out"], "out")
    check(final, want["final"], "final")
    for name, got in crf.lccrf_recurrence_grad(dout, **c, state=state)._asdict().items():
        if got is not None:
            assert not torch.isnan(got).any(), name
            value, error = want[name]
            check(got, (value, torch.nan_to_num(error, nan=0.0)), name)


@pytest.mark.parametrize("N", (30, 200, 3000))
def test_recurrence_keeps_infinities_and_nan_where_they_are(crf, N):
    """An infinite input makes its channel infinite from there on, over blocks and segments whose decays together are below every float; a NaN
    too; other channels and earlier positions see nothing of it."""
    B, D = 2, 10
    c, _, _, _ = recur_case(14, B, N, D, torch.float32, bias=False, carry=False, gate=False)
    c["decay"][:] = 1.0  # decays around exp(-5) a position
    c["x"][0, 5, 3], c["x"][1, N - 9, 4] = float("inf"), float("nan")
    out, final = crf.lccrf_recurrence(**c)
    spoiled = {k: v.clone() if v is not None else None for k, v in c.items()}
    spoiled["x"][0, 5, 3], spoiled["x"][1, N - 9, 4] = 0.0, 0.0
    want = ref.recurrence(**spoiled)
    assert bool(torch.isposinf(out[0, 5:, 3]).all()) and bool(torch.isposinf(final[0, 3]))
    assert bool(torch.isnan(out[1, N - 9:, 4]).all()) and bool(torch.isnan(final[1, 4]))
    out[0, 5:, 3], out[1, N - 9:, 4] = want["out"][0][0, 5:, 3].float().to(DEV), want["out"][0][1, N - 9:, 4].float().to(DEV)
    check(out, want["out"], "the others")


# ---- group norm -----------------------------------------------------------------------------------------------

def check_norm(crf, g, B, N, D, G, t, kind, alone, silu, affine, rows, what, shift=0.5, eps=1e-5):
    lengths = ragged(g, B, N, kind)
    x = poison(rows(g, B, N, D, dtype=t).mul_(2).add_(shift), lengths)
    dout = poison(rows(g, B, N, D, dtype=t), lengths)
    weight, bias = (1 + normal(g, D, scale=0.3), normal(g, D, scale=0.3)) if affine else (None, None)
    how = {"groups": G, "eps": eps, "silu": silu, "per_position": alone}
    want = ref.group_norm(torch.nan_to_num(x.float(), nan=0.0), weight, bias, lengths, G, eps, silu, alone, torch.nan_to_num(dout.float(), nan=0.0))
    stats = crf.group_norm_stats(x, G, per_position=alone)
    out = crf.lccrf_group_norm(x, weight, bias, lengths, **how, stats=stats)
    check(out, want["out"], f"{what}: out")
    check(stats, want["stats"], f"{what}: stats")
    assert torch.equal(out, crf.lccrf_group_norm(x, weight, bias, lengths, **how))
    grads = crf.lccrf_group_norm_grad(dout, x, weight, bias, lengths, **how, stats=stats)
    for name, got in grads._asdict().items():
        assert (got is None) == (not affine and name != "dx")
        if got is not None:
            check(got, want[name], f"{what}: {name}")
    for got, same in zip(grads, crf.lccrf_group_norm_grad(dout, x, weight, bias, lengths, **how)):
        assert got is None or torch.equal(got, same), f"{what}: not the same without stats"


NORMS = [(1, 1, 1, 1), (2, 3, 4, 4), (2, 5, 6, 2), (3, 7, 15, 3), (2, 40, 64, 1), (4, 33, 96, 32), (2, 65, 301, 7), (1, 300, 130, 1), (3, 20, 1024, 8), (2, 9, 1001, 7), (2, 6, 2048, 1),
         (70, 4, 24, 6), (2, 5, 4100, 1), (1, 3, 9000, 2), (2, 50, 520, 65)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("alone", (False, True))
@pytest.mark.parametrize("B,N,D,G", NORMS)
def test_group_norm(crf, t, alone, B, N, D, G):
    g = generator(B * 31 + N * 7 + D)
    for kind, rows, silu, affine in (("whole", normal, True, True), ("ragged", strided, True, True), ("ends", normal, False, True), ("ragged", normal, True, False)):
        check_norm(crf, g, B, N, D, G, t, kind, alone, silu, affine, rows, f"{kind} {rows.__name__} silu={silu}")


@pytest.mark.parametrize("alone", (False, True))
def test_group_norm_far_from_zero(crf, alone):
    """A mean a thousand times the deviation: no difference of large squares."""
    check_norm(crf, generator(3), 3, 50, 96, 3, torch.float32, "ragged", alone, True, True, normal, "far", shift=3000.0)
    check_norm(crf, generator(4), 2, 700, 40, 2, torch.float32, "ragged", alone, False, True, normal, "long", shift=-500.0, eps=1e-2)


def test_group_norm_long(crf):
    check_norm(crf, generator(5), 1, 9001, 24, 2, torch.bfloat16, "whole", False, True, True, normal, "long")
    check_norm(crf, generator(6), 2, 5000, 33, 3, torch.float32, "ragged", False, True, True, strided, "long")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,N,D,G", [(70, 130, 520, 65), (46, 201, 1001, 7), (1100, 9, 1000, 25), (9, 1023, 1024, 16)])
def test_group_norm_of_many_sequences(crf, t, B, N, D, G):
    """What caches do not hold: eight pieces a thread, or two passes."""
    check_norm(crf, generator(7 * B + N), B, N, D, G, t, "ragged", False, True, True, normal, "many")


@pytest.mark.parametrize("alone", (False, True))
def test_group_norm_of_equal_values(crf, alone):
    """No spread: the activation of the bias, and no gradient but the bias's."""
    x, bias = torch.full((2, 9, 20), 3.0, device=DEV), normal(generator(1), 20)
    out = crf.lccrf_group_norm(x, None, bias, groups=4, per_position=alone)
    want = torch.nn.functional.silu(bias.double())
    assert float((out.double() - want).abs().max()) <= 16 * U
    g = crf.lccrf_group_norm_grad(torch.ones_like(x), x, None, bias, groups=4, per_position=alone)
    assert float(g.dx.abs().max()) < 1e5 and not torch.isnan(g.dx).any()


@pytest.mark.parametrize("alone", (False, True))
def test_group_norm_keeps_nan_in_its_group(crf, alone):
    g = generator(2)
    x = normal(g, 3, 30, 32)
    whole = crf.lccrf_group_norm(x, groups=4, per_position=alone)
    x[1, 7, 9] = float("nan")
    x[2, 4, 31] = float("inf")
    out = crf.lccrf_group_norm(x, groups=4, per_position=alone)
    spoiled = torch.zeros_like(out, dtype=torch.bool)
    if alone:
        spoiled[1, 7, 8:16] = spoiled[2, 4, 24:32] = True
    else:
        spoiled[1, :, 8:16] = spoiled[2, :, 24:32] = True
    assert bool(torch.isnan(out[spoiled]).all()) and torch.equal(out[~spoiled], whole[~spoiled])


# ---- distillation ---------------------------------------------------------------------------------------------

def top_of(g, logits, K, kind):
    """A teacher's entries: the largest of noisy logits, some of them not there, or anything."""
    lead, V = logits.shape[:-1], logits.shape[-1]
    if kind == "top":
        teacher, ids = torch.topk(logits.float() + normal(g, *lead, V), min(K, V), -1)
        if K > V:
            teacher, ids = (torch.cat([t, t[..., :1].expand(*lead, K - V)], -1) for t in (teacher, ids))
    else:
        teacher, ids = normal(g, *lead, K, scale=3.0), torch.randint(-V // 2 - 1, V + V // 2 + 1, (*lead, K), generator=g, device=DEV)
        teacher[torch.rand(*lead, K, generator=g, device=DEV) < 0.2] = -math.inf
    ids = ids.to(torch.int32).contiguous()
    ids.view(-1, K)[1::4] = -1  # positions without an entry
    return ids, teacher.contiguous()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kind", ("top", "any"))
@pytest.mark.parametrize("n,V,K", [(1, 1, 1), (5, 2, 3), (9, 7, 2), (40, 5, 8), (33, 64, 16), (10, 100, 64), (17, 128, 8), (6, 301, 65), (5, 1001, 1), (3, 2049, 256), (4, 5003, 16), (3, 20011, 100),
                                   (2, 70001, 64)])
def test_distill(crf, t, kind, n, V, K):
    g = generator(n + V + K)
    temperature = (1.0, 2.5)[V % 2]
    for rows in (normal, strided):
        logits = rows(g, n, V, dtype=t).mul_(2)
        ids, teacher = top_of(g, logits, K, kind)
        dloss = normal(g, n)
        none = ~((ids >= 0) & (ids < V) & (teacher != -math.inf)).any(-1)
        logits[none] = float("nan")  # never read
        clean = torch.nan_to_num(logits.float(), nan=0.0)
        want, given = ref.distill(clean, ids, teacher, temperature, dloss), ref.distill(clean, ids, teacher, temperature, dloss, from_lse=True)
        loss, lse = crf.lccrf_distill(logits, ids, teacher, temperature=temperature)
        check(loss, want["loss"], "loss")
        check(lse, want["lse"], "lse")
        with_loss = torch.full_like(loss, float("nan"))
        dlogits = crf.lccrf_distill_grad(dloss, logits, ids, teacher, temperature=temperature, loss=with_loss)
        check(dlogits, want["dlogits"], "dlogits")
        check(with_loss, want["loss"], "loss with the gradient")  # (summed in another order than by itself)
        check(crf.lccrf_distill_grad(dloss, logits, ids, teacher, temperature=temperature, lse=lse), given["dlogits"], "dlogits of lse")
        over = logits.clone().contiguous()
        assert torch.equal(crf.lccrf_distill_grad(dloss, over, ids, teacher, temperature=temperature, out=over), dlogits), "over the logits"
        over = logits.clone().contiguous()
        also = torch.full_like(loss, float("nan"))
        check(crf.lccrf_distill_grad(dloss, over, ids, teacher, temperature=temperature, lse=lse, loss=also, out=over), given["dlogits"], "of lse, over the logits")
        check(also, given["loss"], "loss of lse")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("V,K", [(40, 6), (64, 12), (200, 30), (500, 60), (110, 86), (1000, 200), (3000, 20)])
def test_distill_beside_a_class_named_twice(crf, t, V, K):
    """Entries that name a class twice change their own position alone, whoever shares its wave: the others keep their bits."""
    g = generator(V + K)
    logits, dloss = normal(g, 301, V, dtype=t), normal(g, 301)
    ids, teacher = top_of(g, logits, K, "top")
    before = crf.lccrf_distill_grad(dloss, logits, ids, teacher)
    twice = [7, 150, 299]  # (positions that have entries)
    assert bool((ids[twice] >= 0).all())
    moved = ids[twice, 1].long()
    ids[twice, 1] = ids[twice, 0]
    after = crf.lccrf_distill_grad(dloss, logits, ids, teacher)
    others = torch.ones(301, dtype=torch.bool, device=DEV)
    others[twice] = False
    assert torch.equal(after[others], before[others])
    for row, was in zip(twice, moved.tolist()):
        changed = (after[row] != before[row]).nonzero().flatten().tolist()
        assert sorted(changed) == sorted({int(ids[row, 0]), was}), row


@pytest.mark.parametrize("V", (40, 3001, 30000))
def test_distill_of_masked_classes(crf, V):
    """Classes masked with -inf or the type's lowest value have probability 0; where the teacher names one, the loss is infinite and the gradient
    is not."""
    g = generator(V)
    logits = normal(g, 6, V)
    logits[:, ::3] = -math.inf
    logits[:, 1::7] = torch.finfo(torch.float32).min
    logits[0, 2:] = -math.inf
    teacher, ids = torch.topk(normal(g, 6, V).where(torch.isfinite(logits) & (logits > -1e30), torch.full((), -1e9, device=DEV)), 4, -1)
    teacher[teacher < -1e8] = -math.inf
    ids = ids.to(torch.int32)
    ids[5, 0] = 3 * (V // 6)
    dloss = torch.ones(6, device=DEV)
    want = ref.distill(logits, ids, teacher, 1.0, dloss)
    loss, lse = crf.lccrf_distill(logits, ids, teacher)
    assert float(loss[5]) == math.inf
    check(loss[:5], tuple(v[:5] for v in want["loss"]), "loss")
    check(lse, want["lse"], "lse")
    dlogits = crf.lccrf_distill_grad(dloss, logits, ids, teacher)
    check(dlogits, want["dlogits"], "dlogits")


def test_distill_of_many_positions(crf):
    g = generator(8)
    logits = normal(g, 3, 30011, 9)
    ids, teacher = top_of(g, logits, 3, "any")
    dloss = normal(g, 3, 30011)
    want = ref.distill(logits, ids, teacher, 1.5, dloss)
    loss, lse = crf.lccrf_distill(logits, ids, teacher, temperature=1.5)
    check(loss, want["loss"], "loss")
    check(crf.lccrf_distill_grad(dloss, logits, ids, teacher, temperature=1.5), want["dlogits"], "dlogits")
    empty = torch.zeros(0, 4, 9, device=DEV)
    assert crf.lccrf_distill_grad(torch.zeros(0, 4, device=DEV), empty, torch.zeros(0, 4, 2, dtype=torch.int32, device=DEV), torch.zeros(0, 4, 2, device=DEV)).shape == (0, 4, 9)
