"""The encoder and the chain as one model (paper_2308_03291_amd/tagger.py): its gradients against automatic differentiation of
the same formulas in 64 bits, its training, its single tokens."""
import math

import pytest
import torch

import encoder_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tagger_module():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2308_03291_amd import binding, tagger
    binding.load_library()
    return tagger


def loss64(p, ids, tags, lengths, E, D, S, G):
    """The loss from the formulas, differentiable, in 64 bits on the CPU."""
    total = 0.0
    B = ids.shape[0]
    for b in range(B):
        n = int(lengths[b])
        keep = ids[b, :n] >= 0
        e = p["table"][ids[b, :n].clamp_min(0)] * math.sqrt(E) * keep[:, None]
        xz = e @ p["w_in"]
        K = p["conv_w"].shape[1]
        rows = torch.cat([torch.zeros(K - 1, D, dtype=torch.float64), xz[:, :D]])
        u = ref.silu(sum(rows[k:k + n] * p["conv_w"][:, k] for k in range(K)) + p["conv_b"])
        proj = u @ p["w_x"]
        step = torch.nn.functional.softplus(proj[:, :D] + p["dt_bias"])
        Bm, Cm = (v.view(n, G, S).repeat_interleave(D // G, 1) for v in proj[:, D:].split(G * S, 1))
        h, y = torch.zeros(D, S, dtype=torch.float64), []
        for l in range(n):
            h = torch.exp(-step[l, :, None] * torch.exp(p["A_log"])) * h + (step[l] * u[l])[:, None] * Bm[l]
            y.append((h * Cm[l]).sum(1) + p["skip"] * u[l])
        emit = (torch.stack(y) * ref.silu(xz[:, D:])) @ p["w_out"]
        alpha, score, last = p["trans"][0] + emit[0], 0.0, 0
        for l in range(n):
            if l:
                alpha = torch.logsumexp(alpha[:, None] + p["trans"], 0) + emit[l]
            score = score + emit[l, tags[b, l]] + p["trans"][last, tags[b, l]]
            last = int(tags[b, l])
        total = total + torch.logsumexp(alpha, 0) - score
    return total / B


def test_gradients_of_the_whole_model(tagger_module):
    V, T, E, D, S, G = 23, 5, 12, 20, 6, 2
    t = tagger_module.Tagger(V, T, E, D, S, G, seed=3)
    ids, tags, lengths = tagger_module.language(4, 17, V, T, seed=4)
    loss, grads = t.loss_and_gradients(ids, tags, lengths)
    p = {k: v.double().cpu().requires_grad_(True) for k, v in t.params.items()}
    want = loss64(p, ids.cpu().long(), tags.cpu().long(), lengths.cpu(), E, D, S, G)
    assert abs(float(loss) - float(want.detach())) <= 1e-5 * abs(float(want.detach()))
    for (k, v), g in zip(p.items(), torch.autograd.grad(want, list(p.values()))):
        off, size = (grads[k].double().cpu() - g).abs().max(), g.abs().max()
        assert off <= 2e-4 * size, f"{k}: off by {float(off):.2e} of {float(size):.2e}"


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_training_decoding_and_streams(tagger_module, dtype):
    V, T, N = 50, 4, 40
    t = tagger_module.Tagger(V, T, 32, 64, 8, dtype=dtype, seed=1)
    losses = [float(t.train_step(*tagger_module.language(32, N, V, T, seed=k))) for k in range(60)]
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5])
    ids, tags, lengths = tagger_module.language(32, N, V, T, seed=999)
    got = t.decode(ids, lengths)
    assert (got[tags < 0] == -1).all() and float((got == tags)[tags >= 0].float().mean()) > 0.6
    stream, emit = t.stream(32), t.forward(ids, lengths)["emit"]
    bound = (1e-4 if dtype == torch.float32 else 0.1) * float(emit.abs().max())
    for l in range(int(lengths.min())):
        assert float((stream.feed(ids[:, l].contiguous()) - emit[:, l]).abs().max()) <= bound, l
