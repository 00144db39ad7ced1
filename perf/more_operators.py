"""The operators of a student tagger: what is measured of them.

A gated linear recurrence with one state a channel, group norm with an activation over channels that lie last, and distillation from a
teacher's top logits; each forwards, in training, and the first two as they run for single tokens.  A case is one pass of one of them.
``op`` names it; ``B`` sequences of at most ``N`` positions (the shortest ``min_len``), ``D`` channels, ``G`` groups of them, ``V`` classes
(tags or words) of which the teacher names ``K``.  Batch sizes and lengths are those of ``paper_2308_03291_amd.workloads``, widths
and numbers of classes are generic.
"""
from __future__ import annotations

import math

import torch

DEVICE = "cuda"

#: False: ``run`` computes the plain forms below.  True: it calls the framework.
own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
RATE, EPS = 8.0, 1e-5


def _case(op, B, N, *, name=None, dtype="bf16", min_len=None, D=0, G=1, silu=True, gate=True, carry=False, V=0, K=0, temperature=1.0):
    c = {"op": op, "B": B, "N": N, "dtype": dtype, "min_len": N if min_len is None else min_len}
    if op.startswith("rec"):
        c |= {"D": D, "gate": gate, "carry": carry}
    elif op.startswith("distill"):
        c |= {"V": V, "K": K, "temperature": temperature}
    else:
        c |= {"D": D, "G": G, "silu": silu}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # One token for a few streams, the recurrence's part: latency is all there is.
        _case("rec_step", 4, 1, name="rec_step_few", dtype="f32", D=1024),
        # One token for every stream of a busy server.
        _case("rec_step", 512, 1, name="rec_step_many", D=2048),
        # Prompts of the headline batch that continue earlier ones.
        _case("rec", 64, 512, name="rec_prompt", D=2048, carry=True),
        # Very long documents in a tiny batch, an odd width, no gate.
        _case("rec", 4, 16384, name="rec_long", D=514, gate=False),
        # Training step on ragged sentences.
        _case("rec_train", 128, 256, name="rec_train", D=1024, min_len=64),
        # One token for every stream, each position normalised by itself: latency.
        _case("norm_position", 64, 1, name="norm_step", dtype="f32", D=1024, G=16),
        # Training step with every position by itself: ragged sentences, groups of an odd width, single precision.
        _case("norm_position_train", 128, 128, name="norm_position_train_odd", dtype="f32", D=1001, G=7, min_len=16),
        # Training step with the statistics of whole sequences, the headline batch.
        _case("norm_train", 64, 512, name="norm_sequence_train", D=1024, G=32),
        # Very long documents in a tiny batch, few and large groups.
        _case("norm", 4, 16384, name="norm_sequence_long", D=512, G=8, min_len=9000),
        # Training on a handful of short sentences against a small vocabulary.
        _case("distill_train", 4, 8, name="distill_small", dtype="f32", V=5003, K=16),
        # How far a tagger's emissions are from a larger tagger's, over the headline batch.
        _case("distill", 64, 512, name="distill_tags", dtype="f32", V=128, K=8, temperature=2.0, min_len=200),
        # Training step of a word model over a large table, from a teacher's stored top logits.
        _case("distill_train", 16, 256, name="distill_words", V=100003, K=64, min_len=128),
    ]


OPS = ("rec", "rec", "rec_train", "rec_train", "rec_step", "norm", "norm_train", "norm_train", "norm_position", "norm_position_train", "distill", "distill_train",
       "distill_train")
MAX_ENTRIES = 1 << 26  # positions * channels of a drawn case
MAX_LOGITS = 1 << 28   # positions * classes: the listed ones reach 4e8


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op, dtype = rng.choice(OPS), rng.choice(("f32", "bf16"))
    if op.endswith("step"):
        B, N = _log_int(rng, 1, 512), 1
    elif rng.random() < 0.25:  # long documents in a small batch
        B, N = rng.randint(1, 8), _log_int(rng, 1024, 16384)
    else:
        B, N = _log_int(rng, 1, 128), _log_int(rng, 1, 512)
    if op.startswith("distill"):
        V = _log_int(rng, 5, 120000)
        while B * N * V > MAX_LOGITS:
            B, N = max(1, B // 2), N if B > 1 else N // 2
        return _case(op, B, N, dtype=dtype, min_len=N if rng.random() < 0.4 else rng.randint(0, N), V=V, K=min(V, _log_int(rng, 1, 128)),
                     temperature=rng.choice((1.0, 1.0, 2.0, 3.5)))
    D = _log_int(rng, 32, 2048)
    if rng.random() < 0.5:
        D = -(-D // 8) * 8
    G = 1
    if op.startswith("norm"):
        G = _log_int(rng, 1, 64)
        D = max(4, -(-D // G)) * G
    while B * N * D > MAX_ENTRIES:
        B, N = max(1, B // 2), N if B > 1 else N // 2
    min_len = N if op == "rec_step" or rng.random() < 0.4 else rng.randint(0, N)
    if op.startswith("rec"):
        return _case(op, B, N, dtype=dtype, min_len=min_len, D=D, gate=rng.random() < 0.7, carry=rng.random() < 0.5)
    return _case(op, B, N, dtype=dtype, min_len=min_len, D=D, G=G, silu=rng.random() < 0.7)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    op, B, N, t = case["op"], case["B"], case["N"], DTYPES[case["dtype"]]

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return torch.randn(shape, generator=g, device=DEVICE).mul_(scale).to(dtype)

    s = {"op": op, "lengths": None}
    if case["min_len"] < N:
        s["lengths"] = torch.randint(case["min_len"], N + 1, (B,), generator=g, device=DEVICE).to(torch.int32)
    if op.startswith("distill"):
        # The teacher knows more than the student: its largest logits are the student's, moved.  Padding has no entry of the teacher's.
        V, K = case["V"], case["K"]
        logits = torch.randn(B, N, V, generator=g, device=DEVICE).mul_(2.0)
        teacher, ids = torch.topk(logits + torch.randn(B, N, V, generator=g, device=DEVICE), K, -1)
        ids = ids.to(torch.int32)
        if s["lengths"] is not None:
            ids[torch.arange(N, device=DEVICE)[None, :] >= s["lengths"][:, None]] = -1
        s |= {"logits": logits.to(t), "ids": ids, "teacher": teacher, "temperature": case["temperature"]}
        if op == "distill_train":
            s["dloss"] = torch.full((B, N), 1.0 / (B * N), device=DEVICE)
        return s
    D = case["D"]
    if op.startswith("norm"):
        s |= {"G": case["G"], "silu": case["silu"], "weight": 1 + normal(D, scale=0.1), "bias": normal(D, scale=0.1),
              "x": (normal(B, N, D, scale=2.0) + normal(D, scale=0.5)).to(t)}
        if op.endswith("train"):
            s["dout"] = normal(B, N, D, dtype=t)
        return s
    rows = (B,) if op == "rec_step" else (B, N)
    # Decays between 0.9 and 0.999 where the gate is wide open.
    c = -torch.log(0.9 + 0.099 * torch.rand(D, generator=g, device=DEVICE)) / RATE
    s |= {"decay": torch.log(torch.expm1(c)), "f_bias": normal(D, scale=0.1), "g_bias": normal(D, scale=0.1), "x": normal(*rows, D, dtype=t), "z": None,
          "state": None}
    # The gates are the halves of one projection's output.
    gates = normal(*rows, 2 * D, dtype=t)
    s |= {"f": gates[..., :D], "g": gates[..., D:]}
    if case["gate"]:
        s["z"] = normal(*rows, D, dtype=t)
    if case["carry"] or op == "rec_step":
        s["state"] = normal(B, D)
    if op == "rec_train":
        s["dout"] = normal(B, N, D, dtype=t)
    return s


# ---- plain forms: elementary operations in 32 bits, rounded once ----------------------------------------------

def _inside(s, B, N):
    """[B, N, 1]: which positions lie within their sequence."""
    if s["lengths"] is None:
        return torch.ones(B, N, 1, dtype=torch.bool, device=DEVICE)
    return (torch.arange(N, device=DEVICE)[None, :] < s["lengths"][:, None])[..., None]


def _recursion(a, b):
    """h with h[l] = a[l] h[l-1] + b[l] along dimension 1, all positions at a time: spans that double."""
    span, N = 1, a.shape[1]
    while span < N:
        b = torch.cat([b[:, :span], b[:, span:] + a[:, span:] * b[:, :-span]], 1)
        a = torch.cat([a[:, :span], a[:, span:] * a[:, :-span]], 1)
        span *= 2
    return b


def _gates(s):
    """x, the decay's logarithm and gate, what the input is taken with (of the decay, of its gate)."""
    open_ = torch.sigmoid(s["f"].float() + s["f_bias"])
    u = -RATE * torch.log1p(torch.exp(s["decay"])) * open_
    return s["x"].float(), u, open_, torch.sqrt(-torch.expm1(2 * u)), torch.sigmoid(s["g"].float() + s["g_bias"])


def _plain_rec(s):
    x, u, open_, m, take = _gates(s)
    inside = _inside(s, *x.shape[:2])
    x, u = torch.where(inside, x, 0.0), torch.where(inside, u, 0.0)
    a, b = torch.exp(u), torch.where(inside, m * take * x, 0.0)
    if s["state"] is not None:
        b[:, 0] += a[:, 0] * s["state"]
    h = _recursion(a, b)
    out = h if s["z"] is None else h * s["z"].float() * torch.sigmoid(s["z"].float())
    return torch.where(inside, out, 0.0).to(s["x"].dtype), h[:, -1].contiguous(), inside, x, u, open_, m, take, a, h


def _plain_rec_train(s):
    out, final, inside, x, u, open_, m, take, a, h = _plain_rec(s)
    t = s["x"].dtype
    dy = torch.where(inside, s["dout"].float(), 0.0)
    grads = {"out": out, "final": final}
    if s["z"] is not None:
        z = s["z"].float()
        gate = torch.sigmoid(z)
        grads["dz"] = torch.where(inside, dy * h * gate * (1 + z * (1 - gate)), 0.0).to(t)
        dy = torch.where(inside, dy * z * gate, 0.0)
    after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    dh = _recursion(after.flip(1), dy.flip(1)).flip(1)
    first = torch.zeros_like(h[:, :1]) if s["state"] is None else s["state"][:, None]
    du = dh * a * torch.cat([first, h[:, :-1]], 1) - dh * take * x * a * a / m
    dlog = torch.where(inside, du * u, 0.0)  # by the logarithm of u
    df = dlog * (1 - open_)
    dg = torch.where(inside, dh * m * x * take * (1 - take), 0.0)
    if s["state"] is not None:
        grads["dstate"] = dh[:, 0] * a[:, 0]
    slope = torch.sigmoid(s["decay"]) / torch.log1p(torch.exp(s["decay"]))
    return grads | {"dx": torch.where(inside, dh * m * take, 0.0).to(t), "df": df.to(t), "dg": dg.to(t), "ddecay": dlog.sum((0, 1)) * slope,
                    "df_bias": df.sum((0, 1)), "dg_bias": dg.sum((0, 1))}


def _plain_rec_step(s):
    x, u, _, m, take = _gates(s)
    h = torch.exp(u) * s["state"] + m * take * x
    s["state"].copy_(h)
    out = h if s["z"] is None else h * s["z"].float() * torch.sigmoid(s["z"].float())
    return out.to(s["x"].dtype), s["state"]


def _plain_norm(s):
    """The result, statistics [B, G, 2] or [B, N, G, 2], and for the gradient the normalised values, what the mean goes over, the activation's argument."""
    (B, N, D), G = s["x"].shape, s["G"]
    over = (3,) if s["op"].startswith("norm_position") else (1, 3)
    inside = _inside(s, B, N)[..., None]
    x = torch.where(inside, s["x"].float().view(B, N, G, D // G), 0.0)
    count = (inside.float().sum(1, keepdim=True) if len(over) == 2 else inside.float()).clamp_min(1) * (D // G)
    mean = x.sum(over, keepdim=True) / count
    away = torch.where(inside, x - mean, 0.0)
    rstd = torch.rsqrt((away * away).sum(over, keepdim=True) / count + EPS)
    hat = away * rstd
    y = hat * s["weight"].view(G, -1) + s["bias"].view(G, -1)
    out = torch.where(inside, y * torch.sigmoid(y) if s["silu"] else y, 0.0).view(B, N, D).to(s["x"].dtype)
    some = inside if len(over) == 1 else inside.any(1, keepdim=True)
    stats = torch.where(some, torch.cat([mean, rstd], 3), 0.0)
    return out, stats if len(over) == 1 else stats[:, 0], hat, y, inside, over, count, rstd


def _plain_norm_train(s):
    out, stats, hat, y, inside, over, count, rstd = _plain_norm(s)
    (B, N, D), G = s["x"].shape, s["G"]
    dy = torch.where(inside, s["dout"].float().view(hat.shape), 0.0)
    if s["silu"]:
        gate = torch.sigmoid(y)
        dy = dy * gate * (1 + y * (1 - gate))
    dhat = dy * s["weight"].view(G, -1)
    dx = rstd * (dhat - dhat.sum(over, keepdim=True) / count - hat * (dhat * hat).sum(over, keepdim=True) / count)
    return {"out": out, "stats": stats, "dx": torch.where(inside, dx, 0.0).view(B, N, D).to(s["x"].dtype), "dweight": (dy * hat).sum((0, 1)).flatten(),
            "dbias": dy.sum((0, 1)).flatten()}


def _plain_distill(s):
    t, V = s["temperature"], s["logits"].shape[-1]
    there = s["ids"] >= 0
    any_, ids = there.any(-1), s["ids"].clamp_min(0).long()
    x = s["logits"].float() / t
    top = x.amax(-1, keepdim=True)
    lse = top[..., 0] + torch.log(torch.exp(x - top).sum(-1))
    v = torch.where(there, s["teacher"] / t, -math.inf)
    highest = torch.where(any_, v.amax(-1), 0.0)[..., None]
    e = torch.exp(v - highest)
    total = e.sum(-1, keepdim=True)
    q = torch.where(any_[..., None], e / total, 0.0)
    ratio = v - highest - torch.log(total) - (x.gather(-1, ids) - lse[..., None])  # log q - log p
    loss = t * t * torch.where(q > 0, q * ratio, 0.0).sum(-1)
    return loss, torch.where(any_, lse, 0.0), x, lse, q, ids, any_


def _plain_distill_train(s):
    loss, _, x, lse, q, ids, any_ = _plain_distill(s)
    p = torch.exp(x - lse[..., None])
    p.scatter_add_(-1, ids, -q)
    scale = torch.where(any_, s["dloss"] * s["temperature"], 0.0)
    return {"loss": loss, "dlogits": (p * scale[..., None]).to(s["logits"].dtype)}


PLAIN = {"rec": lambda s: _plain_rec(s)[:2], "rec_train": _plain_rec_train, "rec_step": _plain_rec_step, "norm": lambda s: _plain_norm(s)[0],
         "norm_train": _plain_norm_train, "norm_position": lambda s: _plain_norm(s)[0], "norm_position_train": _plain_norm_train,
         "distill": lambda s: _plain_distill(s)[:2], "distill_train": _plain_distill_train}


# ---- the framework's calls ------------------------------------------------------------------------------------

def _own(s):
    from paper_2308_03291_amd import binding as crf
    op, lengths = s["op"], s["lengths"]
    if op.startswith("distill"):
        if op == "distill":
            return crf.lccrf_distill(s["logits"], s["ids"], s["teacher"], temperature=s["temperature"])
        loss = torch.empty_like(s["dloss"])
        dlogits = crf.lccrf_distill_grad(s["dloss"], s["logits"], s["ids"], s["teacher"], temperature=s["temperature"], loss=loss)
        return {"loss": loss, "dlogits": dlogits}
    if op.startswith("norm"):
        how = {"groups": s["G"], "eps": EPS, "silu": s["silu"], "per_position": op.startswith("norm_position")}
        inputs = s["x"], s["weight"], s["bias"], lengths
        if not op.endswith("train"):
            return crf.lccrf_group_norm(*inputs, **how)
        stats = crf.group_norm_stats(s["x"], s["G"], per_position=how["per_position"])
        out = crf.lccrf_group_norm(*inputs, **how, stats=stats)
        g = crf.lccrf_group_norm_grad(s["dout"], *inputs, **how, stats=stats)
        return {"out": out, "stats": stats, "dx": g.dx, "dweight": g.dweight, "dbias": g.dbias}
    inputs = [s[k] for k in ("x", "f", "g", "decay", "z", "f_bias", "g_bias")]
    if op == "rec_step":
        return crf.lccrf_recurrence_step(*inputs, s["state"], rate=RATE), s["state"]
    if op == "rec":
        return crf.lccrf_recurrence(*inputs, lengths, rate=RATE, state=s["state"])
    saved = crf.recurrence_saved(s["x"])
    out, final = crf.lccrf_recurrence(*inputs, lengths, rate=RATE, state=s["state"], saved=saved)
    g = crf.lccrf_recurrence_grad(s["dout"], *inputs, lengths, rate=RATE, state=s["state"], saved=saved)
    grads = {"out": out, "final": final, "dx": g.dx, "df": g.df, "dg": g.dg, "ddecay": g.ddecay, "df_bias": g.df_bias, "dg_bias": g.dg_bias}
    if s["z"] is not None:
        grads["dz"] = g.dz
    if s["state"] is not None:
        grads["dstate"] = g.dstate
    return grads


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


def work(case):
    """Inputs inside the sequences read once, results written once.  The recurrence takes two gates, the decay, its root and the recursion, some
    twenty-four operations a value, ten with an output gate, its gradient forty and ten more; a normalisation ten, six with its activation, its
    gradient twice that; a logit four (maximum, exponential, sum), in training four more."""
    op, B, N = case["op"], case["B"], case["N"]
    e = 4 if case["dtype"] == "f32" else 2
    n = B * N                                   # positions written
    m = n * 0.5 * (case["min_len"] + N) / N     # positions read
    if op.startswith("distill"):
        V, K = case["V"], case["K"]
        bytes_ = e * m * V + 4.0 * n * (2 * K + 2) + (e * n * V if op == "distill_train" else 0)
        return {"bytes": bytes_, "flops": m * (V * (8.0 if op == "distill_train" else 4.0) + 8.0 * K)}
    D = case["D"]
    if op.startswith("norm"):
        train, stats = op.endswith("train"), 8.0 * case["G"] * (n if op.startswith("norm_position") else B)
        bytes_ = e * D * (m + n) + 8.0 * D
        flops = m * D * (10.0 + 6.0 * case["silu"])
        if train:
            bytes_ += e * D * (m + n) + 8.0 * D + stats
            flops *= 3
        return {"bytes": bytes_, "flops": flops}
    z, state = int(case["gate"]), 4.0 * B * D
    bytes_ = e * D * (m * (3 + z) + n) + state * (2 if case["carry"] or op == "rec_step" else 1) + 12.0 * D
    flops = m * D * (24.0 + 10.0 * z)
    if op == "rec_train":
        bytes_ += e * D * (m + n * (3 + z)) + 12.0 * D + (state if case["carry"] else 0)
        flops += m * D * (40.0 + 10.0 * z)
    return {"bytes": bytes_, "flops": flops}


# ---- the same values in 64 bits -------------------------------------------------------------------------------

def _silu64(v):
    return v / (1 + torch.exp(-v))


def _dsilu64(v):
    return (1 + torch.exp(-v) * (1 + v)) / (1 + torch.exp(-v)) ** 2


def exact(case, seed):
    s = prepare(case, seed)
    op, B, N = case["op"], case["B"], case["N"]
    lens = torch.full((B,), N, device=DEVICE) if s["lengths"] is None else s["lengths"].long()
    if op.startswith("distill"):
        return _exact_distill(case, s)
    if op.startswith("norm"):
        return _exact_norm(case, s, lens)
    return _exact_rec(case, s, lens)


def _exact_rec(case, s, lens):
    """Position by position."""
    op, N = case["op"], case["N"]
    one = op == "rec_step"
    get = lambda k: (s[k][:, None] if one else s[k]).double()  # noqa: E731
    x, f, g, lam = get("x"), get("f") + s["f_bias"].double(), get("g") + s["g_bias"].double(), s["decay"].double()
    z = None if s["z"] is None else get("z")
    soft = torch.logaddexp(lam, torch.zeros_like(lam))
    u = -RATE * soft / (1 + torch.exp(-f))
    a, take = torch.exp(u), 1 / (1 + torch.exp(-g))
    m = torch.sqrt(-torch.expm1(2 * u))
    B, _, D = x.shape
    h = torch.zeros(B, D, dtype=torch.float64, device=DEVICE) if s["state"] is None else s["state"].double()
    y, before = torch.empty_like(x), torch.empty_like(x)
    for l in range(N):
        before[:, l] = h
        h = torch.where((lens > l)[:, None], a[:, l] * h + m[:, l] * take[:, l] * x[:, l], h)
        y[:, l] = h
    on = (torch.arange(N, device=DEVICE)[None, :] < lens[:, None])[..., None]
    out = torch.where(on, y if z is None else y * _silu64(z), 0.0)
    if one:
        return out[:, 0], h
    if op == "rec":
        return out, h
    grads = {"out": out, "final": h}
    dout = torch.where(on, s["dout"].double(), 0.0)
    dy = dout
    if z is not None:
        grads["dz"] = dout * y * _dsilu64(z)
        dy = dout * _silu64(z)
    dh, carry = torch.empty_like(x), torch.zeros_like(h)
    for l in range(N - 1, -1, -1):
        now = dy[:, l] + carry
        dh[:, l] = torch.where((lens > l)[:, None], now, 0.0)
        carry = torch.where((lens > l)[:, None], now * a[:, l], carry)
    grads["dx"] = dh * m * take
    grads["dg"] = dh * m * x * torch.exp(-g) * take ** 2
    du = dh * (before * a - take * x * a * a / m)
    grads["df"] = du * u * torch.exp(-f) / (1 + torch.exp(-f))
    grads["ddecay"] = (du * u).sum((0, 1)) / soft / (1 + torch.exp(-lam))
    grads["df_bias"], grads["dg_bias"] = grads["df"].sum((0, 1)), grads["dg"].sum((0, 1))
    if s["state"] is not None:
        grads["dstate"] = carry
    return grads


def _exact_norm(case, s, lens):
    """Sequence by sequence."""
    op, (B, N, D), G = case["op"], s["x"].shape, s["G"]
    alone, train = op.startswith("norm_position"), op.endswith("train")
    w, bias = s["weight"].double(), s["bias"].double()
    out = torch.zeros(B, N, D, dtype=torch.float64, device=DEVICE)
    stats = torch.zeros(*((B, N) if alone else (B,)), G, 2, dtype=torch.float64, device=DEVICE)
    dx, dweight, dbias = torch.zeros_like(out), torch.zeros_like(w), torch.zeros_like(w)
    for b, n in enumerate(lens.tolist()):
        if n == 0:
            continue
        # one line for each set of values that is normalised together
        lines = lambda v: v.view(n * G, D // G) if alone else v.view(n, G, D // G).transpose(0, 1).reshape(G, -1)  # noqa: E731
        back = lambda v: v.view(n, D) if alone else v.view(G, n, D // G).transpose(0, 1).reshape(n, D)  # noqa: E731
        v = lines(s["x"][b, :n].double())
        var, mean = torch.var_mean(v, 1, unbiased=False, keepdim=True)
        rstd = 1 / torch.sqrt(var + EPS)
        hat = (v - mean) * rstd
        stats_b = torch.cat([mean, rstd], 1)
        if alone:
            stats[b, :n] = stats_b.view(n, G, 2)
        else:
            stats[b] = stats_b
        y = back(hat) * w + bias
        out[b, :n] = _silu64(y) if s["silu"] else y
        if train:
            dy = s["dout"][b, :n].double() * (_dsilu64(y) if s["silu"] else 1.0)
            dhat = lines(dy * w)
            dx[b, :n] = back(rstd * (dhat - dhat.mean(1, keepdim=True) - hat * (dhat * hat).mean(1, keepdim=True)))
            dweight += (dy * back(hat)).sum(0)
            dbias += dy.sum(0)
    return {"out": out, "stats": stats, "dx": dx, "dweight": dweight, "dbias": dbias} if train else out


def _exact_distill(case, s):
    t, op = s["temperature"], case["op"]
    ids, there = s["ids"].long(), s["ids"] >= 0
    some = there.any(-1)
    q = torch.zeros(*ids.shape, dtype=torch.float64, device=DEVICE)
    q[some] = torch.softmax(torch.where(there, s["teacher"].double() / t, -math.inf)[some], -1)
    loss, lse = torch.zeros_like(q[..., 0]), torch.zeros_like(q[..., 0])
    dlogits = torch.zeros(s["logits"].shape, dtype=torch.float64, device=DEVICE) if op == "distill_train" else None
    for b in range(ids.shape[0]):  # a sequence at a time: 64 bits take room
        x = s["logits"][b].double() / t
        of = torch.logsumexp(x, -1)
        logp = (x - of[:, None]).gather(-1, ids[b].clamp_min(0))
        loss[b] = t * t * (torch.special.xlogy(q[b], q[b]) - q[b] * torch.where(there[b], logp, 0.0)).sum(-1)
        lse[b] = torch.where(some[b], of, 0.0)
        if dlogits is not None:
            p = torch.softmax(x, -1)
            p.scatter_add_(-1, ids[b].clamp_min(0), -q[b])
            dlogits[b] = p * (s["dloss"][b].double() * t * some[b])[:, None]
    return (loss, lse) if op == "distill" else {"loss": loss, "dlogits": dlogits}
