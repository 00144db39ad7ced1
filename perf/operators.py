"""The operators of a tagger's encoder, the part in front of the chain: what is measured of them.

Embedding lookup and its gradient, the short causal convolution and the selective state space scan, each as a prompt (or a
batch of sentences), in training and for single tokens.  A case is one pass of one of them.  ``op`` names it; ``B`` sequences
of at most ``N`` positions (the shortest ``min_len``), ``D`` channels, ``S`` states a channel, ``G`` groups of channels that
share the input and output vectors, ``K`` taps, ``V`` rows of the table.  Batch sizes and lengths are those of
``paper_2308_03291_amd.workloads``, widths and table sizes are generic.
"""
from __future__ import annotations

import math

import torch

DEVICE = "cuda"

#: False: ``run`` computes the plain forms below.  True: it calls the framework.
own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(op, B, N, D, *, name=None, dtype="bf16", min_len=None, V=0, K=4, S=16, G=1, gate=True, carry=False):
    c = {"op": op, "B": B, "N": N, "D": D, "dtype": dtype, "min_len": N if min_len is None else min_len}
    if op.startswith("embed"):
        c |= {"V": V}
    elif op.startswith("conv"):
        c |= {"K": K, "carry": carry}
    else:
        c |= {"S": S, "G": G, "gate": gate, "carry": carry}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # Looking up a handful of short sentences: latency is all there is.
        _case("embed", 4, 8, 256, name="embed_tiny", dtype="f32", V=5000),
        # A batch of the size the paper times its chain on, half precision.
        _case("embed", 128, 256, 1024, name="embed_batch", V=50000, min_len=64),
        # Gradient of a small table with an odd width, a small ragged batch.
        _case("embed_grad", 32, 64, 301, name="embed_grad_small_odd", dtype="f32", V=4099, min_len=32),
        # Gradient of a large table over the tokens of the headline batch, token frequencies as in text.
        _case("embed_grad", 64, 512, 1024, name="embed_grad_large", V=100003),
        # Convolution over a batch of prompts that continue earlier ones.
        _case("conv", 64, 512, 2048, name="conv_prompt", carry=True),
        # Training step of the convolution on ragged sentences, an odd width, single precision.
        _case("conv_train", 128, 128, 1001, name="conv_train_odd", dtype="f32", min_len=16),
        # One token for every stream of a server, the convolution's part.
        _case("conv_step", 64, 1, 2048, name="conv_step"),
        # One token for a few streams, the scan's part: latency.
        _case("scan_step", 4, 1, 1024, name="scan_step_few", dtype="f32"),
        # One token for many streams: the states are read and written.
        _case("scan_step", 512, 1, 2048, name="scan_step_many"),
        # Prompts of the headline batch.
        _case("scan", 64, 512, 2048, name="scan_prompt", carry=True),
        # Very long documents in a tiny batch, an odd width, two groups, no gate.
        _case("scan", 4, 16384, 514, name="scan_long", S=16, G=2, gate=False),
        # Training step on ragged sentences.
        _case("scan_train", 128, 256, 1024, name="scan_train", min_len=64),
    ]


OPS = ("embed", "embed_grad", "embed_grad", "conv", "conv_train", "conv_train", "conv_step", "scan", "scan", "scan_train", "scan_train", "scan_step")
MAX_UPDATES = 1 << 29   # positions * channels * states of a drawn scan: the listed ones reach 1 << 30
MAX_ENTRIES = 1 << 26   # positions * channels, and entries of a table


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op, dtype = rng.choice(OPS), rng.choice(("f32", "bf16"))
    D = _log_int(rng, 32, 2048)
    if rng.random() < 0.5:
        D = -(-D // 8) * 8
    if op.endswith("step"):
        B, N = _log_int(rng, 1, 512), 1
    elif rng.random() < 0.25:  # long documents in a small batch
        B, N = rng.randint(1, 8), _log_int(rng, 1024, 16384)
    else:
        B, N = _log_int(rng, 1, 128), _log_int(rng, 1, 512)
    while B * N * D > MAX_ENTRIES:
        B, N = max(1, B // 2), N if B > 1 else N // 2
    min_len = N if rng.random() < 0.4 else rng.randint(0, N)
    gate, carry = rng.random() < 0.7, rng.random() < 0.5
    if op.startswith("embed"):
        return _case(op, B, N, D, dtype=dtype, min_len=min_len, V=_log_int(rng, 100, MAX_ENTRIES // D))
    if op.startswith("conv"):
        return _case(op, B, N, D, dtype=dtype, min_len=min_len, K=rng.choice((2, 3, 4, 4, 4, 5, 8)), carry=carry)
    S = rng.choice((4, 8, 13, 16, 16, 16, 32, 64))
    G = rng.choice((1, 1, 1, 2, 4))
    D = -(-D // G) * G
    while B * N * D * S > MAX_UPDATES:
        B, N = max(1, B // 2), N if B > 1 else N // 2
    return _case(op, B, N, D, dtype=dtype, min_len=min(min_len, N), S=S, G=G, gate=gate, carry=carry)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    op, B, N, D, t = case["op"], case["B"], case["N"], case["D"], DTYPES[case["dtype"]]

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(shape, generator=g, device=DEVICE) * scale).to(dtype)

    s = {"op": op, "lengths": None}
    if case["min_len"] < N:
        s["lengths"] = torch.randint(case["min_len"], N + 1, (B,), generator=g, device=DEVICE).to(torch.int32)
    if op.startswith("embed"):
        # Frequencies fall with the rank, as in text; padding is -1.
        u = torch.rand(B, N, generator=g, device=DEVICE, dtype=torch.float64)
        rank = (float(case["V"]) ** u - 1).long().clamp(0, case["V"] - 1)
        ids = torch.randperm(case["V"], generator=g, device=DEVICE)[rank].to(torch.int32)
        if s["lengths"] is not None:
            ids[torch.arange(N, device=DEVICE)[None, :] >= s["lengths"][:, None]] = -1
        s |= {"ids": ids, "V": case["V"], "scale": math.sqrt(D)}
        if op == "embed":
            s["table"] = normal(case["V"], D, dtype=t, scale=0.02)
        else:
            s["dout"] = normal(B, N, D, dtype=t)
        return s
    if op.startswith("conv"):
        K = case["K"]
        s |= {"weight": normal(D, K, scale=K ** -0.5), "bias": normal(D, scale=0.1), "state": None}
        if op == "conv_step":
            s |= {"x": normal(B, D, dtype=t), "state": normal(B, K - 1, D, dtype=t)}
            return s
        # The input is one half of a projection's output, rows twice as long as it is wide.
        s["x"] = normal(B, N, 2 * D, dtype=t)[:, :, :D]
        if case["carry"]:
            s["state"] = normal(B, K - 1, D, dtype=t)
        if op == "conv_train":
            s["dout"] = normal(B, N, D, dtype=t)
        return s
    S, G = case["S"], case["G"]
    rows = (B,) if op == "scan_step" else (B, N)
    step = torch.exp(torch.rand(D, generator=g, device=DEVICE) * math.log(100.0) + math.log(1e-3))  # 0.001 .. 0.1
    s |= {
        "A": -torch.arange(1, S + 1, device=DEVICE).float().repeat(D, 1) * torch.exp(normal(D, S, scale=0.1)),
        "D": 1 + normal(D, scale=0.1), "dt_bias": step + torch.log(-torch.expm1(-step)),
        "x": normal(*rows, D, dtype=t), "dt": normal(*rows, D, dtype=t, scale=0.5),
        "Bm": normal(*rows, G, S, dtype=t), "Cm": normal(*rows, G, S, dtype=t), "z": None, "state": None,
    }
    if case["gate"]:
        s["z"] = normal(*rows, 2 * D, dtype=t)[..., D:]
    if case["carry"] or op == "scan_step":
        s["state"] = normal(B, D, S)
    if op == "scan_train":
        s["dout"] = normal(B, N, D, dtype=t)
    return s


# ---- plain forms: elementary operations in 32 bits, rounded once ----------------------------------------------

def _plain_embed(s):
    ids = s["ids"].long()
    out = s["table"][ids.clamp_min(0)].float() * s["scale"]
    return torch.where((ids >= 0)[..., None], out, 0.0).to(s["table"].dtype)


def _plain_embed_grad(s):
    ids, dout = s["ids"].reshape(-1).long(), s["dout"].reshape(-1, s["dout"].shape[-1])
    grad = torch.zeros(s["V"] + 1, dout.shape[1], device=DEVICE)
    grad.index_add_(0, torch.where(ids < 0, s["V"], ids), dout.float() * s["scale"])
    return grad[:-1].to(dout.dtype)


def _inside(s, B, N):
    """[B, N, 1]: which positions lie within their sequence."""
    if s["lengths"] is None:
        return torch.ones(B, N, 1, dtype=torch.bool, device=DEVICE)
    return (torch.arange(N, device=DEVICE)[None, :] < s["lengths"][:, None])[..., None]


def _plain_conv(s):
    """The output, the last inputs (what a later call continues from) and what the gradient takes from the way there."""
    x, w = s["x"], s["weight"]
    (B, N, D), K = x.shape, w.shape[1]
    before = torch.zeros(B, K - 1, D, device=DEVICE) if s["state"] is None else s["state"].float()
    inside = _inside(s, B, N)
    rows = torch.cat([before, torch.where(inside, x.float(), 0.0)], 1)
    taps = rows.unfold(1, K, 1)  # [B, N, D, K]
    pre = (taps * w).sum(-1) + s["bias"]
    out = torch.where(inside, pre * torch.sigmoid(pre), 0.0).to(x.dtype)
    length = inside.sum(1)  # [B, 1]
    last = length + torch.arange(K - 1, device=DEVICE)
    final = torch.gather(rows, 1, last[..., None].expand(-1, -1, D)).to(x.dtype)
    return out, final, taps, pre, inside


def _plain_conv_train(s):
    out, final, taps, pre, inside = _plain_conv(s)
    K, t = s["weight"].shape[1], s["x"].dtype
    gate = torch.sigmoid(pre)
    dpre = torch.where(inside, s["dout"].float() * gate * (1 + pre * (1 - gate)), 0.0)
    dweight, dbias = (taps * dpre[..., None]).sum((0, 1)), dpre.sum((0, 1))
    around = torch.nn.functional.pad(dpre, (0, 0, K - 1, K - 1)).unfold(1, K, 1)
    drows = (around * s["weight"].flip(1)).sum(-1)  # [B, K - 1 + N, D]
    grads = {"out": out, "final": final, "dx": drows[:, K - 1:].to(t), "dweight": dweight, "dbias": dbias}
    if s["state"] is not None:
        grads["dstate"] = drows[:, : K - 1].to(t)
    return grads


def _plain_conv_step(s):
    rows = torch.cat([s["state"], s["x"][:, None]], 1)
    pre = (rows.float().transpose(1, 2) * s["weight"]).sum(-1) + s["bias"]
    s["state"].copy_(rows[:, 1:])
    return (pre * torch.sigmoid(pre)).to(s["x"].dtype), s["state"]


def _recursion(a, b):
    """h with h[l] = a[l] h[l-1] + b[l] along dimension 1, all positions at a time: spans that double."""
    span, N = 1, a.shape[1]
    while span < N:
        b = torch.cat([b[:, :span], b[:, span:] + a[:, span:] * b[:, :-span]], 1)
        a = torch.cat([a[:, :span], a[:, span:] * a[:, :-span]], 1)
        span *= 2
    return b


def _wide(m, D):
    """[..., G, S] to [..., D, S]: every channel its group's vector."""
    return m.float().repeat_interleave(D // m.shape[-2], -2)


def _plain_scan(s):
    x, D = s["x"].float(), s["x"].shape[-1]
    inside = _inside(s, *x.shape[:2])
    x = torch.where(inside, x, 0.0)
    v = s["dt"].float() + s["dt_bias"]
    step = torch.where(inside, torch.clamp_min(v, 0) + torch.log1p(torch.exp(-v.abs())), 0.0)
    decay = torch.exp(step[..., None] * s["A"])
    put = (step * x)[..., None] * _wide(s["Bm"], D)
    if s["state"] is not None:
        put[:, 0] += decay[:, 0] * s["state"]
    h = _recursion(decay, put)
    y = (h * _wide(s["Cm"], D)).sum(-1) + s["D"] * x
    out = y if s["z"] is None else y * s["z"].float() * torch.sigmoid(s["z"].float())
    return torch.where(inside, out, 0.0).to(s["x"].dtype), h[:, -1].contiguous(), inside, x, v, step, decay, h, y


def _plain_scan_train(s):
    out, final, inside, x, v, step, decay, h, y = _plain_scan(s)
    t, (B, N, D), (G, S) = s["x"].dtype, x.shape, s["Bm"].shape[-2:]
    dy = torch.where(inside, s["dout"].float(), 0.0)
    grads = {"out": out, "final": final}
    if s["z"] is not None:
        z = s["z"].float()
        gate = torch.sigmoid(z)
        grads["dz"] = torch.where(inside, dy * y * gate * (1 + z * (1 - gate)), 0.0).to(t)
        dy = torch.where(inside, dy * z * gate, 0.0)
    grads["dCm"] = (dy[..., None] * h).view(B, N, G, D // G, S).sum(3).to(t)
    after = torch.cat([decay[:, 1:], torch.zeros_like(decay[:, :1])], 1)
    dh = _recursion(after.flip(1), (dy[..., None] * _wide(s["Cm"], D)).flip(1)).flip(1)
    first = torch.zeros_like(h[:, :1]) if s["state"] is None else s["state"][:, None]
    back = dh * decay * torch.cat([first, h[:, :-1]], 1)  # by the decay's logarithm
    if s["state"] is not None:
        grads["dstate"] = dh[:, 0] * decay[:, 0]
    grads["dBm"] = torch.where(inside[..., None], (dh * (step * x)[..., None]).view(B, N, G, D // G, S).sum(3), 0.0).to(t)
    dput = (dh * _wide(s["Bm"], D)).sum(-1)
    dv = torch.where(inside, (dput * x + (back * s["A"]).sum(-1)) * torch.sigmoid(v), 0.0)
    grads |= {
        "dx": torch.where(inside, dput * step + s["D"] * dy, 0.0).to(t), "ddt": dv.to(t), "ddt_bias": dv.sum((0, 1)),
        "dA": (back * step[..., None]).sum((0, 1)), "dD": (dy * x).sum((0, 1)),
    }
    return grads


def _plain_scan_step(s):
    x, D = s["x"].float(), s["x"].shape[-1]
    v = s["dt"].float() + s["dt_bias"]
    step = torch.clamp_min(v, 0) + torch.log1p(torch.exp(-v.abs()))
    h = torch.exp(step[..., None] * s["A"]) * s["state"] + (step * x)[..., None] * _wide(s["Bm"], D)
    s["state"].copy_(h)
    y = (h * _wide(s["Cm"], D)).sum(-1) + s["D"] * x
    if s["z"] is not None:
        y = y * s["z"].float() * torch.sigmoid(s["z"].float())
    return y.to(s["x"].dtype), s["state"]


PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "conv": lambda s: _plain_conv(s)[:2],
         "conv_train": _plain_conv_train, "conv_step": _plain_conv_step, "scan": lambda s: _plain_scan(s)[:2],
         "scan_train": _plain_scan_train, "scan_step": _plain_scan_step}


# ---- the framework's calls ------------------------------------------------------------------------------------

def _own(s):
    from paper_2308_03291_amd import binding as crf
    op, lengths = s["op"], s["lengths"]
    if op == "embed":
        return crf.lccrf_embed(s["table"], s["ids"], scale=s["scale"])
    if op == "embed_grad":
        return crf.lccrf_embed_grad(s["dout"], s["ids"], s["V"], scale=s["scale"])
    if op == "conv_step":
        return crf.lccrf_conv_step(s["x"], s["weight"], s["bias"], s["state"]), s["state"]
    if op.startswith("conv"):
        out, final = crf.lccrf_conv(s["x"], s["weight"], s["bias"], lengths, state=s["state"])
        if op == "conv":
            return out, final
        g = crf.lccrf_conv_grad(s["dout"], s["x"], s["weight"], s["bias"], lengths, state=s["state"])
        grads = {"out": out, "final": final, "dx": g.dx, "dweight": g.dweight, "dbias": g.dbias}
        if s["state"] is not None:
            grads["dstate"] = g.dstate
        return grads
    inputs = [s[k] for k in ("x", "dt", "A", "Bm", "Cm", "D", "z", "dt_bias")]
    if op == "scan_step":
        return crf.lccrf_state_step(*inputs, s["state"]), s["state"]
    if op == "scan":
        return crf.lccrf_state_scan(*inputs, lengths, state=s["state"])
    saved = crf.state_scan_saved(s["x"], s["A"])
    out, final = crf.lccrf_state_scan(*inputs, lengths, state=s["state"], saved=saved)
    g = crf.lccrf_state_scan_grad(s["dout"], *inputs, lengths, state=s["state"], saved=saved)
    grads = {"out": out, "final": final, "dCm": g.dCm, "dBm": g.dBm, "dx": g.dx, "ddt": g.ddt, "ddt_bias": g.ddt_bias,
             "dA": g.dA, "dD": g.dD}
    if s["z"] is not None:
        grads["dz"] = g.dz
    if s["state"] is not None:
        grads["dstate"] = g.dstate
    return grads


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


def work(case):
    """Inputs inside the sequences read once, results written once.  A scan takes for every state a product and an exponential
    for the decay, three operations for the recursion and two for the output; its gradient eighteen more."""
    op, B, N, D = case["op"], case["B"], case["N"], case["D"]
    e = 4 if case["dtype"] == "f32" else 2
    n = B * N                                   # positions written
    m = n * 0.5 * (case["min_len"] + N) / N     # positions read
    if op == "embed":
        V = case["V"]
        rows = V * (1 - math.exp(-m / V)) if m < V else min(m, V)
        return {"bytes": 4.0 * n + e * D * (rows + n), "flops": m * D}
    if op == "embed_grad":
        return {"bytes": 4.0 * n + e * D * (m + case["V"]), "flops": 2.0 * m * D}
    if op.startswith("conv"):
        K = case["K"]
        state = e * B * (K - 1) * D
        bytes_ = e * D * (m + n) + state * (2 if case["carry"] or op == "conv_step" else 1) + 4.0 * D * (K + 1)
        flops = m * D * (2.0 * K + 5)
        if op == "conv_train":
            bytes_ += e * D * (m + n) + 4.0 * D * (K + 1) + (state if case["carry"] else 0)
            flops += m * D * (4.0 * K + 10)
        return {"bytes": bytes_, "flops": flops}
    S, G, z = case["S"], case["G"], int(case["gate"])
    state = 4.0 * B * D * S
    bytes_ = e * (m * D * (2 + z) + n * D + 2 * m * G * S) + state * (2 if case["carry"] or op == "scan_step" else 1)
    bytes_ += 4.0 * D * (S + 2)
    flops = m * D * (7.0 * S + 12)
    if op == "scan_train":
        bytes_ += e * (m * D + n * D * (2 + z) + 2 * n * G * S) + 4.0 * D * (S + 2) + (state if case["carry"] else 0)
        flops += m * D * (18.0 * S + 20)
    return {"bytes": bytes_, "flops": flops}


# ---- the same values in 64 bits, position by position ---------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op, B, N, D = case["op"], case["B"], case["N"], case["D"]
    if op == "embed":
        table = torch.cat([s["table"].double(), torch.zeros(1, D, dtype=torch.float64, device=DEVICE)])
        return table[s["ids"].long()] * s["scale"]
    if op == "embed_grad":
        ids, rows = s["ids"].flatten().long(), s["dout"].flatten(0, 1).double() * s["scale"]
        out = torch.zeros(s["V"], D, dtype=torch.float64, device=DEVICE)
        return out.index_put_((ids[ids >= 0],), rows[ids >= 0], accumulate=True)
    lens = torch.full((B,), N, device=DEVICE) if s["lengths"] is None else s["lengths"].long()
    silu = lambda v: v / (1 + torch.exp(-v))  # noqa: E731
    dsilu = lambda v: (1 + torch.exp(-v) * (1 + v)) / (1 + torch.exp(-v)) ** 2  # noqa: E731
    if op.startswith("conv"):
        return _exact_conv(case, s, lens, silu, dsilu)
    return _exact_scan(case, s, lens, silu, dsilu)


def _exact_conv(case, s, lens, silu, dsilu):
    op, B, N, D, K = case["op"], case["B"], case["N"], case["D"], case["K"]
    w, bias = s["weight"].double(), s["bias"].double()
    x = (s["x"][:, None] if op == "conv_step" else s["x"]).double()
    rows = torch.zeros(B, K - 1 + N, D, dtype=torch.float64, device=DEVICE)
    if s["state"] is not None:
        rows[:, : K - 1] = s["state"].double()
    at = torch.arange(N, device=DEVICE)
    on = (at[None, :] < lens[:, None]).double()[..., None]
    rows[:, K - 1:] = x * on
    pre = bias.expand(B, N, D).clone()
    for k in range(K):
        pre += rows[:, k: k + N] * w[:, k]
    out = silu(pre) * on
    final = torch.stack([rows[torch.arange(B, device=DEVICE), lens + k] for k in range(K - 1)], 1)
    if op == "conv_step":
        return out[:, 0], final
    if op == "conv":
        return out, final
    dpre = s["dout"].double() * dsilu(pre) * on
    drows, dweight = torch.zeros_like(rows), torch.zeros_like(w)
    for k in range(K):
        drows[:, k: k + N] += dpre * w[:, k]
        dweight[:, k] = (dpre * rows[:, k: k + N]).sum((0, 1))
    grads = {"out": out, "final": final, "dx": drows[:, K - 1:], "dweight": dweight, "dbias": dpre.sum((0, 1))}
    if s["state"] is not None:
        grads["dstate"] = drows[:, : K - 1]
    return grads


def _exact_scan(case, s, lens, silu, dsilu):
    op, B, N, D, S, G = (case[k] for k in ("op", "B", "N", "D", "S", "G"))
    one = op == "scan_step"
    get = lambda k: (s[k][:, None] if one else s[k]).double()  # noqa: E731
    x, v, Bm, Cm = get("x"), get("dt") + s["dt_bias"].double(), get("Bm"), get("Cm")
    z = None if s["z"] is None else get("z")
    A, skip = s["A"].double(), s["D"].double()
    step = torch.logaddexp(v, torch.zeros_like(v))
    of = torch.arange(D, device=DEVICE) // (D // G)  # the group of a channel
    h = torch.zeros(B, D, S, dtype=torch.float64, device=DEVICE) if s["state"] is None else s["state"].double()
    train = op == "scan_train"
    y, states = torch.empty_like(x), [h]
    for l in range(N):
        new = torch.exp(step[:, l, :, None] * A) * h + (step[:, l] * x[:, l])[..., None] * Bm[:, l, of]
        h = torch.where((lens > l)[:, None, None], new, h)
        y[:, l] = (h * Cm[:, l, of]).sum(-1) + skip * x[:, l]
        if train:
            states.append(h)
    on = (torch.arange(N, device=DEVICE)[None, :] < lens[:, None])[..., None]
    out = torch.where(on, y if z is None else y * silu(z), 0.0)
    if one:
        return out[:, 0], h
    if not train:
        return out, h
    dout = torch.where(on, s["dout"].double(), 0.0)
    dy = dout if z is None else dout * silu(z)
    grads = {"out": out, "final": h}
    if z is not None:
        grads["dz"] = dout * y * dsilu(z)
    dA, dx, dv = torch.zeros_like(A), torch.zeros_like(x), torch.zeros_like(x)
    dBm, dCm = torch.zeros_like(Bm), torch.zeros_like(Cm)
    carry = torch.zeros_like(h)
    for l in range(N - 1, -1, -1):
        alive = (lens > l)[:, None, None]
        a = torch.exp(step[:, l, :, None] * A)
        dh = torch.where(alive, carry + dy[:, l, :, None] * Cm[:, l, of], 0.0)
        dCm[:, l] = (dy[:, l, :, None] * states[l + 1]).view(B, G, D // G, S).sum(2)
        dBm[:, l] = (dh * (step[:, l] * x[:, l])[..., None]).view(B, G, D // G, S).sum(2)
        dput = (dh * Bm[:, l, of]).sum(-1)
        dlog = dh * a * states[l]
        dx[:, l] = dput * step[:, l] + skip * dy[:, l]
        dv[:, l] = (dput * x[:, l] + (dlog * A).sum(-1)) / (1 + torch.exp(-v[:, l]))
        dA += (dlog * step[:, l, :, None]).sum(0)
        carry = torch.where(alive, dh * a, carry)
    grads |= {"dCm": dCm, "dBm": dBm, "dx": dx, "ddt": dv, "ddt_bias": dv.sum((0, 1)), "dA": dA,
              "dD": (dy * x).sum((0, 1))}
    if s["state"] is not None:
        grads["dstate"] = carry
    return grads
