"""A tagger: the library's encoder in front of its chain, trained, decoded and run token by token.

    ids -> embedding -> projection (x, z) -> short convolution -> projection (dt, Bm, Cm) -> state space scan, gated by z
        -> projection -> emissions -> linear-chain CRF with transitions ``trans``

The projections are plain matrix products; everything else runs in the library's kernels, forwards (``lccrf_embed``, ``lccrf_conv``,
``lccrf_state_scan``, ``lccrf_marginals_structured``, ``lccrf_argmax_structured``), backwards (the ``_grad`` calls, by hand, in reverse
order) and for single tokens (``lccrf_conv_step``, ``lccrf_state_step``).  ``python -m paper_2308_03291_amd.tagger`` trains one on a
synthetic language in which a word's tag depends on an earlier word, and prints loss, accuracy and what a stream of tokens gives.

``Student`` is a smaller one, which learns from a tagger's largest emissions besides the tags (``--student`` trains it after the tagger):

    ids -> embedding -> projection (x, z) -> short convolution -> projection (f, g) -> gated linear recurrence, gated by z
        -> group norm with its activation, every position by itself -> projection -> emissions -> chain
"""
from __future__ import annotations

import argparse
import math
from typing import Dict, Optional

import torch

from . import binding as crf


def _mm(a: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
    """a [..., k] @ w [k, n] as one two-dimensional product."""
    return (a.reshape(-1, a.shape[-1]) @ w).view(*a.shape[:-1], w.shape[1])


class Tagger:
    """Parameters in float32 (``params``), activations in ``dtype``.  V words, T tags (at most 128), E channels a word, D channels
    and S states of the scan, G groups, K taps."""

    def __init__(self, V: int, T: int, E: int = 64, D: int = 128, S: int = 16, G: int = 1, K: int = 4, *, dtype=torch.float32, device="cuda", seed: int = 0):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(shape, generator=g) * scale).to(device)

        step = torch.exp(torch.rand(D, generator=g) * math.log(100.0) + math.log(1e-3))
        self.params: Dict[str, torch.Tensor] = {
            "table": normal(V, E, scale=1.0 / math.sqrt(E)), "w_in": normal(E, 2 * D, scale=E ** -0.5),
            "conv_w": normal(D, K, scale=K ** -0.5), "conv_b": torch.zeros(D, device=device),
            "w_x": normal(D, D + 2 * G * S, scale=0.5 * D ** -0.5), "dt_bias": (step + torch.log(-torch.expm1(-step))).to(device),
            "A_log": torch.log(torch.arange(1, S + 1, dtype=torch.float32)).repeat(D, 1).to(device), "skip": torch.ones(D, device=device),
            "w_out": normal(D, T, scale=D ** -0.5), "trans": torch.zeros(T, T, device=device)}
        self.V, self.T, self.E, self.D, self.S, self.G, self.K, self.dtype, self.device = V, T, E, D, S, G, K, dtype, device

    def _w(self, name: str) -> torch.Tensor:
        return self.params[name].to(self.dtype)

    def forward(self, ids: torch.Tensor, lengths: Optional[torch.Tensor] = None, *, train: bool = False) -> Dict[str, torch.Tensor]:
        """Emissions [B, N, T] float32 (``emit``) of ids int32 [B, N], with what the way back needs."""
        p, D, GS, (B, N) = self.params, self.D, self.G * self.S, ids.shape
        a = {"ids": ids, "lengths": lengths}
        a["e"] = crf.lccrf_embed(self._w("table"), ids, scale=math.sqrt(self.E))
        a["xz"] = _mm(a["e"], self._w("w_in"))
        a["u"], _ = crf.lccrf_conv(a["xz"][..., :D], p["conv_w"], p["conv_b"], lengths)
        a["proj"] = _mm(a["u"], self._w("w_x"))
        a["inputs"] = self._scan_inputs(a["u"], a["proj"], a["xz"][..., D:])
        a["saved"] = crf.state_scan_saved(a["u"], p["A_log"]) if train else None
        a["y"], _ = crf.lccrf_state_scan(*a["inputs"], lengths, saved=a["saved"])
        a["emit"] = _mm(a["y"], self._w("w_out")).float()
        return a

    def _scan_inputs(self, u, proj, z):
        """x, dt, A, Bm, Cm, D, z, dt_bias: dt and the vectors are pieces of one projection's rows."""
        p, D, GS = self.params, self.D, self.G * self.S
        vectors = (*u.shape[:-1], self.G, self.S)
        return (u, proj[..., :D], -torch.exp(p["A_log"]), proj[..., D:D + GS].view(vectors), proj[..., D + GS:].view(vectors), p["skip"], z, p["dt_bias"])

    def _through_chain(self, emit, tags, lengths):
        """The mean negative log-likelihood a sequence, its gradient by emissions and transitions, float32."""
        trans, (B, N) = self.params["trans"], tags.shape
        logZ, mu = crf.lccrf_marginals_structured(emit, trans, lengths)
        inside = torch.ones(B, N, dtype=torch.bool, device=tags.device) if lengths is None else torch.arange(N, device=tags.device)[None] < lengths[:, None]
        y = tags.long().clamp(0, self.T - 1)
        before = torch.cat([torch.zeros_like(y[:, :1]), y[:, :-1]], 1)  # a chain starts from row 0 of the transitions
        score = torch.where(inside, emit.gather(2, y[..., None])[..., 0] + trans[before, y], 0.0).sum(1)
        loss = (logZ - score).mean()
        gold = torch.zeros_like(emit).scatter_(2, y[..., None], inside[..., None].float())
        demit = (mu.sum(2) - gold) / B
        return loss, demit, (mu.sum((0, 1)) - torch.zeros_like(trans).index_put_((before[inside], y[inside]), torch.ones((), device=tags.device), accumulate=True)) / B

    def loss_and_gradients(self, ids: torch.Tensor, tags: torch.Tensor, lengths: Optional[torch.Tensor] = None):
        """(the mean negative log-likelihood a sequence of tags int32 [B, N], its gradient by every parameter)."""
        p, D = self.params, self.D
        a = self.forward(ids, lengths, train=True)
        loss, demit, dtrans = self._through_chain(a["emit"], tags, lengths)
        demit = demit.to(self.dtype)
        grads = {"trans": dtrans}
        grads["w_out"] = a["y"].reshape(-1, D).t().float() @ demit.reshape(-1, self.T).float()
        g = crf.lccrf_state_scan_grad(_mm(demit, self._w("w_out").t()), *a["inputs"], lengths, saved=a["saved"])
        dproj = torch.cat([g.ddt, g.dBm.flatten(2), g.dCm.flatten(2)], 2)
        grads |= {"A_log": -g.dA * torch.exp(p["A_log"]), "skip": g.dD, "dt_bias": g.ddt_bias,
                  "w_x": a["u"].reshape(-1, D).t().float() @ dproj.reshape(-1, dproj.shape[2]).float()}
        du = g.dx + _mm(dproj, self._w("w_x").t())
        c = crf.lccrf_conv_grad(du, a["xz"][..., :D], p["conv_w"], p["conv_b"], lengths)
        dxz = torch.cat([c.dx, g.dz], 2)
        grads |= {"conv_w": c.dweight, "conv_b": c.dbias, "w_in": a["e"].reshape(-1, self.E).t().float() @ dxz.reshape(-1, 2 * D).float()}
        grads["table"] = crf.lccrf_embed_grad(_mm(dxz, self._w("w_in").t()), ids, self.V, scale=math.sqrt(self.E)).float()
        return loss, grads

    def train_step(self, ids, tags, lengths=None, lr: float = 0.5, **more) -> torch.Tensor:
        """One step of gradient descent, the gradient's norm cut off at 1."""
        loss, grads = self.loss_and_gradients(ids, tags, lengths, **more)
        norm = torch.sqrt(sum((v * v).sum() for v in grads.values()))
        for k, v in grads.items():
            self.params[k] -= lr * v / norm.clamp_min(1.0)
        return loss

    def decode(self, ids, lengths=None) -> torch.Tensor:
        """The most probable tags int32 [B, N], -1 past the lengths."""
        return crf.lccrf_argmax_structured(self.forward(ids, lengths)["emit"], self.params["trans"], lengths)[1]

    def stream(self, B: int) -> "Stream":
        return Stream(self, B)


class Stream:
    """B streams of tokens: ``feed`` takes one id a stream and gives that position's emissions."""

    def __init__(self, tagger: Tagger, B: int):
        self.tagger = tagger
        self.conv = torch.zeros(B, tagger.K - 1, tagger.D, dtype=tagger.dtype, device=tagger.device)
        self.state = torch.zeros(B, tagger.D, tagger.S, device=tagger.device)

    def feed(self, ids: torch.Tensor) -> torch.Tensor:
        t = self.tagger
        xz = crf.lccrf_embed(t._w("table"), ids, scale=math.sqrt(t.E)) @ t._w("w_in")
        u = crf.lccrf_conv_step(xz[:, :t.D], t.params["conv_w"], t.params["conv_b"], self.conv)
        y = crf.lccrf_state_step(*t._scan_inputs(u, u @ t._w("w_x"), xz[:, t.D:]), self.state)
        return (y @ t._w("w_out")).float()


def top_emissions(emit: torch.Tensor, K: int, lengths: Optional[torch.Tensor] = None):
    """(tags int32 [B, N, K], emissions float32 [B, N, K]): a teacher's K largest of every position, no tag (-1) past the lengths."""
    values, tags = torch.topk(emit, K, -1)
    tags = tags.to(torch.int32)
    if lengths is not None:
        tags.masked_fill_((torch.arange(emit.shape[1], device=emit.device)[None] >= lengths[:, None])[..., None], -1)
    return tags, values


class Student(Tagger):
    """A tagger with one state a channel: parameters and manner of a ``Tagger``, ``groups`` of its channels normalised together."""

    def __init__(self, V: int, T: int, E: int = 32, D: int = 64, groups: int = 4, K: int = 4, *, dtype=torch.float32, device="cuda", seed: int = 0):
        super().__init__(V, T, E, D, 1, 1, K, dtype=dtype, device=device, seed=seed)
        g = torch.Generator().manual_seed(seed + 1)
        for name in ("w_x", "dt_bias", "A_log", "skip"):
            del self.params[name]
        # decays between 0.9 and 0.999 a position where their gate is wide open
        c = -torch.log(0.9 + 0.099 * torch.rand(D, generator=g)) / 8.0
        self.params |= {"w_g": (torch.randn(D, 2 * D, generator=g) * D ** -0.5).to(device), "decay": torch.log(torch.expm1(c)).to(device),
                        "f_bias": torch.zeros(D, device=device), "g_bias": torch.zeros(D, device=device), "norm_w": torch.ones(D, device=device),
                        "norm_b": torch.zeros(D, device=device)}
        self.groups = groups

    def _norm(self) -> Dict:
        return {"groups": self.groups, "per_position": True}

    def _recurrence_inputs(self, u, gates, z):
        p, D = self.params, self.D
        return u, gates[..., :D], gates[..., D:], p["decay"], z, p["f_bias"], p["g_bias"]

    def forward(self, ids, lengths=None, *, train: bool = False) -> Dict[str, torch.Tensor]:
        p, D = self.params, self.D
        a = {"ids": ids, "lengths": lengths}
        a["e"] = crf.lccrf_embed(self._w("table"), ids, scale=math.sqrt(self.E))
        a["xz"] = _mm(a["e"], self._w("w_in"))
        a["u"], _ = crf.lccrf_conv(a["xz"][..., :D], p["conv_w"], p["conv_b"], lengths)
        a["inputs"] = self._recurrence_inputs(a["u"], _mm(a["u"], self._w("w_g")), a["xz"][..., D:])
        a["saved"] = crf.recurrence_saved(a["u"]) if train else None
        a["h"], _ = crf.lccrf_recurrence(*a["inputs"], lengths, saved=a["saved"])
        a["stats"] = crf.group_norm_stats(a["h"], self.groups, per_position=True) if train else None
        a["y"] = crf.lccrf_group_norm(a["h"], p["norm_w"], p["norm_b"], lengths, **self._norm(), stats=a["stats"])
        a["emit"] = _mm(a["y"], self._w("w_out")).float()
        return a

    def loss_and_gradients(self, ids, tags, lengths=None, *, teacher=None, share: float = 0.5, temperature: float = 2.0):
        """(the loss, its gradient by every parameter).  ``teacher``: (tags, emissions) of ``top_emissions``; then ``share`` of the loss is the mean distance a
        sequence of the student's emissions from those, summed over its positions within the lengths (whether the teacher's tags are masked past them or
        not), the rest the tags' negative log-likelihood."""
        p, D = self.params, self.D
        a = self.forward(ids, lengths, train=True)
        loss, demit, dtrans = self._through_chain(a["emit"], tags, lengths)
        grads = {"trans": dtrans}
        if teacher is not None:
            weights = torch.full(ids.shape, share / ids.shape[0], device=ids.device)
            if lengths is not None:
                weights.masked_fill_(torch.arange(ids.shape[1], device=ids.device)[None] >= lengths[:, None], 0.0)
            far = torch.empty_like(weights)
            dfar = crf.lccrf_distill_grad(weights, a["emit"], *teacher, temperature=temperature, loss=far)
            loss = (1 - share) * loss + (weights * far).sum()
            demit = (1 - share) * demit + dfar
            grads["trans"] = (1 - share) * dtrans
        demit = demit.to(self.dtype)
        grads["w_out"] = a["y"].reshape(-1, D).t().float() @ demit.reshape(-1, self.T).float()
        n = crf.lccrf_group_norm_grad(_mm(demit, self._w("w_out").t()), a["h"], p["norm_w"], p["norm_b"], lengths, **self._norm(), stats=a["stats"])
        g = crf.lccrf_recurrence_grad(n.dx, *a["inputs"], lengths, saved=a["saved"])
        dgates = torch.cat([g.df, g.dg], 2)
        grads |= {"norm_w": n.dweight, "norm_b": n.dbias, "decay": g.ddecay, "f_bias": g.df_bias, "g_bias": g.dg_bias,
                  "w_g": a["u"].reshape(-1, D).t().float() @ dgates.reshape(-1, 2 * D).float()}
        c = crf.lccrf_conv_grad(g.dx + _mm(dgates, self._w("w_g").t()), a["xz"][..., :D], p["conv_w"], p["conv_b"], lengths)
        dxz = torch.cat([c.dx, g.dz], 2)
        grads |= {"conv_w": c.dweight, "conv_b": c.dbias, "w_in": a["e"].reshape(-1, self.E).t().float() @ dxz.reshape(-1, 2 * D).float()}
        grads["table"] = crf.lccrf_embed_grad(_mm(dxz, self._w("w_in").t()), ids, self.V, scale=math.sqrt(self.E)).float()
        return loss, grads

    def stream(self, B: int) -> "StudentStream":
        return StudentStream(self, B)


class StudentStream:
    """B streams of tokens through a student: ``feed`` takes one id a stream and gives that position's emissions."""

    def __init__(self, student: Student, B: int):
        self.student = student
        self.conv = torch.zeros(B, student.K - 1, student.D, dtype=student.dtype, device=student.device)
        self.state = torch.zeros(B, student.D, device=student.device)

    def feed(self, ids: torch.Tensor) -> torch.Tensor:
        t, p = self.student, self.student.params
        xz = crf.lccrf_embed(t._w("table"), ids, scale=math.sqrt(t.E)) @ t._w("w_in")
        u = crf.lccrf_conv_step(xz[:, :t.D], p["conv_w"], p["conv_b"], self.conv)
        h = crf.lccrf_recurrence_step(*t._recurrence_inputs(u, u @ t._w("w_g"), xz[:, t.D:]), self.state)
        y = crf.lccrf_group_norm(h[:, None], p["norm_w"], p["norm_b"], **t._norm())[:, 0]
        return (y @ t._w("w_out")).float()


def language(B: int, N: int, V: int, T: int, device="cuda", seed: int = 0):
    """Sentences whose tag at a position is that of the last word out of the first T, and their lengths: to be remembered, not read off."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.where(torch.rand(B, N, generator=g) < 0.2, torch.randint(0, T, (B, N), generator=g), torch.randint(T, V, (B, N), generator=g))
    ids[:, 0] = torch.randint(0, T, (B,), generator=g)
    at = torch.where(ids < T, torch.arange(N)[None], 0).cummax(1).values
    lengths = torch.randint(N // 2, N + 1, (B,), generator=g)
    past = torch.arange(N)[None] >= lengths[:, None]
    tags = ids.gather(1, at).masked_fill(past, -1)
    return tuple(v.to(torch.int32).to(device) for v in (ids.masked_fill(past, -1), tags, lengths))


def _report(tagger: Tagger, V: int, N: int, T: int) -> None:
    ids, tags, lengths = language(64, N, V, T, seed=10 ** 6)
    right = tagger.decode(ids, lengths) == tags
    print(f"tags right on new sentences: {float(right[tags >= 0].float().mean()):.4f}")
    stream, emit = tagger.stream(64), tagger.forward(ids, lengths)["emit"]
    alive = torch.arange(N, device=ids.device)[None] < lengths[:, None]
    off = max(float((stream.feed(ids[:, l].contiguous()) - emit[:, l])[alive[:, l]].abs().max()) for l in range(int(lengths.min())))
    print(f"emissions token by token are off by {off:.2e} at most")


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--student", action="store_true", help="train a smaller tagger from this one's largest emissions, too")
    args = ap.parse_args(argv)
    V, T, N = 200, 8, 64
    dtype = torch.float32 if args.dtype == "f32" else torch.bfloat16
    tagger = Tagger(V, T, dtype=dtype)
    for k in range(args.steps):
        loss = tagger.train_step(*language(64, N, V, T, seed=k))
        if k % 50 == 0 or k == args.steps - 1:
            print(f"step {k}: negative log-likelihood {float(loss):.3f} a sentence", flush=True)
    _report(tagger, V, N, T)
    if not args.student:
        return
    student = Student(V, T, dtype=dtype)
    for k in range(args.steps):
        ids, tags, lengths = language(64, N, V, T, seed=args.steps + k)
        teacher = top_emissions(tagger.forward(ids, lengths)["emit"], 4, lengths)
        loss = student.train_step(ids, tags, lengths, teacher=teacher)
        if k % 50 == 0 or k == args.steps - 1:
            print(f"student, step {k}: loss {float(loss):.3f} a sentence", flush=True)
    _report(student, V, N, T)


if __name__ == "__main__":
    main()
