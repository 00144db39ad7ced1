"""The encoder's operators in 64 bits on the CPU, from their formulas, position by position; test infrastructure only.

Every function takes ``absolute``: the same sums with the absolute value of every product, which bounds how far rounded
arithmetic can be from the exact result.
"""
import torch


def f64(t):
    return None if t is None else t.detach().double().cpu()


def lengths_of(lengths, B, N):
    return torch.full((B,), N) if lengths is None else lengths.cpu().long().clamp(0, N)


def silu(v):
    return v * torch.sigmoid(v)


def dsilu(v):
    g = torch.sigmoid(v)
    return g * (1 + v * (1 - g))


def embed(table, ids, scale):
    table, ids = f64(table), ids.cpu().long()
    inside = (ids >= 0) & (ids < table.shape[0])
    return torch.where(inside[..., None], table[ids.clamp(0, table.shape[0] - 1)] * scale, 0.0)


def embed_grad(dout, ids, V, scale, absolute=False):
    dout, ids = f64(dout).flatten(0, -2), ids.cpu().long().flatten()
    if absolute:
        dout, scale = dout.abs(), abs(scale)
    keep = (ids >= 0) & (ids < V)
    return torch.zeros(V, dout.shape[1], dtype=torch.float64).index_add_(0, ids[keep], dout[keep]) * scale


def conv(x, weight, bias, lengths, state, dout=None, absolute=False):
    """A dict: out, final, and with dout the gradients.  absolute: of pre, then the factors of the gradient."""
    x, w, dout = f64(x), f64(weight), f64(dout)
    (B, N, D), K = x.shape, w.shape[1]
    b = torch.zeros(D, dtype=torch.float64) if bias is None else f64(bias)
    st = torch.zeros(B, K - 1, D, dtype=torch.float64) if state is None else f64(state)
    lens = lengths_of(lengths, B, N)
    on = (torch.arange(N)[None] < lens[:, None])[..., None]
    rows = torch.cat([st, torch.where(on, x, 0.0)], 1)
    exact = sum(rows[:, k:k + N] * w[:, k] for k in range(K)) + b
    if absolute:
        rows, w, b = rows.abs(), w.abs(), b.abs()
        dout = None if dout is None else dout.abs()
    pre = sum(rows[:, k:k + N] * w[:, k] for k in range(K)) + b
    res = {"pre": pre, "out": torch.where(on, silu(exact), 0.0)}
    res["final"] = torch.stack([rows[i, int(lens[i]):int(lens[i]) + K - 1] for i in range(B)])
    if dout is None:
        return res
    slope = torch.full_like(exact, 1.1) if absolute else dsilu(exact)  # |dsilu| < 1.1, and where it is near 0 its error is not
    dpre = torch.where(on, dout * slope, 0.0)
    drows = torch.zeros_like(rows)
    for k in range(K):
        drows[:, k:k + N] += dpre * w[:, k]
    res["dx"], res["dstate"] = torch.where(on, drows[:, K - 1:], 0.0), drows[:, :K - 1]
    res["dweight"] = torch.stack([(dpre * rows[:, k:k + N]).sum((0, 1)) for k in range(K)], 1)
    res["dbias"] = dpre.sum((0, 1))
    return res


def scan(x, dt, A, Bm, Cm, D, z, dt_bias, lengths, state, dout=None, absolute=False):
    x, dt, A, Bm, Cm, D, z, dt_bias, state, dout = (f64(t) for t in (x, dt, A, Bm, Cm, D, z, dt_bias, state, dout))
    B, N, W = x.shape
    G, S = Bm.shape[2:]
    of = torch.arange(W) // (W // G)
    lens = lengths_of(lengths, B, N)
    on = (torch.arange(N)[None] < lens[:, None])[..., None]
    # nothing past the end takes part
    x, dt = torch.where(on, x, 0.0), torch.where(on, dt, 0.0)
    Bm, Cm = torch.where(on[..., None], Bm, 0.0), torch.where(on[..., None], Cm, 0.0)
    z = None if z is None else torch.where(on, z, 0.0)
    v = dt + (0.0 if dt_bias is None else dt_bias)
    step = torch.where(on, torch.logaddexp(v, torch.zeros_like(v)), 0.0)
    skip = torch.zeros(W, dtype=torch.float64) if D is None else D
    back_A, gate, gate_slope = A, None, None
    if z is not None:
        gate, gate_slope = silu(z), dsilu(z)
    if absolute:
        x, Bm, Cm, skip, back_A = x.abs(), Bm.abs(), Cm.abs(), skip.abs(), A.abs()
        state = None if state is None else state.abs()
        dout = None if dout is None else dout.abs()
        if z is not None:
            gate, gate_slope = gate.abs(), torch.full_like(gate, 1.1)
    h = torch.zeros(B, W, S, dtype=torch.float64) if state is None else state.clone()
    hs, y = [h], torch.zeros_like(x)
    for l in range(N):
        new = torch.exp(step[:, l, :, None] * A) * h + (step[:, l] * x[:, l])[..., None] * Bm[:, l, of]
        h = torch.where(on[:, l, :, None], new, h)
        hs.append(h)
        y[:, l] = (h * Cm[:, l, of]).sum(-1) + skip * x[:, l]
    res = {"y": y, "out": torch.where(on, y if z is None else y * gate, 0.0), "final": h}
    if dout is None:
        return res
    dout = torch.where(on, dout, 0.0)
    dy = dout if z is None else dout * gate
    if z is not None:
        res["dz"] = dout * y * gate_slope
    carry = torch.zeros_like(h)
    dA, dx, dv = torch.zeros_like(A), torch.zeros_like(x), torch.zeros_like(x)
    dBm, dCm = torch.zeros_like(Bm), torch.zeros_like(Cm)
    for l in range(N - 1, -1, -1):
        alive = on[:, l, :, None]
        a = torch.exp(step[:, l, :, None] * A)
        dh = torch.where(alive, carry + dy[:, l, :, None] * Cm[:, l, of], 0.0)
        dCm[:, l] = (dy[:, l, :, None] * hs[l + 1]).view(B, G, W // G, S).sum(2)
        dBm[:, l] = (dh * (step[:, l] * x[:, l])[..., None]).view(B, G, W // G, S).sum(2)
        dput = (dh * Bm[:, l, of]).sum(-1)
        back = dh * a * hs[l]
        dx[:, l] = dput * step[:, l] + skip * dy[:, l]
        dv[:, l] = (dput * x[:, l] + (back * back_A).sum(-1)) * torch.sigmoid(v[:, l])
        dA += (back * step[:, l, :, None]).sum(0)
        carry = torch.where(alive, dh * a, carry)
    res |= {"dCm": dCm, "dBm": dBm, "dx": dx, "ddt": dv, "ddt_bias": dv.sum((0, 1)), "dA": dA, "dD": (dy * x).sum((0, 1)), "dstate": carry}
    return res
