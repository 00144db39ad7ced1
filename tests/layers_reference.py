"""The layers of include/lccrf_layers.h in 64 bits on the CPU, from their formulas; test infrastructure only.

Every function gives pairs (value, error): how far arithmetic in float may be from the value, in units of U = 2^-24 (half a step next to 1) before
the last rounding.  The errors follow the formulas: a product has those of its factors and one of its own, an exponential the absolute
error of its argument and two (the hardware's is off by a whole step), a reciprocal or a root two, a sum those of its terms and one for
every addition that a term goes through.
"""
import math

import torch

from encoder_reference import dsilu, f64, lengths_of, silu

U = 2.0 ** -24


def _sigmoid(v):
    """s(v) and its relative error: the argument rounded, times log2(e), exponential, sum, reciprocal."""
    return torch.sigmoid(v), 2 * v.abs() + 7


def _dsilu_error(v):
    """Of g (1 + v (1 - g)), absolutely."""
    g, r = _sigmoid(v)
    return g * (1 + v.abs()) * (2 * r + 6)


def recurrence(x, f, g, decay, z=None, f_bias=None, g_bias=None, lengths=None, rate=8.0, state=None, dout=None):
    """{name: (value, error)}: out, final and, with dout, the gradients."""
    x, f, g, lam, z, dout = f64(x), f64(f), f64(g), f64(decay), f64(z), f64(dout)
    f = f if f_bias is None else f + f64(f_bias)
    g = g if g_bias is None else g + f64(g_bias)
    B, N, D = x.shape
    lens = lengths_of(lengths, B, N)
    on = (torch.arange(N)[None] < lens[:, None])[..., None]
    soft = torch.nn.functional.softplus(lam)
    opened, r_o = _sigmoid(f)
    u = -rate * soft * opened
    r_u = r_o + 6
    a, m = torch.exp(u), torch.sqrt(-torch.expm1(2 * u))
    r_a, r_m = u.abs() * (r_u + 2) + 2, r_u / 2 + 12
    take, r_t = _sigmoid(g)
    one = lambda v: torch.where(on, v, 0.0)  # noqa: E731
    b = one(m * take * x)
    # Exponentials below 2^-126 are 0: the open gate and log(1 + exp(decay)) are off by as much, u by rate (1 + soft) 2^-126, and a root of something
    # off by d by no more than sqrt(2 d): |sqrt(1 - exp(2 u)) - sqrt(1 - exp(2 u - 2 d))| <= sqrt(2 d); so is u / m, which is at most m / 2 in size
    # (-u <= -expm1(2 u) for small u).  4e-19 at a rate of 8.
    e_root = torch.sqrt(2 * rate * (1 + soft) * 2.0 ** -126) / U
    e_b = b.abs() * (r_m + r_t + 3) + one(take * x.abs() * e_root)

    def along(values, errors, decays, r_decays, first, first_error, order):
        """v = a v + value over the positions in order; a position's decay is that towards it.  (values, sums of absolute values, errors)"""
        v, size, err = first.clone(), first.abs(), first_error.clone()
        at_v, at_size, at_err = torch.zeros(B, N, D, dtype=torch.float64), torch.zeros(B, N, D, dtype=torch.float64), torch.zeros(B, N, D, dtype=torch.float64)
        for l in order:
            alive = (lens > l)[:, None]
            k = decays[:, l]
            new_size = k * size + values[:, l].abs()
            new_err = k * err + k * size * (r_decays[:, l] + 4) + errors[:, l] + new_size
            v = torch.where(alive, k * v + values[:, l], v)
            size, err = torch.where(alive, new_size, size), torch.where(alive, new_err, err)
            at_v[:, l], at_size[:, l], at_err[:, l] = v, size, err
        return at_v, at_size, at_err, v, err

    zero = torch.zeros(B, D, dtype=torch.float64)
    start = zero if state is None else f64(state)
    h, h_size, h_err, final, final_err = along(b, e_b, a, r_a, start, zero, range(N))
    gate, r_gate = (torch.ones_like(h), torch.zeros_like(h)) if z is None else (silu(z), 2 * z.abs() + 9)
    res = {"out": (one(h * gate), one(h_err * gate.abs() + h_size * gate.abs() * r_gate)), "final": (final, final_err)}
    if dout is None:
        return res
    dout = one(dout)
    dy, e_dy = dout * gate, (dout * gate).abs() * r_gate
    after = torch.cat([a[:, 1:], torch.ones(B, 1, D, dtype=torch.float64)], 1)
    r_after = torch.cat([r_a[:, 1:], torch.zeros(B, 1, D, dtype=torch.float64)], 1)
    dh, size, e_dh, _, _ = along(dy, e_dy, after, r_after, zero, zero, range(N - 1, -1, -1))
    dh, size, e_dh = one(dh), one(size), one(e_dh)
    dx, e_dx = dh * m * take, (e_dh + size * (r_m + r_t + 3)) * m * take + size * e_root * take
    res["dx"] = dx, e_dx
    res["dg"] = dx * x * (1 - take), (e_dx * (1 - take) + size * m * take * (take * r_t + 4)) * x.abs()
    before = torch.cat([start[:, None], h[:, :-1]], 1)
    before_size, before_err = torch.cat([start.abs()[:, None], h_size[:, :-1]], 1), torch.cat([zero[:, None], h_err[:, :-1]], 1)
    ratio = torch.where(m > 0, u / m, 0.0)
    one_term, other = before_size * a * u.abs(), (take * x * a * a * ratio).abs()
    dlog = dh * (before * a * u - take * x * a * a * ratio)
    e_dlog = e_dh * (one_term + other) + size * (before_err * a * u.abs() + one_term * (r_a + r_u + 5) + other * (r_t + 2 * r_a + r_u + r_m + 16) + take * x.abs() * e_root)
    dlog_size = size * (one_term + other)
    df, e_df = dlog * (1 - opened), e_dlog * (1 - opened) + dlog_size * (opened * r_o + 4)
    res["df"] = df, e_df
    depth = N / 2 + B + 64  # additions that a term goes through
    slope = torch.where(lam < -30, 1.0, torch.sigmoid(lam) / soft)
    total = lambda v, e, v_size: (one(v).sum((0, 1)), (one(e) + one(v_size) * depth).sum((0, 1)))  # noqa: E731
    s, e = total(dlog, e_dlog, dlog_size)
    res["ddecay"] = s * slope, (e + one(dlog_size).sum((0, 1)) * (2 * lam.abs() + 16)) * slope
    res["df_bias"] = total(df, e_df, dlog_size * (1 - opened))
    res["dg_bias"] = total(res["dg"][0], res["dg"][1], size * m * take * x.abs() * (1 - take))
    if z is not None:
        slope = dsilu(z)
        res["dz"] = dout * h * slope, dout.abs() * (h_err * slope.abs() + h_size * (_dsilu_error(z) + 3 * slope.abs()))
    if state is not None:
        alive = (lens > 0)[:, None]
        res["dstate"] = torch.where(alive, a[:, 0] * dh[:, 0], 0.0), torch.where(alive, a[:, 0] * (e_dh[:, 0] + size[:, 0] * (r_a[:, 0] + 2)), 0.0)
    return res


def group_norm(x, weight, bias, lengths, groups, eps, act, alone, dout=None):
    """{name: (value, error)}: out, stats and, with dout, dx, dweight, dbias."""
    x, dout = f64(x), f64(dout)
    B, N, D = x.shape
    C = D // groups
    lens = lengths_of(lengths, B, N)
    on = (torch.arange(N)[None] < lens[:, None]).view(B, N, 1, 1)
    w = torch.ones(groups, C, dtype=torch.float64) if weight is None else f64(weight).view(groups, C)
    bias = torch.zeros(groups, C, dtype=torch.float64) if bias is None else f64(bias).view(groups, C)
    over = (3,) if alone else (1, 3)
    x = torch.where(on, x.view(B, N, groups, C), 0.0)
    on = on.expand_as(x)
    count = on.double().sum(over, keepdim=True)
    n = count.clamp_min(1)
    mean_of = lambda v: torch.where(on, v, 0.0).sum(over, keepdim=True) / n  # noqa: E731
    mean = mean_of(x)
    away = torch.where(on, x - mean, 0.0)
    var = (away * away).sum(over, keepdim=True) / n
    rstd = 1 / torch.sqrt(var + eps)
    # a mean of means: every joining rounds the mean once, and a value goes through no more than these additions and joinings
    joins = 48 + 6 * math.log2(float(n.max()) + 2) + float(n.max()) / 4096
    e_mean = joins * x.abs().amax(over, keepdim=True)
    r_rstd = (joins + 8) * var / (var + eps) + e_mean ** 2 * U / (var + eps) + 4
    hat = away * rstd
    e_hat = (e_mean + away.abs()) * rstd + hat.abs() * (r_rstd + 2)
    y = hat * w + bias
    e_y = e_hat * w.abs() + (hat * w).abs() + y.abs()
    out, e_out = (silu(y), 1.1 * e_y + silu(y).abs() * (2 * y.abs() + 9)) if act else (y, e_y)
    flat = lambda v: torch.where(on, v, 0.0).reshape(B, N, D)  # noqa: E731
    res = {"out": (flat(out), flat(e_out))}
    some = count > 0
    stats = torch.where(some, torch.cat([mean, rstd], 3), 0.0)
    e_stats = torch.cat([e_mean, rstd * r_rstd], 3)
    res["stats"] = (stats, e_stats) if alone else (stats[:, 0], e_stats[:, 0])
    if dout is None:
        return res
    dout = torch.where(on, dout.view_as(x), 0.0)
    dy, e_dy = (dout * dsilu(y), dout.abs() * (0.5 * e_y + _dsilu_error(y) + 2)) if act else (dout, torch.zeros_like(dout))
    dhat, e_dhat = dy * w, (e_dy + dy.abs()) * w.abs()
    s1, s2 = mean_of(dhat), mean_of(dhat * hat)
    e_s1 = mean_of(e_dhat + joins * dhat.abs())
    e_s2 = mean_of(e_dhat * hat.abs() + e_hat * dhat.abs() + (joins + 2) * (dhat * hat).abs())
    dx = rstd * (dhat - s1 - hat * s2)
    size = rstd * (dhat.abs() + s1.abs() + (hat * s2).abs())
    res["dx"] = flat(dx), flat(rstd * (e_dhat + e_s1 + hat.abs() * e_s2 + s2.abs() * e_hat) + size * (r_rstd + 6))
    depth = B * N / 16 + 64
    res["dweight"] = ((dy * hat).sum((0, 1)).flatten(), (e_dy * hat.abs() + e_hat * dy.abs() + (depth + 2) * (dy * hat).abs()).sum((0, 1)).flatten())
    res["dbias"] = (dy.sum((0, 1)).flatten(), (e_dy + depth * dy.abs()).sum((0, 1)).flatten())
    return res


def distill(logits, ids, teacher, t, dloss=None, from_lse=False):
    """{name: (value, error)}: loss, lse and, with dloss, dlogits.  from_lse: the gradient takes lse as it was rounded to float."""
    V, K = logits.shape[-1], ids.shape[-1]
    lead = logits.shape[:-1]
    x, ids, v = f64(logits).reshape(-1, V), ids.cpu().long().reshape(-1, K), f64(teacher).reshape(-1, K)
    there = (ids >= 0) & (ids < V) & (v != -math.inf)
    some = there.any(-1)
    at = torch.where(there, ids, 0)
    v = torch.where(there, v, -math.inf)
    Mt = torch.where(some, v.amax(-1), 0.0)[:, None]
    e = torch.exp((v - Mt) / t)
    st = torch.where(some, e.sum(-1), 1.0)[:, None]
    q = e / st
    ahead = torch.where(there, v - Mt, 0.0)
    r_q = 4 * ahead.abs() / t + 12 + K / 16
    M = x.amax(-1, keepdim=True)
    behind = (x - M).clamp_min(-1e30)
    s = torch.exp(behind / t).sum(-1, keepdim=True)
    p = torch.exp(behind / t) / s
    r_each = torch.where(behind > -200 * t, 4 * behind.abs() / t, 0.0) + 4
    r_s = (p * r_each).sum(-1, keepdim=True) + 32 + V / 2048
    lse = M / t + torch.log(s)
    e_lse = 2 * M.abs() / t + r_s + 4 * torch.log(s) + 4
    xk = torch.where(there, x.gather(-1, at), 0.0)
    logs = ahead / t - torch.log(st) - (xk / t - lse)
    used = q > 0
    e_log = (4 * ahead.abs() + (8 * xk.abs() + 4 * M.abs() if from_lse else 4 * (xk - M).abs())) / t + 4 * torch.log(s).abs() + 4 * torch.log(st) + r_s + K / 16 + 12
    loss = torch.where(used & there, q * torch.where(used, logs, 0.0), 0.0).sum(-1) * t * t
    e_loss = torch.where(used & there, q * (r_q * logs.abs() + e_log + (K / 16 + 8) * logs.abs()), 0.0).sum(-1) * t * t
    if from_lse:
        e_loss = e_loss + (lse.abs()[:, 0] + e_lse[:, 0]) * t * t
    back = lambda w: torch.where(some, w, 0.0).reshape(lead)  # noqa: E731
    res = {"loss": (back(loss), back(e_loss)), "lse": (back(lse[:, 0]), back(e_lse[:, 0]))}
    if dloss is None:
        return res
    scale = (f64(dloss).reshape(-1, 1) * t) * some[:, None]
    named = torch.zeros_like(x).scatter_add_(-1, at, torch.where(there, q, 0.0))
    e_named = torch.zeros_like(x).scatter_add_(-1, at, torch.where(there, q * (r_q + K / 16), 0.0))
    r_p = r_each + r_s + 6 + (6 * torch.maximum(x.abs().clamp_max(1e30), lse.abs()) / t + 4 * lse.abs() + e_lse if from_lse else 0)
    value = scale * (p - named)
    error = scale.abs() * (p * r_p + e_named + 4 * (p + named))
    res["dlogits"] = value.reshape(*lead, V), error.reshape(*lead, V)
    return res
