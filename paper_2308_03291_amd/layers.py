"""ctypes binding of ``include/lccrf_layers.h`` for torch device tensors: what a smaller tagger adds to the encoder.

A gated linear recurrence with one state a channel, group norm with an activation, and distillation from a teacher's top logits, with their
gradients and the recurrence's single-token form.  Manner and types are those of ``encoder`` (``binding`` exports all of this):
activations share one dtype, float32 or bfloat16, and may be views whose rows are dense; weights, states, statistics, the teacher's logits and losses are
float32 and contiguous; results are contiguous and carry no history for torch's automatic differentiation.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from .encoder import _MOST, _Rows, _activation, _bytes, _call, _dense, _first, _lengths, _lib, _like, _result, _scratch

MAX_TOP = 256
_NOTHING = 256  # a workspace of this size holds nothing and need not be there

_RecurInputs = ctypes.c_int64 * 15  # x, f, g, z as _Rows, decay, f_bias, g_bias
_RecurGrads = ctypes.c_int64 * 8    # dx, df, dg, dz, ddecay, df_bias, dg_bias, dstate


def declare(lib) -> None:
    """Argument types of the library's entry points for these layers."""
    vp, i, i64, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    of = {
        "lccrf_recurrence": [vp, i, f, vp, i, i, i, vp, vp, vp, vp, vp, sz, vp],
        "lccrf_recurrence_grad": [vp, vp, i, f, vp, i, i, i, vp, vp, vp, vp, sz, vp],
        "lccrf_recurrence_step": [vp, i, f, i, i, vp, vp, vp],
        "lccrf_group_norm": [vp, i, vp, vp, vp, i, i, i, i, i, f, i, vp, vp, vp, sz, vp],
        "lccrf_group_norm_grad": [vp, vp, i, vp, vp, vp, i, i, i, i, i, f, i, vp, vp, vp, vp, vp, sz, vp],
        "lccrf_distill": [vp, i64, i, vp, vp, i64, i, i, f, vp, vp, vp],
        "lccrf_distill_grad": [vp, vp, i64, i, vp, vp, i64, i, i, f, vp, vp, vp, vp],
    }
    for name, args in of.items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = i
    sizes = {
        "lccrf_recurrence_saved_bytes": 3, "lccrf_recurrence_workspace_bytes": 3, "lccrf_recurrence_grad_workspace_bytes": 4,
        "lccrf_group_norm_workspace_bytes": 6, "lccrf_group_norm_grad_workspace_bytes": 6,
    }
    for name, count in sizes.items():
        getattr(lib, name).argtypes = [i] * count
        getattr(lib, name).restype = sz


# ---- gated linear recurrence ----------------------------------------------------------------------------------

def _weights(names, *tensors, size: int, dev: int):
    """Addresses of contiguous float32 [size] tensors; 0 for those that are not there."""
    f32, shape = torch.float32, (size,)
    for t in tensors:
        if t is not None and not (t.dtype is f32 and t.shape == shape and t.get_device() == dev and (size == 1 or t.stride()[0] == 1)):
            for t, name in zip(tensors, names):  # one by one, to say what is wrong
                _dense(t, name, shape, f32, dev, True)
    return [0 if t is None else t.data_ptr() for t in tensors]


def _recur_args(x, f, g, decay, z, f_bias, g_bias):
    """Checks what all calls of the recurrence share; (dtype's code, device number, shape of x, dtype, the inputs' block)."""
    code, dtype, dev = _first(x, "x")
    shape = x.shape
    if 0 in shape or max(shape) > _MOST:
        raise ValueError(f"x must be [B, N, D] (one position: [B, D]), its sizes at most {_MOST}, got {list(shape)}")
    xs, fs, gs, zs, pz = x.stride(), f.stride(), g.stride(), (0, 0, 1), 0
    if z is not None:
        zs, pz = z.stride(), z.data_ptr()
    # all at once; one by one only to say what is wrong
    if not (f.shape == shape and g.shape == shape and f.dtype is dtype and g.dtype is dtype and xs[-1] == fs[-1] == gs[-1] == zs[-1] == 1
            and f.get_device() == g.get_device() == dev and (z is None or (z.shape == shape and z.dtype is dtype and z.get_device() == dev))):
        for t, name in ((x, "x"), (f, "f"), (g, "g"), (z, "z")):
            if t is not None:
                _activation(t, name, shape, dtype, dev)
    if decay is None:
        raise ValueError("decay is missing")
    pd, pf, pg = _weights(("decay", "f_bias", "g_bias"), decay, f_bias, g_bias, size=shape[-1], dev=dev)
    # (one position: the second stride is that of the channels, which nothing looks at)
    return code, dev, shape, dtype, _RecurInputs(x.data_ptr(), xs[0], xs[1], f.data_ptr(), fs[0], fs[1], g.data_ptr(), gs[0], gs[1], pz, zs[0], zs[1], pd, pf, pg)


def _scratch_at(name: str, sizes, device, workspace):
    """(address, bytes, tensor) of a call's workspace: none where the library keeps nothing there."""
    need = _bytes(f"{name}_workspace_bytes", *sizes)
    if workspace is None and need == _NOTHING:
        return 0, 0, None
    ws = _scratch(need, name, device, workspace)
    return ws.data_ptr(), ws.numel(), ws


def recurrence_saved(x: torch.Tensor) -> torch.Tensor:
    """Device memory for ``saved=`` of ``lccrf_recurrence`` on x [B, N, D]: what the gradient would otherwise compute again.  To be kept until
    ``lccrf_recurrence_grad`` has it; its layout is the library's."""
    if x.dim() != 3 or max(x.shape) > _MOST:
        raise ValueError(f"x must be [B, N, D], its sizes at most {_MOST}, got {list(x.shape)}")
    return _scratch(_bytes("lccrf_recurrence_saved_bytes", *x.shape), "recurrence_saved", x.device, None)


def _recur_saved(saved, shape, dev: int) -> int:
    if saved is None:
        return 0
    if saved.dtype != torch.uint8 or saved.get_device() != dev or not saved.is_contiguous() or saved.numel() < _bytes("lccrf_recurrence_saved_bytes", *shape):
        raise ValueError("saved must come from recurrence_saved for a tensor of x's shape")
    return saved.data_ptr()


def lccrf_recurrence(x: torch.Tensor, f: torch.Tensor, g: torch.Tensor, decay: torch.Tensor, z: Optional[torch.Tensor] = None,
                     f_bias: Optional[torch.Tensor] = None, g_bias: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None, *,
                     rate: float = 8.0, state: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                     final: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(out [B, N, D], final [B, D]) of the gated linear recurrence, with s the logistic function,

        u = -rate log(1 + exp(decay)) s(f + f_bias),  h = exp(u) h + sqrt(1 - exp(2 u)) s(g + g_bias) x,  out = h z s(z)

    over x, f, g, z [B, N, D] and decay, f_bias, g_bias [D]; without ``z`` out = h.  ``state`` [B, D] stands before the first position (0 without
    it); ``final`` after the last one within the length, and may be ``state`` itself."""
    if x.dim() != 3:
        raise ValueError(f"x must be [B, N, D], got {list(x.shape)}")
    code, dev, shape, dtype, block = _recur_args(x, f, g, decay, z, f_bias, g_bias)
    (B, N, D), device, f32 = shape, x.device, torch.float32
    plen = _lengths(lengths, B, dev)
    pstate = _dense(state, "state", (B, D), f32, dev, True)
    psaved = _recur_saved(saved, shape, dev)
    out = _result(out, "out", shape, dtype, None, dev, x)
    final = _result(final, "final", (B, D), f32, device, dev, state)
    pws, nws, ws = _scratch_at("lccrf_recurrence", (B, N, D), device, workspace)
    _call("lccrf_recurrence", dev, _lib().lccrf_recurrence, block, code, rate, plen, B, N, D, pstate, out.data_ptr(), final.data_ptr(), psaved, pws, nws)
    return out, final


class RecurrenceGrad(NamedTuple):
    dx: torch.Tensor
    df: torch.Tensor
    dg: torch.Tensor
    dz: Optional[torch.Tensor]
    ddecay: torch.Tensor
    df_bias: Optional[torch.Tensor]
    dg_bias: Optional[torch.Tensor]
    dstate: Optional[torch.Tensor]


def lccrf_recurrence_grad(dout: torch.Tensor, x: torch.Tensor, f: torch.Tensor, g: torch.Tensor, decay: torch.Tensor, z: Optional[torch.Tensor] = None,
                          f_bias: Optional[torch.Tensor] = None, g_bias: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None, *,
                          rate: float = 8.0, state: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None) -> RecurrenceGrad:
    """Gradients of a loss by what ``lccrf_recurrence`` takes, given its gradient ``dout`` by ``out`` (what follows through ``final`` is not part
    of it); None for what is not there.  ``saved``: of the forward call on the same inputs; without it that part is run again."""
    if x.dim() != 3:
        raise ValueError(f"x must be [B, N, D], got {list(x.shape)}")
    code, dev, shape, dtype, block = _recur_args(x, f, g, decay, z, f_bias, g_bias)
    strides = _activation(dout, "dout", shape, dtype, dev)
    B, N, D = shape
    plen = _lengths(lengths, B, dev)
    pstate = _dense(state, "state", (B, D), torch.float32, dev, True)
    psaved = _recur_saved(saved, shape, dev)
    grad = RecurrenceGrad(_like(x), _like(f), _like(g), *[None if t is None else _like(t) for t in (z, decay, f_bias, g_bias, state)])
    pws, nws, ws = _scratch_at("lccrf_recurrence_grad", (B, N, D, int(saved is not None)), x.device, workspace)
    _call("lccrf_recurrence_grad", dev, _lib().lccrf_recurrence_grad, _Rows(dout.data_ptr(), strides[0], strides[1]), block, code, rate, plen, B, N, D, pstate, psaved,
          _RecurGrads(*[0 if t is None else t.data_ptr() for t in grad]), pws, nws)
    return grad


def lccrf_recurrence_step(x: torch.Tensor, f: torch.Tensor, g: torch.Tensor, decay: torch.Tensor, z: Optional[torch.Tensor], f_bias: Optional[torch.Tensor],
                          g_bias: Optional[torch.Tensor], state: torch.Tensor, *, rate: float = 8.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One position of every stream: x, f, g, z [B, D]; state float32 [B, D] moves on in place; the result is [B, D]."""
    if x.dim() != 2:
        raise ValueError(f"x must be [B, D], got {list(x.shape)}")
    code, dev, shape, dtype, block = _recur_args(x, f, g, decay, z, f_bias, g_bias)
    pstate = _dense(state, "state", shape, torch.float32, dev)
    out = _result(out, "out", shape, dtype, None, dev, x)
    _call("lccrf_recurrence_step", dev, _lib().lccrf_recurrence_step, block, code, rate, shape[0], shape[1], pstate, out.data_ptr())
    return out


# ---- group norm -----------------------------------------------------------------------------------------------

def _norm_args(x, weight, bias, groups):
    code, dtype, dev = _first(x, "x")
    shape = x.shape
    if len(shape) != 3 or 0 in shape or max(shape) > _MOST:
        raise ValueError(f"x must be [B, N, D], its sizes at most {_MOST}, got {list(shape)}")
    if groups < 1 or shape[2] % groups:
        raise ValueError(f"{shape[2]} channels cannot be cut into {groups} groups")
    strides = _activation(x, "x", shape, dtype, dev)
    return (code, dtype, dev, shape, _Rows(x.data_ptr(), strides[0], strides[1]), *_weights(("weight", "bias"), weight, bias, size=shape[2], dev=dev))


def _stats_shape(shape, groups: int, per_position: bool):
    return (*shape[:2], groups, 2) if per_position else (shape[0], groups, 2)


def group_norm_stats(x: torch.Tensor, groups: int, *, per_position: bool = False) -> torch.Tensor:
    """Memory for ``stats=`` of ``lccrf_group_norm`` on x [B, N, D]: mean and 1 / deviation of every group, float32 [B, groups, 2], or
    [B, N, groups, 2] per position."""
    if x.dim() != 3 or groups < 1:
        raise ValueError(f"x must be [B, N, D] and groups positive, got {list(x.shape)} and {groups}")
    return torch.empty(_stats_shape(x.shape, groups, per_position), dtype=torch.float32, device=x.device)


def lccrf_group_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None, *,
                     groups: int, eps: float = 1e-5, silu: bool = True, per_position: bool = False, stats: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Group norm of x [B, N, D] over ``groups`` equal groups of channels, times weight [D], plus bias [D], then y * sigmoid(y) (``silu``; without
    it y itself).  A group is normalised together over all positions of a sequence within its length, or (``per_position``) at every position by
    itself, which is what a stream of single tokens can do: x [B, 1, D].  ``stats`` (of ``group_norm_stats``) takes what the gradient would
    otherwise compute again."""
    code, dtype, dev, shape, prows, pw, pb = _norm_args(x, weight, bias, groups)
    (B, N, D), device = shape, x.device
    plen = _lengths(lengths, B, dev)
    pstats = _dense(stats, "stats", _stats_shape(shape, groups, per_position), torch.float32, dev, True)
    out = _result(out, "out", shape, dtype, None, dev, x)
    alone = int(per_position)
    pws, nws, ws = _scratch_at("lccrf_group_norm", (code, B, N, D, groups, alone), device, workspace)
    _call("lccrf_group_norm", dev, _lib().lccrf_group_norm, prows, code, pw, pb, plen, B, N, D, groups, alone, eps, int(silu), out.data_ptr(), pstats, pws, nws)
    return out


class GroupNormGrad(NamedTuple):
    dx: torch.Tensor
    dweight: Optional[torch.Tensor]
    dbias: Optional[torch.Tensor]


def lccrf_group_norm_grad(dout: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                          lengths: Optional[torch.Tensor] = None, *, groups: int, eps: float = 1e-5, silu: bool = True, per_position: bool = False,
                          stats: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> GroupNormGrad:
    """Gradients of a loss by what ``lccrf_group_norm`` takes, given its gradient ``dout`` by ``out``; None for what is not there.  ``stats``: of the
    forward call on the same inputs."""
    code, dtype, dev, shape, prows, pw, pb = _norm_args(x, weight, bias, groups)
    strides = _activation(dout, "dout", shape, dtype, dev)
    B, N, D = shape
    plen = _lengths(lengths, B, dev)
    pstats = _dense(stats, "stats", _stats_shape(shape, groups, per_position), torch.float32, dev, True)
    grad = GroupNormGrad(_like(x), *[None if t is None else _like(t) for t in (weight, bias)])
    alone = int(per_position)
    pws, nws, ws = _scratch_at("lccrf_group_norm_grad", (code, B, N, D, groups, alone), x.device, workspace)
    _call("lccrf_group_norm_grad", dev, _lib().lccrf_group_norm_grad, _Rows(dout.data_ptr(), strides[0], strides[1]), prows, code, pw, pb, plen, B, N, D, groups, alone, eps,
          int(silu), pstats, *[0 if t is None else t.data_ptr() for t in grad], pws, nws)
    return grad


# ---- distillation ---------------------------------------------------------------------------------------------

def _distill_args(logits, ids, teacher):
    """(dtype's code, dtype, device number, shape of the positions, their number, V, K, elements between rows, addresses of ids and teacher)."""
    code, dtype, dev = _first(logits, "logits")
    shape = logits.shape
    if len(shape) < 2 or shape[-1] < 1 or max(shape) > _MOST:
        raise ValueError(f"logits must be [..., V], its sizes at most {_MOST}, got {list(shape)}")
    lead, V, strides = shape[:-1], shape[-1], logits.stride()
    if strides[-1] != 1 and V > 1:
        raise ValueError("logits' last dimension must be dense")
    if logits.is_contiguous():
        n, row = logits.numel() // V, V
    else:
        n, row = 1, 0
        for size, stride in zip(reversed(lead), reversed(strides[:-1])):
            if size > 1:  # one distance between all rows
                if n > 1 and stride != row * n:
                    raise ValueError("logits' rows must lie at one distance from each other")
                row = row if n > 1 else stride
            n *= size
    if ids.dim() != len(shape) or not 1 <= ids.shape[-1] <= MAX_TOP:
        raise ValueError(f"ids must be [..., K] with 1 to {MAX_TOP} entries a position, got {list(ids.shape)}")
    top = (*lead, ids.shape[-1])
    return code, dtype, dev, lead, n, V, ids.shape[-1], row if n > 1 else V, _dense(ids, "ids", top, torch.int32, dev), _dense(teacher, "teacher", top, torch.float32, dev)


def lccrf_distill(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, *, temperature: float = 1.0, loss: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None):
    """(loss, lse), float32 of the positions' shape: how far softmax(logits / t) [..., V] is from a teacher that names K classes a position
    with their logits (ids int32 [..., K], teacher float32 [..., K]),

        loss = t^2 sum_k q_k (log q_k - log p[ids_k]),  q = softmax(teacher / t),  p = softmax(logits / t),  lse = log sum exp(logits / t).

    t is finite and at least 2^-126.  An entry whose id is outside [0, V) or whose logit is -inf is not there; a class may be named twice; a position without
    an entry (padding) has loss and lse 0."""
    code, _, dev, lead, n, V, K, row, pids, pteacher = _distill_args(logits, ids, teacher)
    loss = _result(loss, "loss", lead, torch.float32, logits.device, dev)
    lse = _result(lse, "lse", lead, torch.float32, logits.device, dev)
    _call("lccrf_distill", dev, _lib().lccrf_distill, logits.data_ptr(), row, code, pids, pteacher, n, V, K, temperature, loss.data_ptr(), lse.data_ptr())
    return loss, lse


def lccrf_distill_grad(dloss: torch.Tensor, logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, *, temperature: float = 1.0,
                       lse: Optional[torch.Tensor] = None, loss: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of ``lccrf_distill`` by its logits, dloss t (p - q) [..., V], given dloss (float32, the positions' shape).  ``lse``: of the forward
    call; computed again without it (more closely in rows of many classes where |lse| or |logits| / t is large: p is exp(logits / t - lse) of
    rounded numbers).  ``loss`` takes the loss as well: where dloss is known ahead, this one call is all of a training step's loss.  ``out`` may be ``logits`` itself."""
    code, dtype, dev, lead, n, V, K, row, pids, pteacher = _distill_args(logits, ids, teacher)
    f32 = torch.float32
    pd, ps, pl = _dense(dloss, "dloss", lead, f32, dev), _dense(lse, "lse", lead, f32, dev, True), _dense(loss, "loss", lead, f32, dev, True)
    out = _result(out, "out", logits.shape, dtype, None, dev, logits)
    _call("lccrf_distill_grad", dev, _lib().lccrf_distill_grad, pd, logits.data_ptr(), row, code, pids, pteacher, n, V, K, temperature, ps, pl, out.data_ptr())
    return out
