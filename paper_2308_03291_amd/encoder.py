"""ctypes binding of the encoder's entry points (``include/lccrf_encoder.h``) for torch device tensors.

What stands in front of a tagger's chain: embedding lookup, short causal convolution and selective state space scan, their
gradients and their single-token forms.  As in ``binding`` (which exports all of this): arguments are checked and handed on,
every step of the computation runs in the library's kernels on the current stream, and there is no fallback.

Activations (``table``, ``x``, ``dt``, ``Bm``, ``Cm``, ``z``, ``dout`` and the convolution's state) share one dtype, float32 or
bfloat16; weights (``weight``, ``bias``, ``A``, ``D``, ``dt_bias``), their gradients and the scan's state are float32.
Activations may be views whose rows are dense (half of a projection's output, an expanded row); weights and states are
contiguous, and so are results.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import binding as _b

MIN_TAPS, MAX_TAPS, MAX_STATES = 2, 8, 64

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("row", ctypes.c_int64)]


class _ScanInputs(ctypes.Structure):
    _fields_ = [("x", _Rows), ("dt", _Rows), ("Bm", _Rows), ("Cm", _Rows), ("z", _Rows), ("b_group", ctypes.c_int64),
                ("c_group", ctypes.c_int64), ("A", ctypes.c_void_p), ("D", ctypes.c_void_p), ("dt_bias", ctypes.c_void_p)]


class _ScanGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dx", "ddt", "dBm", "dCm", "dz", "dA", "dD", "ddt_bias", "dstate")]


def declare(lib) -> None:
    """Argument types of the library's encoder entry points."""
    vp, i, i64, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    of = {
        "lccrf_embed": [vp, i, i, i, i64, vp, i64, f, vp, vp],
        "lccrf_embed_grad": [vp, i, vp, i, i, i, i, f, vp, vp, sz, vp],
        "lccrf_conv": [vp, i, vp, vp, vp, vp, i, i, i, i, vp, vp, vp],
        "lccrf_conv_grad": [vp, vp, i, vp, vp, vp, vp, i, i, i, i, vp, vp, vp, vp, vp, sz, vp],
        "lccrf_conv_step": [vp, i64, i, vp, vp, vp, i, i, i, vp, vp],
        "lccrf_state_scan": [vp, i, vp, i, i, i, i, i, vp, vp, vp, vp, vp, sz, vp],
        "lccrf_state_scan_grad": [vp, vp, i, vp, i, i, i, i, i, vp, vp, vp, vp, sz, vp],
        "lccrf_state_step": [vp, i, i, i, i, i, vp, vp, vp],
    }
    for name, args in of.items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = i
    sizes = {
        "lccrf_embed_grad_workspace_bytes": [i64, i, i], "lccrf_conv_grad_workspace_bytes": [i, i, i, i],
        "lccrf_state_scan_saved_bytes": [i, i, i, i], "lccrf_state_scan_workspace_bytes": [i, i, i, i, i],
        "lccrf_state_scan_grad_workspace_bytes": [i, i, i, i, i, i],
    }
    for name, args in sizes.items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = sz


def _type(t: torch.Tensor, name: str) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise ValueError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    return dt


def _activation(t: torch.Tensor, name: str, shape, like: torch.Tensor) -> None:
    """An input whose last dimension is dense."""
    if t.shape != shape or t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name} must be {like.dtype} {list(shape)} on {like.device}, got {t.dtype} {list(t.shape)} on {t.device}")
    if t.stride(-1) != 1 and shape[-1] > 1:
        raise ValueError(f"{name}'s last dimension must be dense")


def _dense(t: Optional[torch.Tensor], name: str, shape, dtype, device, optional: bool = False) -> Optional[int]:
    """A contiguous tensor's address; None for one that is not there."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is missing")
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} {list(shape)} tensor on {device}")
    return t.data_ptr()


def _result(t: Optional[torch.Tensor], name: str, shape, dtype, device) -> torch.Tensor:
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _dense(t, name, shape, dtype, device)
    return t


def _scratch(need: int, what: str, device, workspace: Optional[torch.Tensor]) -> torch.Tensor:
    if need == 0:
        raise ValueError(f"{what}: unsupported sizes")
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if workspace.dtype != torch.uint8 or workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the inputs' device")
    return workspace


def _rows(t: torch.Tensor) -> _Rows:
    return _Rows(t.data_ptr(), t.stride(0), t.stride(1))


def lccrf_embed(table: torch.Tensor, ids: torch.Tensor, *, scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * table[ids]: table [V, D] (rows dense), ids int32 of any shape, contiguous; the result has one dimension, D, more.
    Ids outside [0, V) (padding) give rows of 0."""
    dt = _type(table, "table")
    if table.dim() != 2 or 0 in table.shape:
        raise ValueError(f"table must be [V, D], got {list(table.shape)}")
    V, D = table.shape
    _activation(table, "table", table.shape, table)
    dev = table.device
    pids = _dense(ids, "ids", ids.shape, torch.int32, dev)
    out = _result(out, "out", (*ids.shape, D), table.dtype, dev)
    _b._enqueue("lccrf_embed", dev, _b.load_library().lccrf_embed, table.data_ptr(), dt, V, D, table.stride(0), pids, ids.numel(), scale, out.data_ptr(),
                _b._stream(dev))
    return out


def lccrf_embed_grad(dout: torch.Tensor, ids: torch.Tensor, V: int, *, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of ``lccrf_embed`` by its table, [V, D] in dout's dtype: every row is scale times the sum, in a fixed order, of the
    rows of dout [B, N, D] (or [n, D]) whose id (int32 [B, N] or [n]) it is; ids outside [0, V) have none."""
    dt = _type(dout, "dout")
    if dout.dim() == 2:
        dout, ids = dout[None], ids[None]
    if dout.dim() != 3 or dout.shape[2] == 0 or V < 1:
        raise ValueError(f"dout must be [B, N, D] and V positive, got {list(dout.shape)} and {V}")
    B, N, D = dout.shape
    _activation(dout, "dout", dout.shape, dout)
    dev, lib = dout.device, _b.load_library()
    pids = _dense(ids, "ids", (B, N), torch.int32, dev)
    out = _result(out, "out", (V, D), dout.dtype, dev)
    ws = _scratch(lib.lccrf_embed_grad_workspace_bytes(B * N, V, D), "lccrf_embed_grad", dev, workspace)
    _b._enqueue("lccrf_embed_grad", dev, lib.lccrf_embed_grad, ctypes.byref(_rows(dout)), dt, pids, B, N, V, D, scale, out.data_ptr(), ws.data_ptr(), ws.numel(),
                _b._stream(dev))
    return out


def _conv_args(x: torch.Tensor, weight: torch.Tensor, bias, state):
    dt = _type(x, "x")
    D = x.shape[-1]
    if weight.dim() != 2 or 0 in x.shape:
        raise ValueError(f"x must be [B, N, D] (one position: [B, D]) and weight [D, K], got {list(x.shape)} and {list(weight.shape)}")
    K = weight.shape[1]
    if not MIN_TAPS <= K <= MAX_TAPS:
        raise ValueError(f"{MIN_TAPS} to {MAX_TAPS} taps are served, got {K}")
    _activation(x, "x", x.shape, x)
    return (dt, D, K, _dense(weight, "weight", (D, K), torch.float32, x.device), _dense(bias, "bias", (D,), torch.float32, x.device, True),
            _dense(state, "state", (x.shape[0], K - 1, D), x.dtype, x.device, True))


def lccrf_conv(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None, *,
               state: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, final: Optional[torch.Tensor] = None):
    """(out [B, N, D], final [B, K-1, D]): p * sigmoid(p) of the causal convolution p of x [B, N, D] with weight [D, K] and bias [D].
    ``state`` holds the K - 1 inputs before the sequences (0 without it), ``final`` the last K - 1, from which a later call goes
    on.  Positions past the lengths give 0.  ``final`` must be another tensor than ``state``."""
    if x.dim() != 3:
        raise ValueError(f"x must be [B, N, D], got {list(x.shape)}")
    dt, D, K, pw, pb, ps = _conv_args(x, weight, bias, state)
    B, N, dev = x.shape[0], x.shape[1], x.device
    plen = _b._len_ptr(lengths, B, dev)
    out = _result(out, "out", (B, N, D), x.dtype, dev)
    final = _result(final, "final", (B, K - 1, D), x.dtype, dev)
    _b._enqueue("lccrf_conv", dev, _b.load_library().lccrf_conv, ctypes.byref(_rows(x)), dt, pw, pb, ps, plen, B, N, D, K, out.data_ptr(), final.data_ptr(),
                _b._stream(dev))
    return out, final


class ConvGrad(NamedTuple):
    dx: torch.Tensor
    dweight: torch.Tensor
    dbias: Optional[torch.Tensor]
    dstate: Optional[torch.Tensor]


def lccrf_conv_grad(dout: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                    lengths: Optional[torch.Tensor] = None, *, state: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None) -> ConvGrad:
    """Gradients of a loss by what ``lccrf_conv`` takes, given its gradient ``dout`` by ``out`` (what follows through ``final`` is
    not part of it); ``dbias`` and ``dstate`` are None where there is no bias or state."""
    if x.dim() != 3:
        raise ValueError(f"x must be [B, N, D], got {list(x.shape)}")
    dt, D, K, pw, pb, ps = _conv_args(x, weight, bias, state)
    _activation(dout, "dout", x.shape, x)
    B, N, dev, lib = x.shape[0], x.shape[1], x.device, _b.load_library()
    plen = _b._len_ptr(lengths, B, dev)
    g = ConvGrad(torch.empty((B, N, D), dtype=x.dtype, device=dev), torch.empty((D, K), device=dev),
                 None if bias is None else torch.empty((D,), device=dev), None if state is None else torch.empty((B, K - 1, D), dtype=x.dtype, device=dev))
    ws = _scratch(lib.lccrf_conv_grad_workspace_bytes(B, N, D, K), "lccrf_conv_grad", dev, workspace)
    _b._enqueue("lccrf_conv_grad", dev, lib.lccrf_conv_grad, ctypes.byref(_rows(dout)), ctypes.byref(_rows(x)), dt, pw, pb, ps, plen, B, N, D, K,
                *(None if t is None else t.data_ptr() for t in g), ws.data_ptr(), ws.numel(), _b._stream(dev))
    return g


def lccrf_conv_step(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor], state: torch.Tensor, *,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One position of every stream: x [B, D], state [B, K-1, D], which moves on in place; the result is [B, D]."""
    if x.dim() != 2:
        raise ValueError(f"x must be [B, D], got {list(x.shape)}")
    if state is None:
        raise ValueError("state is missing")
    dt, D, K, pw, pb, ps = _conv_args(x, weight, bias, state)
    out = _result(out, "out", x.shape, x.dtype, x.device)
    _b._enqueue("lccrf_conv_step", x.device, _b.load_library().lccrf_conv_step, x.data_ptr(), x.stride(0), dt, pw, pb, ps, x.shape[0], D, K, out.data_ptr(),
                _b._stream(x.device))
    return out


def _scan_args(x, dt, A, Bm, Cm, D, z, dt_bias):
    """Checks what all calls of the scan share; (dtype, D, S, G, the inputs' block)."""
    code = _type(x, "x")
    if 0 in x.shape or A.dim() != 2 or Bm.dim() != x.dim() + 1:
        raise ValueError(f"x must be [B, N, D], A [D, S] and Bm [B, N, G, S] (one position: [B, D] and [B, G, S]), got {list(x.shape)}, {list(A.shape)} "
                         f"and {list(Bm.shape)}")
    width, S, G, dev, one = x.shape[-1], A.shape[1], Bm.shape[-2], x.device, x.dim() == 2
    if not 1 <= S <= MAX_STATES:
        raise ValueError(f"1 to {MAX_STATES} states a channel are served, got {S}")
    if G < 1 or width % G:
        raise ValueError(f"{width} channels cannot be shared by {G} groups")
    _activation(x, "x", x.shape, x)
    _activation(dt, "dt", x.shape, x)
    vectors = (*x.shape[:-1], G, S)
    _activation(Bm, "Bm", vectors, x)
    _activation(Cm, "Cm", vectors, x)
    if z is not None:
        _activation(z, "z", x.shape, x)
    f32 = torch.float32
    pA, pD, pb = _dense(A, "A", (width, S), f32, dev), _dense(D, "D", (width,), f32, dev, True), _dense(dt_bias, "dt_bias", (width,), f32, dev, True)

    def rows(t):
        if t is None:
            return _Rows(None, 0, 0)
        return _Rows(t.data_ptr(), t.stride(0), 0 if one else t.stride(1))

    return code, width, S, G, _ScanInputs(rows(x), rows(dt), rows(Bm), rows(Cm), rows(z), Bm.stride(-2), Cm.stride(-2), pA, pD, pb)


def state_scan_saved(x: torch.Tensor, A: torch.Tensor) -> torch.Tensor:
    """Device memory for ``saved=`` of ``lccrf_state_scan`` on x [B, N, D] and A [D, S]: what the gradient would otherwise compute
    again.  To be kept until ``lccrf_state_scan_grad`` has it; its layout is the library's."""
    if x.dim() != 3 or A.dim() != 2 or A.shape[0] != x.shape[2]:
        raise ValueError(f"x must be [B, N, D] and A [D, S], got {list(x.shape)} and {list(A.shape)}")
    need = _b.load_library().lccrf_state_scan_saved_bytes(*x.shape, A.shape[1])
    return _scratch(need, "state_scan_saved", x.device, None)


def _saved_ptr(saved, x, S) -> Optional[int]:
    if saved is None:
        return None
    if saved.dtype != torch.uint8 or saved.device != x.device or not saved.is_contiguous() or \
            saved.numel() < _b.load_library().lccrf_state_scan_saved_bytes(*x.shape, S):
        raise ValueError("saved must come from state_scan_saved for tensors of these shapes")
    return saved.data_ptr()


def lccrf_state_scan(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, Bm: torch.Tensor, Cm: torch.Tensor, D: Optional[torch.Tensor] = None,
                     z: Optional[torch.Tensor] = None, dt_bias: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None, *,
                     state: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                     final: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(out [B, N, D], final [B, D, S]) of the selective state space scan

        step = log(1 + exp(dt + dt_bias)),  h = exp(step A) h + step x Bm,  y = sum_s Cm h + D x,  out = y z sigmoid(z)

    over x, dt, z [B, N, D], Bm, Cm [B, N, G, S], A [D, S], D and dt_bias [D]; without ``z`` out = y.  ``state`` [B, D, S] stands before
    the first position (0 without it); ``final`` after the last one within the length, and may be ``state`` itself."""
    if x.dim() != 3:
        raise ValueError(f"x must be [B, N, D], got {list(x.shape)}")
    code, width, S, G, block = _scan_args(x, dt, A, Bm, Cm, D, z, dt_bias)
    B, N, dev, lib = x.shape[0], x.shape[1], x.device, _b.load_library()
    plen = _b._len_ptr(lengths, B, dev)
    pstate = _dense(state, "state", (B, width, S), torch.float32, dev, True)
    psaved = _saved_ptr(saved, x, S)
    out = _result(out, "out", (B, N, width), x.dtype, dev)
    final = _result(final, "final", (B, width, S), torch.float32, dev)
    ws = _scratch(lib.lccrf_state_scan_workspace_bytes(B, N, width, S, G), "lccrf_state_scan", dev, workspace)
    _b._enqueue("lccrf_state_scan", dev, lib.lccrf_state_scan, ctypes.byref(block), code, plen, B, N, width, S, G, pstate, out.data_ptr(), final.data_ptr(), psaved,
                ws.data_ptr(), ws.numel(), _b._stream(dev))
    return out, final


class ScanGrad(NamedTuple):
    dx: torch.Tensor
    ddt: torch.Tensor
    dBm: torch.Tensor
    dCm: torch.Tensor
    dz: Optional[torch.Tensor]
    dA: torch.Tensor
    dD: Optional[torch.Tensor]
    ddt_bias: Optional[torch.Tensor]
    dstate: Optional[torch.Tensor]


def lccrf_state_scan_grad(dout: torch.Tensor, x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, Bm: torch.Tensor, Cm: torch.Tensor,
                          D: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None, dt_bias: Optional[torch.Tensor] = None,
                          lengths: Optional[torch.Tensor] = None, *, state: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None) -> ScanGrad:
    """Gradients of a loss by what ``lccrf_state_scan`` takes, given its gradient ``dout`` by ``out`` (what follows through ``final``
    is not part of it); None for what is not there.  ``saved``: of the forward call on the same inputs; without it that part is run
    again.  dBm and dCm are sums over the channels of their group."""
    if x.dim() != 3:
        raise ValueError(f"x must be [B, N, D], got {list(x.shape)}")
    code, width, S, G, block = _scan_args(x, dt, A, Bm, Cm, D, z, dt_bias)
    _activation(dout, "dout", x.shape, x)
    B, N, dev, lib = x.shape[0], x.shape[1], x.device, _b.load_library()
    plen = _b._len_ptr(lengths, B, dev)
    pstate = _dense(state, "state", (B, width, S), torch.float32, dev, True)
    psaved = _saved_ptr(saved, x, S)

    def like(shape, dtype, wanted=True):
        return torch.empty(shape, dtype=dtype, device=dev) if wanted else None

    f32, rows, vectors = torch.float32, (B, N, width), (B, N, G, S)
    g = ScanGrad(like(rows, x.dtype), like(rows, x.dtype), like(vectors, x.dtype), like(vectors, x.dtype), like(rows, x.dtype, z is not None),
                 like((width, S), f32), like((width,), f32, D is not None), like((width,), f32, dt_bias is not None),
                 like((B, width, S), f32, state is not None))
    ws = _scratch(lib.lccrf_state_scan_grad_workspace_bytes(B, N, width, S, G, saved is not None), "lccrf_state_scan_grad", dev, workspace)
    grads = _ScanGrads(*(None if t is None else t.data_ptr() for t in g))
    _b._enqueue("lccrf_state_scan_grad", dev, lib.lccrf_state_scan_grad, ctypes.byref(_rows(dout)), ctypes.byref(block), code, plen, B, N, width, S, G, pstate, psaved,
                ctypes.byref(grads), ws.data_ptr(), ws.numel(), _b._stream(dev))
    return g


def lccrf_state_step(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, Bm: torch.Tensor, Cm: torch.Tensor, D: Optional[torch.Tensor],
                     z: Optional[torch.Tensor], dt_bias: Optional[torch.Tensor], state: torch.Tensor, *,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One position of every stream: x, dt, z [B, D], Bm, Cm [B, G, S]; state float32 [B, D, S] moves on in place; the result is [B, D]."""
    if x.dim() != 2:
        raise ValueError(f"x must be [B, D], got {list(x.shape)}")
    code, width, S, G, block = _scan_args(x, dt, A, Bm, Cm, D, z, dt_bias)
    B, dev = x.shape[0], x.device
    pstate = _dense(state, "state", (B, width, S), torch.float32, dev)
    out = _result(out, "out", x.shape, x.dtype, dev)
    _b._enqueue("lccrf_state_step", dev, _b.load_library().lccrf_state_step, ctypes.byref(block), code, B, width, S, G, pstate, out.data_ptr(), _b._stream(dev))
    return out
