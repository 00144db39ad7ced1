"""ctypes binding of the encoder's entry points (``include/lccrf_encoder.h``) for torch device tensors.

What stands in front of a tagger's chain: embedding lookup, short causal convolution and selective state space scan, their
gradients and their single-token forms.  As in ``binding`` (which exports all of this): arguments are checked and handed on,
every step of the computation runs in the library's kernels on the current stream, and there is no fallback.

Activations (``table``, ``x``, ``dt``, ``Bm``, ``Cm``, ``z``, ``dout`` and the convolution's state) share one dtype, float32 or
bfloat16; weights (``weight``, ``bias``, ``A``, ``D``, ``dt_bias``), their gradients and the scan's state are float32.
Activations may be views whose rows are dense (half of a projection's output, an expanded row); weights and states are
contiguous, and so are results.

As everywhere in ``binding``, results carry no history for torch's automatic differentiation, whether inputs require gradients or
not: a backward pass is the ``_grad`` calls, by hand (``tagger`` has one) or inside a ``torch.autograd.Function``.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

import torch

from . import binding as _b

MIN_TAPS, MAX_TAPS, MAX_STATES = 2, 8, 64
_MOST = 2 ** 31 - 1  # the C ABI takes sizes as int: ctypes would cut larger ones (an expanded view can have them) to 32 bits without a word

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


# A call for one token takes the GPU a few microseconds, so the host's part of it counts: the argument blocks of the C ABI (lccrf_rows,
# lccrf_scan_inputs, lccrf_scan_grads: nothing but 8-byte fields) are filled as arrays in one go, devices are compared by their numbers, sizes
# of workspaces are asked for once (lccrf_state_step, B=4 D=1024 S=16: 15.2 us of host work -> 11).
_Rows = ctypes.c_int64 * 3         # address, elements between sequences, elements between positions
_ScanInputs = ctypes.c_int64 * 20  # x, dt, Bm, Cm, z as _Rows, elements between groups of Bm and Cm, A, D, dt_bias
_ScanGrads = ctypes.c_int64 * 9    # dx, ddt, dBm, dCm, dz, dA, dD, ddt_bias, dstate


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


def _lib():
    return _b._lib or _b.load_library()


@functools.lru_cache(maxsize=4096)
def _bytes(name: str, *sizes: int) -> int:
    return getattr(_b.load_library(), name)(*sizes)


def _first(t: torch.Tensor, name: str):
    """(dtype's code, dtype, device number) of the tensor that the others have to go with."""
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise ValueError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must live on the GPU")
    return dt, t.dtype, dev


def _activation(t: torch.Tensor, name: str, shape, dtype, dev: int):
    """The strides of an input whose last dimension is dense."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{name} must be {dtype} {list(shape)} on GPU {dev}, got {t.dtype} {list(t.shape)} on {t.device}")
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}'s last dimension must be dense")
    return strides


def _dense(t: Optional[torch.Tensor], name: str, shape, dtype, dev: int, optional: bool = False) -> int:
    """A contiguous tensor's address; 0 for one that is not there."""
    if t is None:
        if optional:
            return 0
        raise ValueError(f"{name} is missing")
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} {list(shape)} tensor on GPU {dev}")
    return t.data_ptr()


def _like(t: torch.Tensor) -> torch.Tensor:
    """Memory of t's shape and type (empty_like takes half of empty's two microseconds; strides other than dense ones it must not take over)."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _result(t: Optional[torch.Tensor], name: str, shape, dtype, device, dev: int, like: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The caller's tensor, or a new one (``like``: one of the same shape and type, if there is one)."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device) if like is None else _like(like)
    _dense(t, name, shape, dtype, dev)
    return t


def _lengths(lengths: Optional[torch.Tensor], B: int, dev: int) -> int:
    return _dense(lengths, "lengths", (B,), torch.int32, dev, True)


def _scratch(need: int, what: str, device, workspace: Optional[torch.Tensor]) -> torch.Tensor:
    if need == 0:
        raise ValueError(f"{what}: unsupported sizes")
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if workspace.dtype != torch.uint8 or workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the inputs' device")
    return workspace


def _call(name: str, dev: int, call, *args) -> None:
    """call(*args, the current stream) with GPU `dev` current; raises if it reports an error."""
    if _b._current_device() == dev:
        rc = call(*args, _b._raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = call(*args, _b._raw_stream(dev))
    if rc != 0:
        _b._check(rc, name)


def lccrf_embed(table: torch.Tensor, ids: torch.Tensor, *, scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * table[ids]: table [V, D] (rows dense), ids int32 of any shape, contiguous; the result has one dimension, D, more.
    Ids outside [0, V) (padding) give rows of 0."""
    dt, dtype, dev = _first(table, "table")
    if table.dim() != 2 or 0 in table.shape:
        raise ValueError(f"table must be [V, D], got {list(table.shape)}")
    V, D = table.shape
    if V > _MOST or D > _MOST:
        raise ValueError(f"a table of at most {_MOST} rows and columns is served, got {list(table.shape)}")
    row = _activation(table, "table", table.shape, dtype, dev)[0]
    shape = ids.shape
    pids = _dense(ids, "ids", shape, torch.int32, dev)
    out = _result(out, "out", (*shape, D), dtype, table.device, dev)
    _call("lccrf_embed", dev, _lib().lccrf_embed, table.data_ptr(), dt, V, D, row, pids, ids.numel(), scale, out.data_ptr())
    return out


def lccrf_embed_grad(dout: torch.Tensor, ids: torch.Tensor, V: int, *, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of ``lccrf_embed`` by its table, [V, D] in dout's dtype: every row is scale times the sum, in a fixed order, of the
    rows of dout [B, N, D] (or [n, D]) whose id (int32 [B, N] or [n]) it is; ids outside [0, V) have none.  Summed in float32 and
    rounded once: the gradient of a bfloat16 table is bfloat16, and where the master copy is float32 (as in ``tagger``) that rounding is the
    only one it adds."""
    dt, dtype, dev = _first(dout, "dout")
    if dout.dim() == 2:
        dout, ids = dout[None], ids[None]
    shape = dout.shape
    if len(shape) != 3 or shape[2] == 0 or not 1 <= V <= _MOST or max(shape) > _MOST:
        raise ValueError(f"dout must be [B, N, D] and V positive, all of them at most {_MOST}, got {list(shape)} and {V}")
    B, N, D = shape
    strides = _activation(dout, "dout", shape, dtype, dev)
    pids = _dense(ids, "ids", (B, N), torch.int32, dev)
    device = dout.device
    out = _result(out, "out", (V, D), dtype, device, dev)
    ws = _scratch(_bytes("lccrf_embed_grad_workspace_bytes", B * N, V, D), "lccrf_embed_grad", device, workspace)
    _call("lccrf_embed_grad", dev, _lib().lccrf_embed_grad, _Rows(dout.data_ptr(), strides[0], strides[1]), dt, pids, B, N, V, D, scale, out.data_ptr(),
          ws.data_ptr(), ws.numel())
    return out


def _conv_args(x: torch.Tensor, weight: torch.Tensor, bias, state):
    """Checks what all calls of the convolution share; (dtype's code, device number, D, K, strides of x, the others' addresses)."""
    dt, dtype, dev = _first(x, "x")
    shape = x.shape
    if weight.dim() != 2 or 0 in shape or max(shape) > _MOST:
        raise ValueError(f"x must be [B, N, D] (one position: [B, D]), its sizes at most {_MOST}, and weight [D, K], got {list(shape)} and {list(weight.shape)}")
    D, K = shape[-1], weight.shape[1]
    if not MIN_TAPS <= K <= MAX_TAPS:
        raise ValueError(f"{MIN_TAPS} to {MAX_TAPS} taps are served, got {K}")
    strides = _activation(x, "x", shape, dtype, dev)
    return (dt, dev, D, K, strides, _dense(weight, "weight", (D, K), torch.float32, dev), _dense(bias, "bias", (D,), torch.float32, dev, True),
            _dense(state, "state", (shape[0], K - 1, D), dtype, dev, True))


def lccrf_conv(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None, *,
               state: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, final: Optional[torch.Tensor] = None):
    """(out [B, N, D], final [B, K-1, D]): p * sigmoid(p) of the causal convolution p of x [B, N, D] with weight [D, K] and bias [D].
    ``state`` holds the K - 1 inputs before the sequences (0 without it), ``final`` the last K - 1, from which a later call goes
    on.  Positions past the lengths give 0.  ``final`` must be another tensor than ``state``."""
    if x.dim() != 3:
        raise ValueError(f"x must be [B, N, D], got {list(x.shape)}")
    dt, dev, D, K, strides, pw, pb, ps = _conv_args(x, weight, bias, state)
    (B, N, _), device = x.shape, x.device
    plen = _lengths(lengths, B, dev)
    out = _result(out, "out", x.shape, x.dtype, None, dev, x)
    final = _result(final, "final", (B, K - 1, D), x.dtype, device, dev, state)
    _call("lccrf_conv", dev, _lib().lccrf_conv, _Rows(x.data_ptr(), strides[0], strides[1]), dt, pw, pb, ps, plen, B, N, D, K, out.data_ptr(), final.data_ptr())
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
    dt, dev, D, K, strides, pw, pb, ps = _conv_args(x, weight, bias, state)
    shape, dtype, device = x.shape, x.dtype, x.device
    dstrides = _activation(dout, "dout", shape, dtype, dev)
    B, N, _ = shape
    plen = _lengths(lengths, B, dev)
    g = ConvGrad(_like(x), _like(weight), None if bias is None else _like(bias), None if state is None else _like(state))
    ws = _scratch(_bytes("lccrf_conv_grad_workspace_bytes", B, N, D, K), "lccrf_conv_grad", device, workspace)
    _call("lccrf_conv_grad", dev, _lib().lccrf_conv_grad, _Rows(dout.data_ptr(), dstrides[0], dstrides[1]), _Rows(x.data_ptr(), strides[0], strides[1]), dt, pw, pb,
          ps, plen, B, N, D, K, *[0 if t is None else t.data_ptr() for t in g], ws.data_ptr(), ws.numel())
    return g


def lccrf_conv_step(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor], state: torch.Tensor, *,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One position of every stream: x [B, D], state [B, K-1, D], which moves on in place; the result is [B, D]."""
    if x.dim() != 2:
        raise ValueError(f"x must be [B, D], got {list(x.shape)}")
    if state is None:
        raise ValueError("state is missing")
    dt, dev, D, K, strides, pw, pb, ps = _conv_args(x, weight, bias, state)
    shape = x.shape
    out = _result(out, "out", x.shape, x.dtype, None, dev, x)
    _call("lccrf_conv_step", dev, _lib().lccrf_conv_step, x.data_ptr(), strides[0], dt, pw, pb, ps, shape[0], D, K, out.data_ptr())
    return out


def _scan_args(x, dt, A, Bm, Cm, D, z, dt_bias):
    """Checks what all calls of the scan share; (dtype's code, device number, channels, S, G, shape of x, dtype, the inputs' block)."""
    code, dtype, dev = _first(x, "x")
    shape = x.shape
    if 0 in shape or max(shape) > _MOST or A.dim() != 2 or Bm.dim() != len(shape) + 1:
        raise ValueError(f"x must be [B, N, D], its sizes at most {_MOST}, A [D, S] and Bm [B, N, G, S] (one position: [B, D] and [B, G, S]), got {list(shape)}, {list(A.shape)} "
                         f"and {list(Bm.shape)}")
    width, S, G = shape[-1], A.shape[1], Bm.shape[-2]
    if not 1 <= S <= MAX_STATES:
        raise ValueError(f"1 to {MAX_STATES} states a channel are served, got {S}")
    if G < 1 or width % G:
        raise ValueError(f"{width} channels cannot be shared by {G} groups")
    vectors = (*shape[:-1], G, S)
    xs, ts, bs, cs, zs, pz = x.stride(), dt.stride(), Bm.stride(), Cm.stride(), (0, 0, 1), 0
    if z is not None:
        zs, pz = z.stride(), z.data_ptr()
    # all at once; one by one only to say what is wrong
    if not (dt.shape == shape and Bm.shape == vectors and Cm.shape == vectors and dt.dtype is dtype and Bm.dtype is dtype and Cm.dtype is dtype
            and xs[-1] == ts[-1] == bs[-1] == cs[-1] == zs[-1] == 1 and dt.get_device() == Bm.get_device() == Cm.get_device() == dev
            and (z is None or (z.shape == shape and z.dtype is dtype and z.get_device() == dev))):
        for t, name, want in ((x, "x", shape), (dt, "dt", shape), (Bm, "Bm", vectors), (Cm, "Cm", vectors), (z, "z", shape)):
            if t is not None:
                _activation(t, name, want, dtype, dev)
    f32 = torch.float32
    # (one position: the second stride is that of the channels, which nothing looks at)
    return code, dev, width, S, G, shape, dtype, _ScanInputs(
        x.data_ptr(), xs[0], xs[1], dt.data_ptr(), ts[0], ts[1], Bm.data_ptr(), bs[0], bs[1], Cm.data_ptr(), cs[0], cs[1], pz, zs[0], zs[1],
        bs[-2], cs[-2], _dense(A, "A", (width, S), f32, dev), _dense(D, "D", (width,), f32, dev, True), _dense(dt_bias, "dt_bias", (width,), f32, dev, True))


def state_scan_saved(x: torch.Tensor, A: torch.Tensor) -> torch.Tensor:
    """Device memory for ``saved=`` of ``lccrf_state_scan`` on x [B, N, D] and A [D, S]: what the gradient would otherwise compute
    again.  To be kept until ``lccrf_state_scan_grad`` has it; its layout is the library's."""
    if x.dim() != 3 or A.dim() != 2 or A.shape[0] != x.shape[2] or max(x.shape) > _MOST or A.shape[1] > MAX_STATES:
        raise ValueError(f"x must be [B, N, D], its sizes at most {_MOST}, and A [D, S] of at most {MAX_STATES} states, got {list(x.shape)} and {list(A.shape)}")
    return _scratch(_bytes("lccrf_state_scan_saved_bytes", *x.shape, A.shape[1]), "state_scan_saved", x.device, None)


def _saved_ptr(saved, shape, S, dev: int) -> int:
    if saved is None:
        return 0
    if saved.dtype != torch.uint8 or saved.get_device() != dev or not saved.is_contiguous() or \
            saved.numel() < _bytes("lccrf_state_scan_saved_bytes", *shape, S):
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
    code, dev, width, S, G, shape, dtype, block = _scan_args(x, dt, A, Bm, Cm, D, z, dt_bias)
    (B, N, _), device, f32 = shape, x.device, torch.float32
    plen = _lengths(lengths, B, dev)
    pstate = _dense(state, "state", (B, width, S), f32, dev, True)
    psaved = _saved_ptr(saved, shape, S, dev)
    out = _result(out, "out", x.shape, x.dtype, None, dev, x)
    final = _result(final, "final", (B, width, S), f32, device, dev, state)
    ws = _scratch(_bytes("lccrf_state_scan_workspace_bytes", B, N, width, S, G), "lccrf_state_scan", device, workspace)
    _call("lccrf_state_scan", dev, _lib().lccrf_state_scan, block, code, plen, B, N, width, S, G, pstate, out.data_ptr(), final.data_ptr(), psaved, ws.data_ptr(),
          ws.numel())
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
    code, dev, width, S, G, shape, dtype, block = _scan_args(x, dt, A, Bm, Cm, D, z, dt_bias)
    strides = _activation(dout, "dout", shape, dtype, dev)
    (B, N, _), device, f32 = shape, x.device, torch.float32
    plen = _lengths(lengths, B, dev)
    pstate = _dense(state, "state", (B, width, S), f32, dev, True)
    psaved = _saved_ptr(saved, shape, S, dev)

    g = ScanGrad(_like(x), _like(x), _like(Bm), _like(Cm), *[None if t is None else _like(t) for t in (z, A, D, dt_bias, state)])
    ws = _scratch(_bytes("lccrf_state_scan_grad_workspace_bytes", B, N, width, S, G, int(saved is not None)), "lccrf_state_scan_grad", device, workspace)
    _call("lccrf_state_scan_grad", dev, _lib().lccrf_state_scan_grad, _Rows(dout.data_ptr(), strides[0], strides[1]), block, code, plen, B, N, width, S, G, pstate,
          psaved, _ScanGrads(*[0 if t is None else t.data_ptr() for t in g]), ws.data_ptr(), ws.numel())
    return g


def lccrf_state_step(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, Bm: torch.Tensor, Cm: torch.Tensor, D: Optional[torch.Tensor],
                     z: Optional[torch.Tensor], dt_bias: Optional[torch.Tensor], state: torch.Tensor, *,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One position of every stream: x, dt, z [B, D], Bm, Cm [B, G, S]; state float32 [B, D, S] moves on in place; the result is [B, D]."""
    if x.dim() != 2:
        raise ValueError(f"x must be [B, D], got {list(x.shape)}")
    code, dev, width, S, G, shape, dtype, block = _scan_args(x, dt, A, Bm, Cm, D, z, dt_bias)
    B = shape[0]
    pstate = _dense(state, "state", (B, width, S), torch.float32, dev)
    out = _result(out, "out", x.shape, x.dtype, None, dev, x)
    _call("lccrf_state_step", dev, _lib().lccrf_state_step, block, code, B, width, S, G, pstate, out.data_ptr())
    return out
