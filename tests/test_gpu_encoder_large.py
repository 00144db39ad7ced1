"""The encoder at sizes near its limits, and at those from which on it takes other kernels than test_gpu_encoder.py's cases do."""
import pytest
import torch

from test_gpu_encoder import DEV, U, _dirty_memory, crf, generator, normal  # noqa: F401

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1024  # positions of a call


def alike(t, want, roundings):
    """One value everywhere: half a step of its type, and the roundings on the way."""
    half = torch.finfo(t.dtype).eps / 2
    worst = max(abs(float(v) - want) for v in (t.min(), t.max()))
    assert worst <= (half + roundings * U) * abs(want), f"{float(t.min())} .. {float(t.max())} for {want}"


def test_the_longest_sequence(crf):
    """One position repeated: what the operators settle at, and where they begin and end."""
    t = torch.bfloat16
    x = torch.full((1, 1, 1), 1.5, dtype=t, device=DEV).expand(1, MOST, 1)
    silu = lambda v: v * torch.sigmoid(v)  # noqa: E731
    w, pre = torch.tensor([[0.25, 0.5]], device=DEV), torch.tensor([0.75, 1.125], dtype=torch.float64)
    out, final = crf.lccrf_conv(x, w)
    alike(out[:, :1], float(silu(pre[0])), 20)
    alike(out[:, 1:], float(silu(pre[1])), 20)
    assert final.item() == 1.5
    dout = torch.full((1, 1, 1), -0.5, dtype=t, device=DEV).expand(1, MOST, 1)
    g = crf.lccrf_conv_grad(dout, x, w)
    gate = torch.sigmoid(pre)
    first, dpre = (-0.5 * gate * (1 + pre * (1 - gate))).tolist()
    alike(g.dx[:, :1], 0.5 * first + 0.25 * dpre, 30)
    alike(g.dx[:, 1:-1], 0.75 * dpre, 30)
    alike(g.dx[:, -1:], 0.5 * dpre, 30)
    alike(g.dweight, 1.5 * dpre * MOST, 2 ** 14)  # a thread adds 64 positions of 64 runs, a channel 16 x 128 workgroups of 256 threads
    del out, g


def test_the_longest_scan(crf):
    t = torch.bfloat16
    x, Bm, Cm, dout = (torch.full((1, 1, 1), v, dtype=t, device=DEV).expand(1, MOST, 1) for v in (1.5, 0.5, 2.0, -0.5))
    vectors = Bm[..., None], Cm[..., None]
    dt, A, D = torch.zeros(1, 1, 1, dtype=t, device=DEV).expand(1, MOST, 1), torch.full((1, 1), -0.5, device=DEV), torch.full((1,), 0.25, device=DEV)
    step = float(torch.log(torch.tensor(2.0, dtype=torch.float64)))
    a = 2.0 ** -0.5
    saved = crf.state_scan_saved(x, A)
    out, final = crf.lccrf_state_scan(x, dt, A, *vectors, D, saved=saved)
    h = step * 1.5 * 0.5 / (1 - a)
    alike(out[:, :1], 2.0 * step * 1.5 * 0.5 + 0.25 * 1.5, 40)
    alike(out[:, 400:], 2.0 * h + 0.25 * 1.5, 40)
    alike(final, h, 40)
    del out
    g = crf.lccrf_state_scan_grad(dout, x, dt, A, *vectors, D, saved=saved)
    dh = -0.5 * 2.0 / (1 - a)  # away from both ends
    dput, back = dh * 0.5, dh * a * h
    inner = slice(400, MOST - 400)
    alike(g.dx[:, inner], dput * step + 0.25 * -0.5, 80)
    alike(g.dx[:, -1:], -0.5 * 2.0 * 0.5 * step + 0.25 * -0.5, 80)
    alike(g.ddt[:, inner], (dput * 1.5 + back * -0.5) * 0.5, 1000)  # a difference twelve times smaller than what it is of
    alike(g.dBm[:, inner], dh * step * 1.5, 80)
    alike(g.dCm[:, inner], -0.5 * h, 80)
    alike(g.dD, -0.5 * 1.5 * MOST, 2 ** 20 + 400)  # a wave adds a segment's positions, 3072 of them are joined
    alike(g.dA, back * step * MOST, 2 ** 20 + 400)
