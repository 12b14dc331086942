"""Backward of convolution and scan over tensors of more than 2^32 elements: the tokens at either end are what the formulas give for them.

Between them lie a million tokens of zeros that pass the recurrences through; an offset that lost its upper bits would meet the other end."""
import pytest
import torch

import scan_exact as sx
from test_gpu_conv_exact import _exact

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
T, D, N, HEAD, TAIL = (1 << 20) + 40, 4096, 4, 50, 100


def _n(*s, seed=0, std=1.0, to=BF):
    return (torch.randn(*s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) * std).to(to)


def _ends(width, seed, head=True):
    """[1, T, width] bf16 with numbers in the first HEAD and the last TAIL + 3 tokens, zeros between."""
    x = torch.zeros(1, T, *width, dtype=BF, device="cuda")
    if head:
        x[:, :HEAD] = _n(1, HEAD, *width, seed=seed)
    x[:, -TAIL - 3:] = _n(1, TAIL + 3, *width, seed=seed + 1)
    return x


def test_convolution_backward():
    from paper_2606_08804_b200 import binding as qd
    x, dy, w = _ends((D,), 1), _ends((D,), 3, head=False), _n(D, 4, seed=5, std=.5)
    dy[:, -TAIL - 3:-TAIL] = 0
    g = qd.conv_bwd(x, w, None, None, dy, None, silu=True)
    tail, before, up = x[:, -TAIL:].contiguous(), x[:, -TAIL - 3:-TAIL].contiguous(), dy[:, -TAIL:].contiguous()
    want, _ = _exact(tail, w, None, before, up, None, True, 2000)
    sx.close("dx", g["dx"][:, -TAIL:], *want["dx"])
    sx.close("dx before", g["dx"][:, -TAIL - 3:-TAIL], *want["dstate"])
    sx.close("dw", g["dw"], *want["dw"])
    assert not g["dx"][:, :1000].any() and not g["dx"][:, T // 2:T // 2 + 1000].any()


def test_scan_backward():
    from paper_2606_08804_b200 import binding as qd
    u, dy = _ends((D,), 1), _ends((D,), 3, head=False)
    Bm, Cm = _ends((1, N), 5), _ends((1, N), 7)
    dt = torch.zeros(1, T, D, dtype=BF, device="cuda")
    dt[:, -TAIL:] = (_n(1, TAIL, D, seed=9, to=F32) * 0.7 - 3).exp().to(BF)
    for t in (u, dy, Bm, Cm):
        t[:, -TAIL - 3:-TAIL] = 0
    a = dict(u=u, dt=dt, A=-_n(D, N, seed=10, std=.5, to=F32).exp(), Bm=Bm, Cm=Cm)
    y, hT, ws = qd.scan_fwd(**a, save_for_bwd=True)
    part = {n: t[:, -TAIL:].contiguous() if t.dim() > 2 else t for n, t in a.items()}
    # segments: a sum of steps that are 0 but for the last TAIL
    want = sx.scan(**part, dy=dy[:, -TAIL:], cut=(TAIL, TAIL))
    sx.close("y", y[:, -TAIL:], *want["y"])
    sx.close("hT", hT, *want["hT"])
    assert not y[:, :-TAIL].any()
    del y
    g = qd.scan_bwd(**a, D=None, z=None, dt_bias=None, h0=None, dy=dy, workspace=ws, reuse_fwd=True, want_dh0=True)
    for name in ("du", "ddt", "dBm", "dCm"):
        sx.close(name, g[name][:, -TAIL:], *want[name])
    sx.close("dA", g["dA"], *want["dA"])
    sx.close("dh0", g["dh0"], *want["dh0"])                # steps of 0 hand it on as it is
    for name in ("du", "dBm", "dCm"):
        assert not g[name][:, :1000].any() and not g[name][:, T // 2:T // 2 + 1000].any(), name
    # the gradient of a step of 0: u <g, B>, with g as it leaves the tail
    gB = (want["dh0"][0][:, None] * Bm[:, :HEAD].double()).sum(-1)
    size = ((want["dh0"][1][:, None] + 20 * sx.E * want["dh0"][0].abs()[:, None]) * Bm[:, :HEAD].double().abs()).sum(-1)
    sx.close("ddt of the head", g["ddt"][:, :HEAD], gB * u[:, :HEAD].double(), size * u[:, :HEAD].double().abs() + 1e-36)
    assert not g["ddt"][:, HEAD:HEAD + 1000].any()
