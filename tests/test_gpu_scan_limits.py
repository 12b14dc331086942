"""The selective scan at the ends of the number range: what the formulas give in 64 bits, in tokens that there are and behind the last."""
import pytest
import torch

import scan_exact as sx
from test_gpu_scan_exact import _cut, _inputs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("low", [float("-inf"), -torch.finfo(F32).max, -2.5e38])
@pytest.mark.parametrize("B,T,D,N,dt", [(2, 17, 20, 5, F32), (1, 333, 24, 16, BF), (1, 5, 3, 1, BF), (3, 8, 40, 33, F32), (1, 16, 16, 16, F32)])
def test_states_that_forget_at_every_step(B, T, D, N, dt, low):
    """A of minus infinity (a parameter's exponential that overflowed) or near the lowest number: the decay of every step above 0 is 0.
    2^(A dt) is 0 from A = -1e30 on, so that this stands for it in 64 bits, where 0 times infinity in the gradients would be none."""
    from paper_2606_08804_b200 import binding as qd
    a, dy, dhT = _inputs(B, T, D, N, 1, dt)
    a["A"][:, N - 1] = low
    a["A"][D // 2] = low
    ref = dict(a, A=a["A"].clamp(min=-1e30))
    want = sx.scan(**ref, softplus=True, dy=dy, dhT=dhT, cut=_cut(a))
    y, hT, ws = qd.scan_fwd(**a, softplus=True, save_for_bwd=True)
    got = dict(qd.scan_bwd(**a, dy=dy, dhT=dhT, workspace=ws, reuse_fwd=True, softplus=True), y=y, hT=hT)
    for name, (r, bound) in want.items():
        sx.close(name, got[name], r, bound)
    # single tokens, among them one whose step is 0: it leaves the state
    few = {n: t[:, :3].contiguous() if n in ("u", "dt", "Bm", "Cm", "z") else t for n, t in a.items()}
    few["dt"][:, 1:2] = float("-inf")                          # softplus: 0
    want = sx.scan(**dict(few, A=ref["A"], dt=few["dt"].clamp(min=-1e4)), softplus=True)
    state = few.pop("h0").clone()
    y = qd.scan_steps(**few, state=state, softplus=True)
    sx.close("y", y, *want["y"])
    sx.close("state", state, *want["hT"])
    y, hT, _ = qd.scan_fwd(**few, h0=a["h0"], softplus=True)
    sx.close("y", y, *want["y"])
    sx.close("hT", hT, *want["hT"])


@pytest.mark.parametrize("T", [900, 4000])                    # ends joined by each segment itself, and by a kernel of its own
@pytest.mark.parametrize("dt", [BF, F32])
def test_states_of_zero_that_would_have_grown(T, dt):
    """A positive, and nothing in the state till the last tokens (a batch padded in front): zero times a growth that overflows is zero.
    Backward likewise from a gradient that is zero till the first tokens."""
    from paper_2606_08804_b200 import binding as qd
    a, dy, _ = _inputs(1, T, 24, 4, 1, dt, softplus=False, bias=False, state=False)
    a["A"] = (-a["A"]).clamp(min=0.6, max=8)
    a["dt"].fill_(8)
    a["dt"][:, :20] = a["dt"][:, -20:] = 0.0625
    a["u"][:, :-20] = 0
    dy[:, 20:] = 0
    assert _cut(a)[0] > 0 and float(a["A"].min()) * 8 * 32 > 100           # a segment has 32 tokens at least
    last = {n: t[:, -20:].contiguous() if n in ("u", "dt", "Bm", "Cm", "z") else t for n, t in a.items()}
    want = sx.scan(**last)
    y, hT, ws = qd.scan_fwd(**a, save_for_bwd=True)
    sx.close("y", y[:, -20:], *want["y"])
    sx.close("hT", hT, *want["hT"])
    assert not y[:, :-20].any()
    g = qd.scan_bwd(**a, dy=dy, dhT=torch.zeros_like(hT), workspace=ws, reuse_fwd=True)
    first = {n: t[:, :20].contiguous() if n in ("u", "dt", "Bm", "Cm", "z") else t for n, t in a.items()}
    want = sx.scan(**first, dy=dy[:, :20])
    for name in ("du", "ddt", "dBm", "dCm", "dz"):
        sx.close(name, g[name][:, :20], *want[name])
    for name in ("du", "dBm"):                             # what later tokens send back: nothing
        assert not g[name][:, 20:].any(), name
    sx.close("dA", g["dA"], want["dA"][0], want["dA"][1])
