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
