"""The selective scan element by element: every output against 64 bits, each with a bound of its own (scan_exact.py), in one segment and in
several, at the sizes of a layer."""
import ctypes

import pytest
import torch

import scan_exact as sx

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _inputs(B, T, D, N, G, dt, softplus=True, gate=True, skip=True, bias=True, state=True, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + B + T + D + N)
    n = lambda *s, std=1.0, to=dt: (torch.randn(*s, device="cuda", generator=g) * std).to(to)  # noqa: E731
    wave = n(B, T, D, std=0.7, to=F32)
    return dict(u=n(B, T, D), dt=(wave - 3 if softplus else (wave - 3).exp()).to(dt),
                A=-(torch.arange(1, N + 1, device="cuda") * n(D, N, std=0.2, to=F32).exp()), Bm=n(B, T, G, N), Cm=n(B, T, G, N),
                D=n(D, to=F32) if skip else None, z=n(B, T, D) if gate else None,
                dt_bias=n(D, std=0.3, to=F32).abs() if bias else None, h0=n(B, D, N, to=F32) if state else None), \
        n(B, T, D), n(B, D, N, to=F32) if state else None


def _cut(a):
    """Tokens of the longest segment that is walked alone: at most half of a sequence, in whole tiles; none where the forward needs no
    workspace, or there are fewer tokens than two segments have."""
    from paper_2606_08804_b200 import binding as qd
    B, T, D = a["u"].shape
    s = qd.QdScanShape(B, T, D, a["A"].shape[1], a["Bm"].shape[2], 1 if a["u"].dtype == BF else 0)
    forward = qd.load().qdelta_scan_workspace_bytes(ctypes.byref(s), 0) > 0
    return (T // 2 + 16 if forward else 0), (T // 2 + 16 if T >= 64 else 0)


def _check(a, dy, dhT, softplus=True, expect_cut=None, ref=None, grads=True):
    """Forward and backward of `a` against the values and bounds of `ref` (default: `a` itself)."""
    from paper_2606_08804_b200 import binding as qd
    cut = _cut(a)
    if expect_cut is not None:
        assert (cut[0] > 0) == expect_cut
    want = sx.scan(**(ref or a), softplus=softplus, dy=dy if grads else None, dhT=dhT, cut=cut)
    y, hT, ws = qd.scan_fwd(**a, softplus=softplus, save_for_bwd=grads)
    got = {"y": y, "hT": hT}
    if grads:
        got.update(qd.scan_bwd(**a, dy=dy, dhT=dhT, workspace=ws, reuse_fwd=True, softplus=softplus))
    absent = {"d" + n for n, t in a.items() if t is None}
    for name, t in got.items():
        assert (t is None) == (name in absent), name
        if t is not None:
            sx.close(name, t, *want[name])
    return want


CASES = [  # B, T, D, N, G, dtype, softplus, gate, skip, bias, state, the forward cut into segments
    (1, 2500, 20, 16, 1, F32, True, True, True, True, True, True), (4, 1301, 43, 3, 43, BF, True, True, True, True, True, None),
    (2, 606, 50, 2, 50, F32, True, True, True, True, True, None), (1, 1503, 64, 2, 64, BF, True, True, True, True, True, True),
    (5, 303, 40, 4, 40, F32, True, False, True, True, True, None), (1, 4096, 512, 16, 1, BF, True, True, True, True, True, True),
    (1, 777, 2048, 16, 1, BF, True, True, True, True, True, True), (2, 1000, 512, 16, 2, F32, True, True, True, True, True, True),
    (1, 8191, 96, 16, 1, F32, False, True, False, False, True, True), (1, 3001, 40, 33, 2, BF, True, False, True, False, False, True),
    (1, 2049, 72, 64, 1, F32, True, True, True, True, True, True), (2, 1500, 130, 24, 1, BF, True, True, False, True, True, True),
    # as many CTAs as have room at once and more: one segment, or a short one beside a long one
    (8, 200, 2048, 16, 1, BF, True, True, True, True, True, None), (10, 300, 2048, 16, 1, F32, True, True, True, True, False, None),
    (37, 90, 256, 16, 1, BF, True, True, True, True, True, None), (6, 410, 1024, 40, 1, BF, True, True, True, True, True, None)]


@pytest.mark.parametrize("B,T,D,N,G,dt,softplus,gate,skip,bias,state,cut", CASES)
def test_every_element(B, T, D, N, G, dt, softplus, gate, skip, bias, state, cut):
    a, dy, dhT = _inputs(B, T, D, N, G, dt, softplus, gate, skip, bias, state)
    want = _check(a, dy, dhT, softplus, cut)
    for name, (r, bound) in want.items():                  # and the bounds are no excuse: nearly no element could be missing
        assert sx.told(name, r, bound) > 0.9, name


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65])
@pytest.mark.parametrize("dt", [BF, F32])
def test_around_the_tiles(T, dt):
    a, dy, dhT = _inputs(2, T, 36, 16, 1, dt, seed=T)
    _check(a, dy, dhT)


@pytest.mark.parametrize("B,D,N,G,S,dt", [(5, 36, 16, 3, 3, BF), (256, 64, 16, 1, 1, F32), (3, 40, 64, 1, 8, BF), (1, 7, 5, 7, 2, F32)])
def test_steps(B, D, N, G, S, dt):
    from paper_2606_08804_b200 import binding as qd
    a, _, _ = _inputs(B, S, D, N, G, dt)
    want = sx.scan(**a, softplus=True)
    state = a.pop("h0").clone()
    y = qd.scan_steps(**a, state=state, softplus=True)
    sx.close("y", y, *want["y"])
    sx.close("state", state, *want["hT"])


@pytest.mark.parametrize("B,T,D,N,dt", [(1, 5001, 24, 16, F32), (2, 33, 70, 5, BF), (1, 2000, 64, 64, BF), (200, 70, 64, 16, F32)])
def test_steps_of_zero_leave_the_state(B, T, D, N, dt):
    """Tokens masked by a step of 0 (a padded batch): the state's bits, however many there are."""
    from paper_2606_08804_b200 import binding as qd
    a, _, _ = _inputs(B, T, D, N, 1, dt, softplus=False, bias=False)
    a["dt"].zero_()
    h0 = a["h0"]
    y, hT, _ = qd.scan_fwd(**a)
    assert torch.equal(hT, h0)
    state = h0.clone()
    few = {n: t[:, :3].contiguous() if n in ("u", "dt", "Bm", "Cm", "z") else t for n, t in a.items() if n != "h0"}
    qd.scan_steps(**few, state=state)
    assert torch.equal(state, h0)
