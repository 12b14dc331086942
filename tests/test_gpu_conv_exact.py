"""The short convolution over long runs of tokens (the loop without edges, forward and backward), element by element against 64 bits.

Bounds to first order in e = 2^-24: a sum of k products in a row is off by k e of the sum of their sizes; a function of the special function
unit by 4 e, its argument's rounding by 2 |x| e; |SiLU'| <= 1.1, |SiLU''| <= 1/2.  The weights' gradients are added up over a run's tokens, the
threads of a CTA that share channels (128 at most) and the CTAs' parts, of which 32 threads take every 32nd.
"""
import pytest
import torch

from scan_exact import E, close, told

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _parts(B, T, D, W, dt):
    """CTAs that leave a part of the weights' gradients, and the fewest tokens that a full run of the backward can have."""
    from paper_2606_08804_b200 import binding as qd
    gy = qd.load().qdelta_conv_workspace_bytes(B, T, D, W, 1 if dt == BF else 0) // (4 * (W + 1) * D)
    cx, groups = 32, (D + 3) // 4
    while cx > 1 and cx // 2 >= groups:
        cx //= 2
    return gy, T // max(1, gy * (128 // cx) // B)


def _exact(x, w, b, s, dy, dl, silu, parts):
    """{name: (value, bound)}"""
    B, T, D = x.shape
    W = w.shape[1]
    x, w, b, s, dy, dl = (None if t is None else t.double() for t in (x, w, b, s, dy, dl))
    xp = torch.cat([s if s is not None else x.new_zeros(B, W - 1, D), x], 1)
    tap = [xp[:, j:j + T] for j in range(W)]
    pre = sum(w[:, j] * tap[j] for j in range(W)) + (0 if b is None else b)
    e_pre = (W + 1) * E * (sum((w[:, j] * tap[j]).abs() for j in range(W)) + (0 if b is None else b.abs()))
    y, e_y, slope, e_slope = pre, e_pre, torch.ones_like(pre), 0 * pre
    if silu:
        sig = torch.sigmoid(pre)
        y = pre * sig
        e_y = 1.1 * e_pre + y.abs() * (2 * pre.abs() + 12) * E
        slope = sig * (1 + pre * (1 - sig))
        e_slope = 0.5 * e_pre + E * (1 + pre.abs()) * (2 * pre.abs() + 16)
    d = dy * slope
    e_d = dy.abs() * e_slope + 2 * E * d.abs()
    n = T + 134 + parts / 32
    out = {"y": (y, e_y),
           "dw": (torch.stack([(d * t).sum((0, 1)) for t in tap], 1), torch.stack([((e_d + n * E * d.abs()) * t.abs()).sum((0, 1)) for t in tap], 1)),
           "dbias": (d.sum((0, 1)), (e_d + n * E * d.abs()).sum((0, 1)))}
    full, e_full = torch.zeros_like(xp), torch.zeros_like(xp)
    for j in range(W):
        full[:, j:j + T] += w[:, j] * d
        e_full[:, j:j + T] += w[:, j].abs() * (e_d + (W + 1) * E * d.abs())
    if dl is not None:
        full[:, T:] += dl
        e_full[:, T:] += E * (full[:, T:].abs() + dl.abs())
    out["dx"], out["dstate"] = (full[:, W - 1:], e_full[:, W - 1:]), (full[:, :W - 1], e_full[:, :W - 1])
    return {k: (r, 1.05 * e + 1e-36) for k, (r, e) in out.items()}, xp[:, T:]


CASES = [(8, 509, D, W, dt, silu, bias, state) for D in (4096, 4097) for dt in (BF, F32)
         for W, silu, bias, state in ((2, True, False, True), (3, False, True, True), (4, True, True, True))] + [
    (8, 700, 4096, 4, BF, False, False, False), (8, 509, 4098, 4, F32, True, True, False),
    # many sequences, each one run
    (700, 41, 200, 4, BF, True, True, True), (3000, 43, 37, 3, F32, True, True, True), (40000, 47, 7, 2, BF, False, True, True)]


@pytest.mark.parametrize("B,T,D,W,dt,silu,bias,state", CASES)
def test_long_runs(B, T, D, W, dt, silu, bias, state):
    from paper_2606_08804_b200 import binding as qd
    g = torch.Generator(device="cuda").manual_seed(D + W)
    n = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(dt)  # noqa: E731
    x, w, b, s, dy, dl = n(B, T, D), n(D, W, std=0.5), n(D, std=0.2) if bias else None, n(B, W - 1, D) if state else None, n(B, T, D), n(B, W - 1, D)
    dl = dl if state else None
    parts, run = _parts(B, T, D, W, dt)
    # backward the loop without edges begins at the 5th token of a run and ends 16 before its end; forward runs of bf16 are half as long, and
    # 8 tokens do
    assert run >= 36, run
    want, last = _exact(x, w, b, s, dy, dl, silu, parts)
    y, got_last = qd.conv_fwd(x, w, b, s, silu=silu)
    got = dict(qd.conv_bwd(x, w, b, s, dy, dl, silu=silu), y=y)
    assert torch.equal(got_last.double(), last)
    for name, (r, bound) in want.items():
        missing = (name == "dbias" and b is None) or (name == "dstate" and s is None)
        assert (got[name] is None) == missing, name
        if not missing:
            close(name, got[name], r, bound)
            assert told(name, r, bound) > 0.9, name
