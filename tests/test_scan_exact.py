"""The written-out gradients of the scan against those of autograd through its 64-bit form, and what their bounds notice."""
import pytest
import torch

import layer_forms as lf
import scan_exact as sx


def _inputs(B, T, D, N, G, softplus, everything):
    g = torch.Generator().manual_seed(T)
    n = lambda *s: torch.randn(*s, dtype=torch.float64, generator=g)  # noqa: E731
    opt = lambda t: t if everything else None  # noqa: E731
    return dict(u=n(B, T, D), dt=n(B, T, D) - 3 if softplus else (n(B, T, D) - 3).exp(), A=-n(D, N).exp(), Bm=n(B, T, G, N), Cm=n(B, T, G, N), D=opt(n(D)),
                z=opt(n(B, T, D)), dt_bias=opt(n(D)), h0=opt(n(B, D, N))), n(B, T, D), opt(n(B, D, N))


@pytest.mark.parametrize("B,T,D,N,G,softplus,everything", [(2, 7, 6, 3, 2, True, True), (1, 40, 4, 5, 1, False, True), (2, 9, 4, 2, 4, True, False), (1, 1, 2, 1, 1, True, True)])
def test_values(B, T, D, N, G, softplus, everything):
    a, dy, dhT = _inputs(B, T, D, N, G, softplus, everything)
    got = sx.scan(**a, softplus=softplus, dy=dy, dhT=dhT)
    leaves = {k: t.clone().requires_grad_() if t is not None else None for k, t in a.items()}
    outs = lf.scan(**leaves, softplus=softplus)
    want = dict(zip(("y", "hT"), outs), **{"d" + k: t for k, t in zip(leaves, lf.grads(outs, (dy, dhT), list(leaves.values()))) if t is not None})
    for k, t in want.items():
        assert torch.allclose(got[k][0], t, rtol=1e-10, atol=1e-12), k
        assert (got[k][1] >= 0).all() and (got[k][1] < 1e-2 * got[k][0].abs().max() + 1e-12).all(), k


def test_bounds_hold_for_fp32_and_notice_a_lost_state():
    """The same formulas in fp32, operation by operation, are inside; a segment that forgets the state before it is not."""
    a, dy, _ = _inputs(1, 400, 8, 4, 1, True, True)
    a = {k: t.float() if t is not None else None for k, t in a.items()}
    want = sx.scan(**a, softplus=True, dy=dy.float(), cut=(216, 216))
    y, hT = lf.scan(**a, softplus=True)
    sx.close("y", y, *want["y"])
    sx.close("hT", hT, *want["hT"])
    half = lambda lo, hi, h: lf.scan(**{k: t[:, lo:hi] if k in ("u", "dt", "Bm", "Cm", "z") else t for k, t in a.items() if k != "h0"}, h0=h, softplus=True)  # noqa: E731
    first, h = half(0, 200, a["h0"])
    sx.close("y", torch.cat([first, half(200, 400, h)[0]], 1), *want["y"])
    for wrong in (torch.zeros_like(h), h * (1 + 1e-3)):
        with pytest.raises(AssertionError, match="y: "):
            sx.close("y", torch.cat([first, half(200, 400, wrong)[0]], 1), *want["y"])
