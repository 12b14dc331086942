"""The 64-bit forms that the operators around the delta rule are tested against: their gradients against differences, and closed forms."""
import math

import pytest
import torch

import layer_forms as lf


def _r(*s, seed=0):
    return torch.randn(*s, dtype=torch.float64, generator=torch.Generator().manual_seed(seed + sum(s))).requires_grad_()


@pytest.mark.parametrize("W,silu,state", [(2, False, False), (3, True, True), (4, True, True)])
def test_convolution(W, silu, state):
    x, w, b, s = _r(2, 5, 3), _r(3, W), _r(3), _r(2, W - 1, 3) if state else None
    assert torch.autograd.gradcheck(lambda *a: lf.conv(*a, silu=silu), (x, w, b, s))
    if not silu and not state:
        y, _ = lf.conv(x, w, b)
        want = torch.nn.functional.conv1d(torch.nn.functional.pad(x.transpose(1, 2), (W - 1, 0)), w[:, None], b, groups=3).transpose(1, 2)
        assert torch.allclose(y, want, rtol=1e-12, atol=1e-12)


def test_scan_differences_and_closed_form():
    B, T, D, N, G = 2, 4, 4, 3, 2
    a = (_r(B, T, D), _r(B, T, D, seed=1), _r(D, N, seed=2), _r(B, T, G, N, seed=3), _r(B, T, G, N, seed=4), _r(D), _r(B, T, D, seed=5),
         _r(D, seed=6), _r(B, D, N, seed=7))
    assert torch.autograd.gradcheck(lambda *x: lf.scan(*x, softplus=True), a)
    # constant step and input: h_t = B x (1 - a^t) / (1 - a)
    one = lambda *s: torch.ones(*s, dtype=torch.float64)  # noqa: E731
    A = torch.tensor([[-0.5]], dtype=torch.float64)
    y, h = lf.scan(one(1, 6, 1), one(1, 6, 1) * 0.2, A, one(1, 6, 1, 1), one(1, 6, 1, 1))
    e = math.exp(-0.1)
    assert abs(float(h) - 0.2 * (1 - e ** 6) / (1 - e)) < 1e-13 and abs(float(y[0, -1, 0]) - float(h)) < 1e-15


@pytest.mark.parametrize("rms", [False, True])
def test_norm(rms):
    x, w, b = _r(3, 6), _r(6), _r(6, seed=1)
    assert torch.autograd.gradcheck(lambda *a: lf.norm(*a, rms=rms), (x, w, b))
    if not rms:
        assert torch.allclose(lf.norm(x, w, b), torch.nn.functional.layer_norm(x, (6,), w, b), rtol=1e-12, atol=1e-12)
