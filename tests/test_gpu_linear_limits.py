"""The operators of a linear attention layer at the ends of their range: heads that grow in chunks that are not full and behind the first, values
far from 1, outputs that a call names or leaves out."""
import ctypes

import pytest
import torch

import gpu_util as gu
import layer_forms as lf
import linear_forms as f

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _n(*s, seed=0, std=1.0, to=BF):
    return (torch.randn(*s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + sum(s))) * std).to(to)


def _by_length(leaves, decay, up, got, dtype, steps):
    """Every head's outputs and gradients, finite and by the length of their difference: bf16 outputs have two roundings a term (a weight, or a
    state as an operand: half a step of 2^-8 each, 2^-7 together) and their own half step, 2^-6 with what partly cancels; what is fp32 has
    `steps` half steps of 2^-24."""
    ref = [lf.f64(t) for t in leaves]
    ro = f.linear(*ref[:3], decay.double().cpu(), *ref[3:])
    rg = lf.grads(ro, [u.double().cpu() for u in up], ref)
    for name, a, r in zip(("o", "hT", "dq", "dk", "dv", "dh0"), got, tuple(ro) + tuple(rg)):
        a, r = a.detach().double().cpu(), r.detach()
        for h in range(len(decay)):
            x, y = (a[:, :, h], r[:, :, h]) if name not in ("hT", "dh0") else (a[:, h], r[:, h])
            assert x.isfinite().all(), (name, h)
            off = float((x - y).norm() / y.norm())
            assert off < (2.0 ** -6 if dtype == BF and name not in ("hT", "dh0") else steps * lf.ULP), (name, h, off)


def _grown(T, g, dk, dv, dtype):
    """A call through autograd with heads that grow, against the formula in 64 bits.  e^(|g| T) is at most e^80: an exponent costs two half steps
    of its size, 160 together over all chunks, sums of up to 128 products one each."""
    from paper_2606_08804_b200 import autograd as qa
    H, decay = len(g), torch.tensor(g, device="cuda")
    assert max(g) * T <= 80
    q, k = (_n(2, T, H, dk, seed=i, std=dk ** -0.5, to=dtype).requires_grad_() for i in range(2))
    v, h0 = _n(2, T, H, dv, seed=3, to=dtype).requires_grad_(), _n(2, H, dk, dv, seed=4, to=F32).requires_grad_()
    leaves, up = (q, k, v, h0), (_n(2, T, H, dv, seed=5, to=dtype), _n(2, H, dk, dv, seed=6, to=F32))
    o, hT = qa.linear_attention(q, k, v, decay, h0)
    _by_length(leaves, decay, up, (o, hT) + torch.autograd.grad((o, hT), leaves, up), dtype, 2 * 80 + 128)


# ---- heads that grow --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,g", [(1, [60.0, 2.0]), (2, [40.0, 3.0]), (10, [2.0, 4.0, 8.0]), (20, [1.42, 2.0, 4.0]), (50, [1.5, 1.4, 0.8])])
@pytest.mark.parametrize("dk,dv,dtype", [(128, 128, F32), (64, 64, F32), (64, 128, F32), (128, 64, BF), (64, 64, BF)])
def test_few_tokens_of_heads_that_grow_fast(T, g, dk, dv, dtype):
    """A chunk that is not full: past its end factors would be infinite, and nothing there may meet them."""
    _grown(T, g, dk, dv, dtype)
