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


@pytest.mark.parametrize("T,g", [(140, [0.55, 0.2, 0.17]), (160, [0.5, 0.4, 0.1]), (175, [0.45, 0.3, 0.01]), (460, [0.17, 0.1733, 0.1734]), (1500, [0.05, 0.03, 0.0])])
@pytest.mark.parametrize("dk,dv,dtype", [(128, 128, BF), (64, 64, BF), (64, 128, BF), (128, 64, F32)])
def test_heads_that_grow_over_several_chunks(T, g, dk, dv, dtype):
    """States of up to e^80 meet no factor but those of the rows that there are."""
    _grown(T, g, dk, dv, dtype)


# ---- values far from 1 ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("powers", [(45, 45, -90), (-45, -45, 90), (-90, 0, 90), (90, 0, -90)])
@pytest.mark.parametrize("T,dk,dv,dtype", [(100, 128, 128, BF), (300, 64, 64, BF), (270, 64, 128, BF), (260, 128, 64, BF), (130, 64, 64, F32)])
def test_weights_and_states_far_from_one(T, dk, dv, dtype, powers):
    """Weights q k and dO v, and states, of 2^-90 to 2^90, with outputs that are ordinary numbers; heads on both sides of where a row's factor is taken
    out of a chunk.  A term's bounds are those of any size.  What is below 2^-126 may be lost; where the row's factor is multiplied in last, what
    is below 2^-110."""
    from paper_2606_08804_b200 import binding as qd
    decay = torch.tensor([-0.69, -0.45, -0.174, -0.173, -0.01, 0.02], device="cuda")
    H, (pq, pk, pv), scale = len(decay), powers, 0.75
    q, k, v = _n(1, T, H, dk, std=2.0 ** pq, to=dtype), _n(1, T, H, dk, seed=1, std=2.0 ** pk, to=dtype), _n(1, T, H, dv, seed=2, std=2.0 ** pv, to=dtype)
    h0, dO, dhT = _n(1, H, dk, dv, std=2.0 ** (pk + pv), to=F32), _n(1, T, H, dv, seed=3, to=dtype), _n(1, H, dk, dv, seed=4, std=2.0 ** pq, to=F32)
    ref = [lf.f64(t) for t in (q, k, v, h0)]
    mag = [t.detach().abs().requires_grad_() for t in ref]
    up, gd = [t.double().cpu() for t in (dO, dhT)], decay.double().cpu()
    r, m = f.linear(*ref[:3], gd, ref[3], scale), f.linear(*mag[:3], gd, mag[3], scale)
    r, m = tuple(r) + tuple(lf.grads(r, up, ref)), tuple(m) + tuple(lf.grads(m, [t.abs() for t in up], mag))
    o, hT, ws = qd.linear_fwd(q, k, v, decay, h0, scale)
    g = qd.linear_bwd(q, k, v, decay, h0, dO, dhT, scale)
    # sums and factors as in test_gpu_linear.py: exponents that count are at most 20
    n = (2 * (max(dk, dv) + 128) + 4 * (T // 64 + 1) + 100) * lf.ULP
    bits, low = (n, 2.0 ** -124) if dtype == F32 else (n + 2.0 ** -7 + 2.0 ** -16, 2.0 ** -110)
    top = lambda t: float(t.float().abs().max())  # noqa: E731
    for i, (name, got, a, b, c) in enumerate((("o", o, q, k, v), ("hT", hT, None, k, None), ("dq", g["dq"], dO, v, k), ("dk", g["dk"], v, dO, q),
                                              ("dv", g["dv"], k, q, dO), ("dh0", g["dh0"], None, q, None))):
        if a is None:            # a term's planes, times the other factor
            lf.close(name, got, r[i], n * m[i].detach() + T * 2.0 ** -124 * top(b))
        else:                    # a weight, times its row of c; an element of the state, times its one of a
            lf.close(name, got, r[i], bits * m[i].detach() + low * (T * top(c) + 128 * top(a)))
    assert qd.workspace_status(ws) == 0


# ---- outputs that a call names or leaves out --------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,width,to", [(33, 64, BF), (40, 36, F32), (7, 129, BF), (300, 2048, BF), (9, 9000, BF), (9, 5001, BF), (5, 4097, F32)])
def test_residual_norm_without_a_scale_writes_both_gradients(rows, width, to):
    """dx has a buffer of its own although it is dresidual: it is written, too."""
    from paper_2606_08804_b200 import binding as qd
    lib, code, stream = qd.load(), 1 if to == BF else 0, torch.cuda.current_stream().cuda_stream
    x, e, dy, dt = (_n(rows, width, seed=i, to=to) for i in range(4))
    w = _n(width, seed=5, to=to)
    _, _, stats = qd.add_norm_fwd(x, e, None, w)
    want = qd.add_norm_bwd(x, e, None, w, dy, dt, stats)
    n = lib.qdelta_fused_norm_workspace_bytes(rows, width, code)
    dx, dr, dw = gu.Guarded((rows, width), to), gu.Guarded((rows, width), to), gu.Guarded((width,), F32)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    p = lambda t: t.data_ptr()  # noqa: E731
    assert lib.qdelta_add_norm_bwd(rows, width, code, p(x), p(e), None, p(w), p(dy), p(dt), p(stats), p(dx.t), p(dr.t), None, p(dw.t), None, p(ws), n, 0, stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(dr.t, want["dresidual"]) and torch.equal(dx.t, want["dresidual"]) and torch.equal(dw.t, want["dweight"])
    assert dx.intact() and dr.intact() and dw.intact()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_constant_initial_state_gets_no_gradient(dtype):
    """No memory for it, and the other gradients are those of a call that does not ask for it."""
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    B, T, H, d = 64, 20, 16, 128
    q, k, v, dO = (_n(B, T, H, d, seed=i, std=0.3, to=dtype) for i in range(4))
    decay, h0 = -torch.linspace(0.01, 0.9, H, device="cuda"), _n(B, H, d, d, to=F32)
    leaves = [t.requires_grad_() for t in (q, k, v)]
    o, _ = qa.linear_attention(q, k, v, decay, h0)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    got = torch.autograd.grad(o, leaves, dO)
    used = torch.cuda.max_memory_allocated() - before
    assert used < 3 * q.numel() * q.element_size() + h0.numel() * 2, used
    want = qd.linear_bwd(*(t.detach() for t in leaves), decay, h0, dO, want_dh0=False)
    assert want["dh0"] is None and all(torch.equal(a, want[n]) for a, n in zip(got, ("dq", "dk", "dv")))
    h0.requires_grad_()                                                  # asked for, it comes
    o, _ = qa.linear_attention(q, k, v, decay, h0)
    assert torch.equal(torch.autograd.grad(o, h0, dO)[0], qd.linear_bwd(*(t.detach() for t in leaves), decay, h0.detach(), dO)["dh0"])


def test_a_state_of_zero_stays_zero_whatever_a_head_grows_by():
    """Long sequences that begin with tokens of zeros (a padded batch): across a segment of them a head's factor is beyond fp32, 0 times it is 0."""
    from paper_2606_08804_b200 import binding as qd
    T, H, d, real = 32768, 2, 64, 700
    decay = torch.tensor([0.1, 0.02], device="cuda")
    for dtype in (BF, F32):
        q, k, v, dO = (_n(1, T, H, d, seed=i, std=0.3, to=dtype) for i in range(4))
        for t in (k, v, dO):
            t[:, :-real] = 0
        o, hT, _ = qd.linear_fwd(q, k, v, decay)
        g = qd.linear_bwd(q, k, v, decay, None, dO)
        assert not o[:, :-real].any() and not g["dq"][:, :-real].any()
        ref = [lf.f64(t[:, -real:]) for t in (q, k, v)]
        ro = f.linear(*ref, decay.double().cpu())
        rg = lf.grads(ro, [dO[:, -real:].double().cpu(), None], ref)
        for name, a, r in zip(("o", "hT", "dq", "dk", "dv"), (o[:, -real:], hT, g["dq"][:, -real:], g["dk"][:, -real:], g["dv"][:, -real:]), ro + tuple(rg)):
            a, r = a.double().cpu(), r.detach()
            assert a.isfinite().all(), name
            off = float((a - r).norm() / r.norm())
            # exponents of at most 70 in two half steps each, a rounding a chunk and sums of 64, or bf16's two roundings a term and its own
            assert off < (2.0 ** -6 if dtype == BF and name != "hT" else (140 + 128 + 40) * lf.ULP), (name, off)
