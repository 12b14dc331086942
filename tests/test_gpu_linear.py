"""Linear attention, gated norm, norm behind a residual sum and rotary positions against their 64-bit forms, at the sizes where kernels go
wrong, every element with a bound of its own: half a step of its type, and what the roundings on the way may cost.  They are counted on the
same operator of absolute values (M: no cancellation, so the sum of the terms' sizes).
"""
import math

import pytest
import torch

import layer_forms as lf
import linear_forms as f

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _abs(t):
    return None if t is None else t.detach().abs().requires_grad_()


# ---- linear attention -------------------------------------------------------------------------------------------------------
LINEAR = [  # B, T, H, dk, dv, dtype, state
    (1, 1, 1, 64, 64, F32, False), (2, 1, 3, 128, 128, BF, True), (1, 2, 2, 64, 128, BF, True), (3, 63, 2, 128, 64, F32, True),
    (2, 64, 2, 64, 64, BF, False), (1, 65, 3, 128, 128, F32, True), (2, 127, 2, 128, 128, BF, True), (1, 128, 5, 64, 64, BF, True),
    (2, 129, 2, 128, 64, BF, True), (1, 130, 2, 64, 128, F32, True), (2, 257, 3, 64, 128, BF, True), (1, 300, 4, 128, 128, BF, False),
    (2, 333, 4, 64, 64, F32, True), (1, 700, 2, 128, 128, BF, True), (1, 1025, 3, 128, 128, F32, True), (1, 1537, 4, 64, 64, BF, True),
    (1, 1300, 2, 128, 64, BF, True), (1, 1300, 3, 64, 128, BF, False), (40, 70, 4, 64, 64, BF, True)]


def _linear_inputs(B, T, H, dk, dv, dt, state, seed=0):
    r = _gen(seed + T)
    n = lambda *s, std=1.0, to=dt: (torch.randn(*s, device="cuda", generator=r) * std).to(to)  # noqa: E731
    g = [-0.003, -math.inf, -0.7, 0.0, -0.05][:H] + [-0.01] * (H - 5)
    return (n(B, T, H, dk, std=dk ** -0.5), n(B, T, H, dk, std=dk ** -0.5), n(B, T, H, dv), torch.tensor(g, device="cuda"),
            n(B, H, dk, dv, std=0.3, to=F32) if state else None), n(B, T, H, dv), n(B, H, dk, dv, std=0.3, to=F32)


def _rounds(T, dk, dv, dt, state_out=False):
    """fp32: products of three planes (2^-22 together) summed over a head, then over a chunk, by an instruction that cuts (two half steps
    each); a sum a chunk; factors whose exponent is at most 20 where they count.  bf16: a term's weight is rounded to bf16 once, half a step of
    2^-8; or, where it has gone into the state, the state has been as an operand, and before that the term cut at 2^-15: 2^-7 and 2^-16 hold
    either; a state that is returned has terms of three planes of 8 bits, 24 together."""
    n = 2 * (max(dk, dv) + 128) + 4 * (T // 64 + 1) + 100
    return n * lf.ULP + (0 if dt == F32 or state_out else 2.0 ** -7 + 2.0 ** -16)


@pytest.mark.parametrize("B,T,H,dk,dv,dt,state", LINEAR)
def test_linear(B, T, H, dk, dv, dt, state):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    (q, k, v, g, h0), dO, dh = _linear_inputs(B, T, H, dk, dv, dt, state)
    scale, gd = -0.75, g.double().cpu()
    ref = [lf.f64(t) for t in (q, k, v, h0)]
    ro, rh = f.linear(*ref[:3], gd, ref[3], scale)
    up = [dO.double().cpu(), dh.double().cpu() if state else None]
    rg = lf.grads((ro, rh), up, ref)
    mag = [_abs(t) for t in ref]
    mo, mh = f.linear(*mag[:3], gd, mag[3], abs(scale))
    mg = lf.grads((mo, mh), [_abs(u) for u in up], mag)
    o, hT, ws = qd.linear_fwd(q, k, v, g, h0, scale)
    out, st = _rounds(T, dk, dv, dt), _rounds(T, dk, dv, dt, True)
    lf.close("o", o, ro, out * mo.detach())
    lf.close("hT", hT, rh, st * mh.detach())
    assert qd.workspace_status(ws) == 0
    gr = qd.linear_bwd(q, k, v, g, h0, dO, dh if state else None, scale)
    for name, r, m, s in zip(("dq", "dk", "dv", "dh0"), rg, mg, (out, out, out, st)):
        assert (gr[name] is None) == (r is None)
        if r is not None:
            lf.close(name, gr[name], r, s * m)
    have = [t.requires_grad_() for t in (q, k, v, h0) if t is not None]
    ao, ah = qa.linear_attention(q, k, v, g, h0, scale)
    assert torch.equal(ao, o) and torch.equal(ah, hT)
    got = torch.autograd.grad((ao, ah) if state else (ao,), have, (dO, dh) if state else (dO,))
    for name, a in zip(("dq", "dk", "dv", "dh0"), got):
        assert torch.equal(a, gr[name]), name


@pytest.mark.parametrize("B,T,H,dk,dv,dt", [(1, 300, 6, 128, 128, BF), (2, 257, 6, 64, 64, BF), (1, 130, 6, 64, 128, F32), (1, 140, 6, 128, 64, BF),
                                            (1, 1300, 6, 64, 64, BF), (1, 700, 6, 128, 128, F32)])
@pytest.mark.parametrize("decay", [[-0.9, -3.0, -0.7, -0.7000001, -20.0, -100.0], [0.01, 0.0, -1e-6, 1e-30, -0.6999999, 0.004]], ids=["steep", "slight"])
def test_linear_with_decays_of_every_size(B, T, H, dk, dv, dt, decay):
    """Heads that forget within a few tokens, on both sides of where a row's factor is taken out of a chunk, and heads that grow (e^(g T) is at
    most e^13 here: the exponents that count are at most 20)."""
    from paper_2606_08804_b200 import binding as qd
    (q, k, v, _, h0), dO, dh = _linear_inputs(B, T, H, dk, dv, dt, True, seed=5)
    g = torch.tensor(decay, device="cuda")
    ref, mag = [lf.f64(t) for t in (q, k, v, h0)], [_abs(lf.f64(t)) for t in (q, k, v, h0)]
    ro, rh = f.linear(*ref[:3], g.double().cpu(), ref[3], 1.25)
    mo, mh = f.linear(*mag[:3], g.double().cpu(), mag[3], 1.25)
    rg = lf.grads((ro, rh), (dO.double().cpu(), dh.double().cpu()), ref)
    mg = lf.grads((mo, mh), (dO.double().cpu().abs(), dh.double().cpu().abs()), mag)
    still = torch.zeros_like(g).double().cpu()
    whole = [_abs(lf.f64(t)) for t in (q, k, v, h0)]
    wo, wh = f.linear(*whole[:3], still, whole[3], 1.25)
    wg = lf.grads((wo, wh), (dO.double().cpu().abs(), dh.double().cpu().abs()), whole)
    o, hT, ws = qd.linear_fwd(q, k, v, g, h0, 1.25)
    out, st = _rounds(T, dk, dv, dt), _rounds(T, dk, dv, dt, True)
    low = 2.0 ** -126
    lf.close("o", o, ro, out * mo.detach() + low * (wo.detach() + T))
    lf.close("hT", hT, rh, st * mh.detach() + low * (wh.detach() + T))
    gr = qd.linear_bwd(q, k, v, g, h0, dO, dh, 1.25)
    for name, r, m, s, w in zip(("dq", "dk", "dv", "dh0"), rg, mg, (out, out, out, st), wg):
        lf.close(name, gr[name], r, s * m + low * (w + T))
    assert qd.workspace_status(ws) == 0


@pytest.mark.parametrize("T,dk,dv", [(3000, 64, 64), (2900, 128, 128)])
def test_slow_heads_keep_their_rate(T, dk, dv):
    """A factor that is rounded once and multiplied in for every chunk is off by the same amount each time.  What may be left of n chunks of 64 is
    their sums' and the state's own rounding, of any sign: 2 sqrt(n) half steps of the state's length."""
    from paper_2606_08804_b200 import binding as qd
    (q, k, v, _, h0), _, _ = _linear_inputs(1, T, 2, dk, dv, F32, True, seed=7)
    g = torch.tensor([-1e-4, -3e-4], device="cuda")
    _, hT, _ = qd.linear_fwd(q, k, v, g, h0)
    n, g64 = torch.arange(T - 1, -1, -1, device="cuda").double(), g.double()
    ref = torch.einsum("hi,bihd,bihv->bhdv", torch.exp(g64[:, None] * n), k.double(), v.double()) + torch.exp(g64 * T)[:, None, None] * h0.double()
    assert float((hT.double() - ref).norm() / ref.norm()) < 2 * math.sqrt(T / 64) * lf.ULP


@pytest.mark.parametrize("B,H,dk,dv,dt", [(1, 1, 64, 64, F32), (3, 5, 128, 128, BF), (2, 3, 64, 128, BF), (2, 2, 128, 64, F32), (40, 16, 128, 128, BF)])
def test_linear_steps_go_on_from_a_prompt(B, H, dk, dv, dt):
    from paper_2606_08804_b200 import binding as qd
    (q, k, v, g, h0), _, _ = _linear_inputs(B, 13, H, dk, dv, dt, True)
    ref, mag = [lf.f64(t) for t in (q, k, v, h0)], None
    ro, rh = f.linear(*ref[:3], g.double().cpu(), ref[3], 0.5)
    mag = [_abs(t) for t in ref]
    mo, mh = f.linear(*mag[:3], g.double().cpu(), mag[3], 0.5)
    state, one, os, at = h0.clone(), h0.clone(), [], 0
    for n in (1, 2, 9, 1):
        os.append(qd.linear_steps(*(t[:, at:at + n].contiguous() for t in (q, k, v)), g, state, scale=0.5))
        at += n
    # a state passes three roundings a token, a read-out's sum one a row
    lf.close("o", torch.cat(os, 1), ro, (4 * 13 + dk + 40) * lf.ULP * mo.detach())
    lf.close("state", state, rh, (4 * 13 + 40) * lf.ULP * mh.detach())
    for t in range(13):                                   # several tokens a call: the bits of one at a time
        assert torch.equal(qd.linear_steps(*(x[:, t:t + 1].contiguous() for x in (q, k, v)), g, one, scale=0.5), torch.cat(os, 1)[:, t:t + 1])
    assert torch.equal(one, state)
    o = torch.empty_like(v[:, :1].contiguous())
    assert qd.linear_steps(*(t[:, :1].contiguous() for t in (q, k, v)), g, h0.clone(), o, scale=0.5) is o and torch.equal(o, os[0])


# ---- norms ------------------------------------------------------------------------------------------------------------------
NORM = [  # rows, width, dtype, rms, weight, bias, other (SiLU, or a scale)
    (1, 1, F32, False, True, True, True), (3, 2, BF, True, True, False, True), (33, 7, F32, False, True, True, False), (700, 8, BF, False, True, True, True),
    (5, 9, BF, False, False, False, True), (300, 64, F32, True, True, False, False), (4099, 128, BF, True, True, False, True),
    (65, 129, BF, False, True, True, True), (257, 200, F32, False, False, True, True), (31, 256, BF, False, True, True, False),
    (64, 257, BF, True, True, True, True), (100, 1000, F32, False, True, True, True), (129, 1001, BF, False, True, False, True),
    (700, 2048, BF, False, True, True, True), (9, 2049, F32, True, True, True, True), (17, 4096, F32, False, True, True, False),
    (3, 5000, BF, False, True, True, True), (5, 8192, BF, True, True, True, False), (2, 16383, F32, False, True, True, True),
    (3, 16384, BF, False, True, True, True), (3, 16384, F32, False, True, True, True), (2, 16383, BF, True, True, True, True),
    (1500, 130, BF, False, True, True, True), (1300, 36, F32, True, True, True, True), (311, 6000, BF, True, True, False, True)]


def _rows(rows, width, dt):
    r = _gen(rows + width)
    n = lambda *s, std=1.0: torch.randn(*s, device="cuda", generator=r) * std  # noqa: E731
    x = (n(rows, width) * n(rows, 1, std=0.5).exp() + 0.3).to(dt)
    if rows > 2:
        x[1] = 0                                   # a row without deviation
    return n, x


def _stats(t, rms, eps):
    return 1 / torch.sqrt((t if rms else t - t.mean(-1, keepdim=True)).square().mean(-1, keepdim=True) + eps)


def _top(t):
    return t.abs().amax(-1, keepdim=True)


def _compare(name, got, ref, slack):
    assert (got is None) == (ref is None), name
    if ref is not None:
        lf.close(name, got, ref, slack)


@pytest.mark.parametrize("rows,width,dt,rms,weight,bias,silu", NORM)
def test_gated_norm(rows, width, dt, rms, weight, bias, silu):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    n, x = _rows(rows, width, dt)
    z, w, b, dy = n(rows, width, std=3).to(dt), (1 + n(width, std=0.2)).to(dt) if weight else None, n(width, std=0.2).to(dt) if bias else None, n(rows, width).to(dt)
    z[0, 0] = 100.0
    z[-1, -1] = -100.0
    eps = 1e-3
    ref = [lf.f64(t) for t in (x, z, w, b)]
    ry = f.gated_norm(*ref, eps=eps, rms=rms, silu=silu)
    rg = lf.grads((ry,), (dy.double().cpu(),), ref)
    xd, zd, dyd = ref[0].detach(), ref[1].detach(), dy.double().cpu()
    # A row's sums pass below 200 roundings (64 terms in a thread, a tree of 10, the products around them), of values as large as |x|
    # before the mean is taken off, times r.  A sigmoid has the relative error of e^-z: |z| half steps and ten more; |z| <= 20 where it counts.
    r = _stats(xd, rms, eps)
    size, fz = _top(xd) * r, f.gate(zd, silu).abs()
    wm, bm = float(w.abs().max()) if weight else 1.0, float(b.abs().max()) if bias else 0.0
    k = (230 + 2 * zd.abs().clamp(max=20)) * lf.ULP
    N = size * wm * (1 + size) + bm
    y, stats = qd.gated_norm_fwd(x, z, w, b, eps, rms=rms, silu=silu)
    tiny = 1e-37                                   # what the special function unit takes for 0
    lf.close("y", y, ry, k * N * fz + tiny)
    g = qd.gated_norm_bwd(x, z, w, b, dy, stats, rms=rms, silu=silu)
    gm = _top(dyd * fz) * wm
    kr = 270 * lf.ULP
    _compare("dx", g["dx"], rg[0], kr * r * gm * (1 + size) ** 2 + tiny)
    _compare("dgate", g["dgate"], rg[1], k * dyd.abs() * N * (1 + zd.abs() if silu else 1) + tiny)
    kw = (270 + rows) * lf.ULP
    _compare("dweight", g["dweight"], rg[2], kw * ((dyd * fz).abs() * size * (1 + size)).sum(0) + tiny)
    _compare("dbias", g["dbias"], rg[3], kw * (dyd * fz).abs().sum(0) + tiny)
    have = [t.requires_grad_() for t in (x, z, w, b) if t is not None]
    ay = qa.gated_norm(x, z, w, b, eps, rms=rms, silu=silu)
    assert torch.equal(ay, y)
    names = [m for m, t in zip(("dx", "dgate", "dweight", "dbias"), (x, z, w, b)) if t is not None]
    for m, t, got in zip(names, have, torch.autograd.grad(ay, have, dy)):
        assert got.dtype == t.dtype and torch.equal(got, g[m].to(t.dtype)), m


@pytest.mark.parametrize("rows,width,dt,rms,weight,bias,scaled", NORM)
def test_add_norm(rows, width, dt, rms, weight, bias, scaled):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    n, e = _rows(rows, width, dt)
    x, c = n(rows, width).to(dt), (n(width, std=0.3) + 0.5).to(dt) if scaled else None
    w, b = (1 + n(width, std=0.2)).to(dt) if weight else None, n(width, std=0.2).to(dt) if bias else None
    dy, dt_ = n(rows, width).to(dt), n(rows, width).to(dt)
    eps = 1e-3
    ref = [lf.f64(t) for t in (x, e, c, w, b)]
    ry, rt = f.add_norm(*ref, eps=eps, rms=rms)
    ups = (dy.double().cpu(), dt_.double().cpu())
    rg = lf.grads((ry, rt), ups, ref)
    xd, cd, dyd, dtd = ref[0].detach(), ref[2].detach() if scaled else torch.ones(width, dtype=torch.float64), *ups
    # as for the gated norm, with what is added in place of x
    r, parts = _stats(rt.detach(), rms, eps), ref[1].detach().abs() + (cd * xd).abs()
    size = _top(parts) * r
    wm, bm = float(w.abs().max()) if weight else 1.0, float(b.abs().max()) if bias else 0.0
    k = 230 * lf.ULP
    y, total, stats = qd.add_norm_fwd(x, e, c, w, b, eps, rms=rms)
    lf.close("total", total, rt, 2 * lf.ULP * parts)
    lf.close("y", y, ry, k * (size * wm * (1 + size) + bm))
    g = qd.add_norm_bwd(x, e, c, w, dy, dt_, stats, rms=rms, want_dbias=bias)
    gm = _top(dyd) * wm
    off = r * gm * k * (1 + size) ** 2 + 4 * lf.ULP * dtd.abs()
    _compare("dresidual", g["dresidual"], rg[1], off)
    _compare("dx", g["dx"], rg[0], off * cd.abs())
    d = rg[1].detach().abs() + off
    _compare("dscale", g["dscale"], rg[2], ((off + rows * lf.ULP * d) * xd.abs()).sum(0))
    _compare("dweight", g["dweight"], rg[3], (k + rows * lf.ULP) * (dyd.abs() * size * (1 + size)).sum(0))
    _compare("dbias", g["dbias"], rg[4], (k + rows * lf.ULP) * dyd.abs().sum(0))
    if not scaled:
        assert g["dx"] is g["dresidual"]
    alone = qd.add_norm_bwd(x, e, c, w, dy, None, stats, rms=rms, want_dscale=False, want_dweight=False)
    assert alone["dscale"] is None and alone["dweight"] is None
    lf.close("norm alone", alone["dresidual"], rg[1] - dtd, off)
    have = [t.requires_grad_() for t in (x, e, c, w, b) if t is not None]
    ay, at = qa.add_norm(x, e, c, w, b, eps, rms=rms)
    assert torch.equal(ay, y) and torch.equal(at, total)
    names = [m for m, t in zip(("dx", "dresidual", "dscale", "dweight", "dbias"), (x, e, c, w, b)) if t is not None]
    for m, t, got in zip(names, have, torch.autograd.grad((ay, at), have, (dy, dt_))):
        assert got.dtype == t.dtype and torch.equal(got, g[m].to(t.dtype)), m


# ---- rotary -----------------------------------------------------------------------------------------------------------------
ROTARY = [  # B, T, Hq, Hk, d, pairs, dtype, interleaved, positions
    (1, 1, 1, 0, 2, 1, F32, False, "count"), (2, 3, 2, 1, 64, 32, BF, False, "start"), (1, 5, 3, 3, 64, 32, F32, True, "far"),
    (3, 1, 16, 4, 128, 32, BF, True, "far"), (2, 9, 4, 2, 128, 64, BF, False, "far"), (1, 7, 2, 2, 65, 32, BF, False, "count"),
    (1, 7, 2, 1, 65, 31, F32, True, "start"), (2, 33, 3, 1, 80, 20, BF, False, "far"), (2, 33, 3, 1, 80, 22, BF, True, "far"),
    (1, 4, 5, 0, 7, 3, BF, True, "count"), (1, 4, 5, 2, 7, 3, F32, False, "count"), (1, 3, 2, 2, 1024, 512, BF, False, "far"),
    (1, 2, 3, 1, 1024, 100, F32, True, "far"), (1, 700, 2, 1, 32, 16, BF, False, "start"), (1, 1, 300, 30, 128, 64, BF, False, "far"),
    (5, 40, 1, 1, 12, 6, BF, False, "far"), (5, 40, 1, 1, 20, 2, F32, False, "far"), (2, 260, 7, 3, 96, 48, BF, True, "count")]


@pytest.mark.parametrize("B,T,Hq,Hk,d,pairs,dt,interleaved,at", ROTARY)
def test_rotary(B, T, Hq, Hk, d, pairs, dt, interleaved, at):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    r = _gen(d + T)
    n = lambda *s: torch.randn(*s, device="cuda", generator=r).to(dt)  # noqa: E731
    q, k, scale = n(B, T, Hq, d), n(B, T, Hk, d) if Hk else None, 0.8
    turns = qd.rotary_turns(pairs, factor=2.0)
    start = {"count": 0, "start": 123456789, "far": -77}[at]
    pos = torch.randint(-(1 << 40), 1 << 40, (B, T), device="cuda", generator=r) if at == "far" else None
    where = pos.flatten().tolist() if pos is not None else [start + t for _ in range(B) for t in range(T)]
    ang = f.angles(turns.tolist(), where).reshape(B, T, pairs)
    how = dict(positions=pos, start=start, interleaved=interleaved, scale=scale)
    got = qd.rotary(q, k, turns, **how)
    # sine and cosine: 4 half steps of 1, two products and a sum
    slack = lambda x: 8 * lf.ULP * scale * _pair_size(x, pairs, interleaved)  # noqa: E731
    for x, y in zip((q, k), got):
        assert (x is None) == (y is None)
        if x is not None:
            lf.close("out", y, f.rotary(x.double().cpu(), ang, interleaved, scale), slack(x))
            assert torch.equal(y[..., 2 * pairs:], x[..., 2 * pairs:])
    back = qd.rotary(got[0], got[1], turns, inverse=True, **dict(how, scale=1.0))
    for x, y in zip((q, k), back):
        if x is not None:        # there and back: two roundings of the type
            ref = torch.cat((x[..., :2 * pairs].double().cpu() * scale, x[..., 2 * pairs:].double().cpu()), -1)
            lf.close("back", y, ref, (16 * lf.ULP + 2 * lf.HALF[dt]) * _pair_size(x, pairs, interleaved))
    place = [x.clone() if x is not None else None for x in (q, k)]
    same = qd.rotary(*place, turns, out=place, **how)
    assert same[0].data_ptr() == place[0].data_ptr()
    for y, p in zip(got, place):
        assert y is None or torch.equal(y, p)
    have = [t.requires_grad_() for t in (q, k) if t is not None]
    a = [t for t in qa.rotary(q, k, turns, **how) if t is not None]
    assert all(torch.equal(x, y) for x, y in zip(a, got))
    ups = [n(*t.shape) for t in a]
    g = torch.autograd.grad(a, have, ups)
    want = qd.rotary(ups[0], ups[1] if Hk else None, turns, inverse=True, **how)
    assert all(torch.equal(x, y) for x, y in zip(g, want))
    if Hk:                        # gradient of the keys alone
        only = torch.autograd.grad(qa.rotary(q, k, turns, **how)[1], have, ups[1], allow_unused=True)
        assert only[0] is None and torch.equal(only[1], want[1])


def _pair_size(x, pairs, interleaved):
    """|a| + |b| of the pair that an element belongs to; 0 behind the pairs."""
    m = x.detach().double().cpu().abs()
    if interleaved:
        s = m[..., 0:2 * pairs:2] + m[..., 1:2 * pairs:2]
        both = torch.stack((s, s), -1).flatten(-2)
    else:
        s = m[..., :pairs] + m[..., pairs:2 * pairs]
        both = torch.cat((s, s), -1)
    return torch.cat((both, torch.zeros_like(m[..., 2 * pairs:])), -1)
