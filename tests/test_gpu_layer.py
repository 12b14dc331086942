"""Convolution, selective scan and layer norm against their 64-bit forms, at the sizes where kernels go wrong.

Tolerances: half a step of the output's type, plus what rounding each 32-bit operation may cost.  The second is counted as
n 2^-24 M: M the largest value of the same operator on the absolute values of its inputs (no cancellation, so a bound on the sum
of the terms' sizes), n the number of roundings that one term passes through.  A sum of k terms in any order passes each through at
most k roundings; exponentials and quotients are counted as 4.
"""
import pytest
import torch

import layer_forms as lf

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _abs(t):
    return None if t is None else t.detach().abs().requires_grad_()


def _most(t):
    return float(t.detach().abs().max())


# ---- convolution ------------------------------------------------------------------------------------------------------------
CONV = [  # B, T, D, W, dtype, silu, bias, state
    (1, 1, 1, 2, BF, False, False, False), (1, 1, 8, 4, BF, True, True, True), (2, 2, 7, 4, F32, True, True, True),
    (3, 3, 64, 4, BF, True, False, True), (2, 5, 257, 3, F32, False, True, True), (1, 130, 40, 3, BF, True, True, False),
    (2, 509, 36, 2, F32, True, False, False), (1, 1025, 24, 4, BF, False, True, True), (5, 33, 2056, 4, BF, True, True, True),
    (40, 4, 72, 4, BF, True, False, True), (1, 4099, 3, 3, F32, True, True, True), (2, 300, 1001, 4, BF, True, True, True)]


def _conv_inputs(B, T, D, W, dt, bias, state, seed=0):
    g = _gen(seed)
    n = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(dt)  # noqa: E731
    return n(B, T, D), n(D, W, std=0.5), n(D, std=0.2) if bias else None, n(B, W - 1, D) if state else None, n(B, T, D), n(B, W - 1, D)


@pytest.mark.parametrize("B,T,D,W,dt,silu,bias,state", CONV)
def test_convolution(B, T, D, W, dt, silu, bias, state):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    x, w, b, s, dy, dl = _conv_inputs(B, T, D, W, dt, bias, state)
    ref = [lf.f64(t) for t in (x, w, b, s)]
    ry, rl = lf.conv(*ref, silu=silu)
    up = [dy.double().cpu(), dl.double().cpu() if state else None]
    rg = lf.grads((ry, rl), up, ref)
    mag = [_abs(t) for t in ref]
    my, ml = lf.conv(*mag, silu=silu)
    mg = lf.grads((my, ml), [_abs(u) for u in up], mag)
    y, last = qd.conv_fwd(x, w, b, s, silu=silu)
    # the sum, its SiLU (slope at most 1.1, the sigmoid of |pre| at least half of any) and the gradient's factors: 3 W + 20 roundings,
    # twice for the factor; the weights' sums run over B T terms more
    k = 2.5 * (3 * W + 20) * lf.ULP
    lf.close("y", y, ry, k * _most(my))
    assert torch.equal(last.double().cpu(), rl.detach())
    g = qd.conv_bwd(x, w, b, s, dy, dl if state else None, silu=silu)
    kw = 2.5 * (3 * W + 20 + B * T) * lf.ULP
    for name, r, m, kk in (("dx", rg[0], mg[0], k), ("dw", rg[1], mg[1], kw), ("dbias", rg[2], mg[2], kw), ("dstate", rg[3], mg[3], k)):
        assert (g[name] is None) == (r is None)
        if r is not None:
            # d silu is at most 1.1 in size, and at least 1/2 on absolute values
            lf.close(name, g[name], r, kk * 1.2 * _most(m))
    for t in (x, w, b, s):
        if t is not None:
            t.requires_grad_()
    ay, al = qa.short_conv(x, w, b, s, silu=silu)
    assert torch.equal(ay, y) and torch.equal(al, last)
    have = [t for t in (x, w, b, s) if t is not None]
    names = [n for n, t in zip(("dx", "dw", "dbias", "dstate"), (x, w, b, s)) if t is not None]
    got = torch.autograd.grad((ay, al) if state else (ay,), have, (dy, dl) if state else (dy,))
    for n, t, a in zip(names, have, got):
        assert a.dtype == t.dtype and torch.equal(a, g[n].to(t.dtype)), n


@pytest.mark.parametrize("D,W,dt", [(64, 4, BF), (33, 3, F32), (7, 2, BF)])
def test_convolution_steps_go_on_from_a_prompt(D, W, dt):
    """Prompt, then tokens one by one and several at a time: the bits of one call over everything."""
    from paper_2606_08804_b200 import binding as qd
    x, w, b, s, _, _ = _conv_inputs(3, 40, D, W, dt, True, True)
    y, last = qd.conv_fwd(x, w, b, s, silu=True)
    y0, state = qd.conv_fwd(x[:, :30].contiguous(), w, b, s, silu=True)
    got, at = [y0], 30
    for n in (1, 1, 2, 5, 1):
        got.append(qd.conv_steps(x[:, at:at + n].contiguous(), w, b, state, silu=True))
        at += n
    assert at == 40 and torch.equal(torch.cat(got, 1), y) and torch.equal(state, last)


# ---- scan -------------------------------------------------------------------------------------------------------------------
SCAN = [  # B, T, D, N, G, dtype, softplus, gate, skip, bias, state
    (1, 1, 1, 1, 1, F32, True, True, True, True, True), (2, 7, 3, 3, 1, BF, True, True, True, True, False),
    (1, 8, 16, 16, 1, F32, False, False, False, False, True), (2, 9, 20, 16, 2, F32, True, True, True, True, True),
    (1, 17, 64, 16, 1, BF, True, True, True, True, True), (3, 33, 40, 17, 1, F32, True, False, True, True, True),
    (1, 130, 66, 16, 2, F32, True, True, False, True, True), (2, 300, 100, 8, 1, BF, True, True, True, True, True),
    (1, 700, 8, 4, 1, F32, True, True, True, True, True), (1, 333, 24, 64, 3, F32, True, True, True, False, True),
    (2, 129, 130, 33, 1, BF, False, True, True, True, True), (1, 200, 36, 48, 2, BF, True, True, True, True, False),
    (1, 64, 4, 16, 4, F32, True, True, True, True, True), (1, 1025, 32, 16, 1, F32, True, False, False, True, True),
    (1, 2500, 20, 16, 1, F32, True, True, True, True, True),         # more segments than one joins by itself
    # segments of unequal lengths backward; in both directions; more CTAs than have room at once
    (5, 303, 40, 4, 40, F32, True, True, True, True, True), (4, 1301, 43, 3, 43, BF, True, True, True, True, True),
    (2, 606, 50, 2, 50, F32, True, True, True, True, True), (1, 1503, 64, 2, 64, BF, True, True, True, True, True),
    # whole groups of channels that do not fill a CTA, of 16, 32 and 64 states
    (1, 410, 136, 16, 1, BF, True, True, True, True, True), (1, 333, 24, 64, 3, BF, True, True, True, True, True),
    (2, 150, 80, 32, 2, BF, True, True, True, True, True), (1, 410, 76, 20, 1, F32, True, True, True, True, True)]


def _scan_inputs(B, T, D, N, G, dt, softplus, gate, skip, bias, state, seed=0):
    g = _gen(seed)
    n = lambda *s, std=1.0, to=dt: (torch.randn(*s, device="cuda", generator=g) * std).to(to)  # noqa: E731
    wave = n(B, T, D, std=0.7, to=F32)
    return dict(u=n(B, T, D), dt=(wave - 3 if softplus else (wave - 3).exp()).to(dt),
                A=-(torch.arange(1, N + 1, device="cuda") * n(D, N, std=0.2, to=F32).exp()), Bm=n(B, T, G, N), Cm=n(B, T, G, N),
                D=n(D, to=F32) if skip else None, z=n(B, T, D) if gate else None,
                dt_bias=n(D, std=0.3, to=F32).abs() if bias else None, h0=n(B, D, N, to=F32) if state else None), \
        n(B, T, D), n(B, D, N, to=F32)


@pytest.mark.parametrize("B,T,D,N,G,dt,softplus,gate,skip,bias,state", SCAN)
def test_scan(B, T, D, N, G, dt, softplus, gate, skip, bias, state):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    a, dy, dh = _scan_inputs(B, T, D, N, G, dt, softplus, gate, skip, bias, state)
    ref = {n: lf.f64(t) for n, t in a.items()}
    ry, rh = lf.scan(**ref, softplus=softplus)
    up = [dy.double().cpu(), dh.double().cpu() if state else None]
    rg = dict(zip(ref, lf.grads((ry, rh), up, list(ref.values()))))
    # decays keep their sign, what they multiply does not; steps likewise
    mag = {n: t if n in ("A", "dt", "dt_bias") else _abs(t) for n, t in ref.items()}
    my, mh = lf.scan(**mag, softplus=softplus)
    mg = dict(zip(mag, lf.grads((my, mh), [_abs(u) for u in up], list(mag.values()))))
    y, hT, ws = qd.scan_fwd(**a, softplus=softplus, save_for_bwd=True)
    # a state passes ten roundings a token (its exponent's size, below 8 where the decay counts, is in them twice), a sum over N states
    # or D channels one a term, the gate and the softplus ten each
    k = (10 * T + 2 * N + 40) * lf.ULP
    lf.close("y", y, ry, 2 * k * _most(my))
    lf.close("hT", hT, rh, k * _most(mh))
    g = qd.scan_bwd(**a, dy=dy, dhT=dh if state else None, workspace=ws, reuse_fwd=True, softplus=softplus)
    kg = 2.5 * (20 * T + 2 * N + 80) * lf.ULP
    more = {"dA": B * T, "dD": B * T, "ddt_bias": B * T, "dBm": D, "dCm": D}
    for n, r in rg.items():
        name = "d" + n
        assert (g[name] is None) == (r is None), name
        if r is None:
            continue
        m = mg[n]
        if n in ("dt", "dt_bias", "A"):
            # terms of both signs meet here (u <g, B> and <g p, A>): the sizes of the two, from the same walk with -A
            neg = {k_: v for k_, v in mag.items()}
            m = m.abs() + 2 * _step_terms(neg, up, softplus)[n]
        lf.close(name, g[name], r, (kg + 2.5 * more.get(name, 0) * lf.ULP) * _most(m))
    again = qd.scan_bwd(**a, dy=dy, dhT=dh if state else None, softplus=softplus)
    for name in g:
        assert (g[name] is None and again[name] is None) or torch.equal(g[name], again[name]), name
    have = [t.requires_grad_() for t in a.values() if t is not None]
    names = ["d" + n for n, t in a.items() if t is not None]
    ay, ah = qa.selective_scan(**a, softplus=softplus)
    assert torch.equal(ay, y) and torch.equal(ah, hT)
    got = torch.autograd.grad((ay, ah) if state else (ay,), have, (dy, dh) if state else (dy,))
    for n, t in zip(names, got):
        assert torch.equal(t, g[n]), n


def _step_terms(mag, up, softplus):
    """Sizes of the two sums in the gradients of dt, dt_bias and A: |u <g, B>| + |<g p, A>|, dt <g p>, on absolute values."""
    d = {n: t.detach() if t is not None else None for n, t in mag.items()}
    a = {n: t.clone().requires_grad_() if t is not None else None for n, t in d.items()}
    # the decay's part alone: the input's step held fixed
    raw = a["dt"] if a["dt_bias"] is None else a["dt"] + a["dt_bias"]
    eff = torch.log1p(torch.exp(-raw.abs())) + torch.clamp(raw, min=0) if softplus else raw
    plain = dict(a, dt=eff, dt_bias=None)
    B, T, C = d["u"].shape
    fixed = dict(plain, u=d["u"] * eff.detach(), dt=eff)
    group = torch.arange(C) // (C // d["Bm"].shape[2])
    h = d["h0"] if d["h0"] is not None else d["u"].new_zeros(B, C, d["A"].shape[1])
    ys = []
    for t in range(T):
        h = torch.exp(fixed["dt"][:, t, :, None] * a["A"]) * h + fixed["u"][:, t, :, None] * d["Bm"][:, t, group]
        y = (d["Cm"][:, t, group] * h).sum(-1)
        ys.append(y if d["z"] is None else y * d["z"][:, t] / (1 + torch.exp(-d["z"][:, t])))
    names = [n for n in ("dt", "dt_bias", "A") if a[n] is not None]
    g = lf.grads((torch.stack(ys, 1), h), [None if u is None else u.abs() for u in up], [a[n] for n in names])
    return {n: v.abs() for n, v in zip(names, g)}


@pytest.mark.parametrize("D,N,G,dt", [(64, 16, 1, BF), (30, 5, 2, F32), (24, 64, 1, F32), (40, 1, 1, BF)])
def test_scan_steps_go_on_from_a_prompt(D, N, G, dt):
    from paper_2606_08804_b200 import binding as qd
    a, _, _ = _scan_inputs(2, 90, D, N, G, dt, True, True, True, True, True)
    part = lambda lo, hi: {n: t[:, lo:hi].contiguous() if n in ("u", "dt", "Bm", "Cm", "z") else t for n, t in a.items()}  # noqa: E731
    ry, rh = lf.scan(**{n: lf.f64(t) for n, t in a.items()}, softplus=True)
    my, mh = lf.scan(**{n: t if n in ("A", "dt", "dt_bias") else _abs(t) for n, t in ((n, lf.f64(t)) for n, t in a.items())}, softplus=True)
    y0, state, _ = qd.scan_fwd(**part(0, 80), softplus=True)
    one = state.clone()
    got, at = [y0], 80
    for n in (1, 2, 7):
        p = part(at, at + n)
        p.pop("h0")
        got.append(qd.scan_steps(**p, state=state, softplus=True))
        at += n
    k = 2 * (10 * 90 + 2 * N + 40) * lf.ULP
    lf.close("y", torch.cat(got, 1), ry, k * _most(my))
    lf.close("state", state, rh, k * _most(mh))
    # several tokens a call: the bits of one at a time
    for t in range(80, 90):
        p = part(t, t + 1)
        p.pop("h0")
        y = qd.scan_steps(**p, state=one, softplus=True)
        assert torch.equal(y, torch.cat(got, 1)[:, t:t + 1])
    assert torch.equal(one, state)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("N", [1, 3, 4, 6, 8, 12, 16, 20, 31, 32, 44, 64])
def test_scan_steps_of_an_odd_batch(N, dt):
    from paper_2606_08804_b200 import binding as qd
    B, S, D, G = 5, 3, 36, 3
    a, _, _ = _scan_inputs(B, S, D, N, G, dt, True, True, True, True, True, seed=N)
    h0 = a.pop("h0")
    ry, rh = lf.scan(**{n: lf.f64(t) for n, t in a.items()}, h0=lf.f64(h0), softplus=True)
    my, mh = lf.scan(**{n: t if n in ("A", "dt", "dt_bias") else _abs(t) for n, t in ((n, lf.f64(t)) for n, t in a.items())}, h0=_abs(lf.f64(h0)), softplus=True)
    state = h0.clone()
    y = qd.scan_steps(**a, state=state, softplus=True)
    k = 2 * (10 * S + 2 * N + 40) * lf.ULP                 # as for the scan
    lf.close("y", y, ry, k * _most(my))
    lf.close("state", state, rh, k * _most(mh))
    # each sequence by itself: the same bits
    for b in range(B):
        one = h0[b:b + 1].clone()
        p = {n: t[b:b + 1].clone() if n in ("u", "dt", "Bm", "Cm", "z") else t for n, t in a.items()}
        assert torch.equal(qd.scan_steps(**p, state=one, softplus=True), y[b:b + 1])
        assert torch.equal(one, state[b:b + 1])


# ---- norm -------------------------------------------------------------------------------------------------------------------
NORM = [  # rows, width, dtype, rms, weight, bias
    (1, 1, F32, False, True, True), (3, 2, BF, True, True, False), (33, 7, F32, False, True, True), (700, 8, BF, False, True, True),
    (5, 9, BF, False, False, False), (300, 64, F32, True, True, False), (4099, 128, BF, True, True, False), (65, 129, BF, False, True, True),
    (257, 200, F32, False, False, True), (31, 256, BF, False, True, True), (64, 257, BF, True, True, True), (100, 1000, F32, False, True, True),
    (129, 1001, BF, False, True, False), (700, 2048, BF, False, True, True), (9, 2049, F32, True, True, True), (17, 4096, F32, False, True, True),
    (3, 5000, BF, False, True, True), (5, 8192, BF, True, True, True), (2, 16383, F32, False, True, True), (3, 16384, BF, False, True, True),
    (3, 16384, F32, False, True, True), (2, 16383, BF, True, True, True)]


@pytest.mark.parametrize("rows,width,dt,rms,weight,bias", NORM)
def test_norm(rows, width, dt, rms, weight, bias):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    g_ = _gen(rows + width)
    n = lambda *s, std=1.0: torch.randn(*s, device="cuda", generator=g_) * std  # noqa: E731
    x = (n(rows, width) * n(rows, 1, std=0.5).exp() + 0.3).to(dt)
    w, b = (1 + n(width, std=0.2)).to(dt) if weight else None, n(width, std=0.2).to(dt) if bias else None
    dy = n(rows, width).to(dt)
    if rows > 2:
        x[1] = 0                                   # a row without deviation
    eps = 1e-3
    ref = [lf.f64(t) for t in (x, w, b)]
    ry = lf.norm(*ref, eps=eps, rms=rms)
    rg = lf.grads((ry,), (dy.double().cpu(),), ref)
    # A row's sums: 64 terms in a thread at most, then a tree of 10: with the products around them below 200 roundings, of values as
    # large as |x| before the mean is taken off, times r.  (width == 1: y is the bias, x - mean exactly 0.)
    xd = ref[0].detach()
    r = 1 / torch.sqrt((xd if rms else xd - xd.mean(-1, keepdim=True)).square().mean(-1, keepdim=True) + eps)
    size = xd.abs().amax(-1, keepdim=True) * r
    wm = _most(ref[1]) if weight else 1.0
    gm = dy.double().cpu().abs().amax(-1, keepdim=True) * wm
    k = 200 * lf.ULP
    y, stats = qd.norm_fwd(x, w, b, eps, rms=rms)
    lf.close("y", y, ry, k * (size * wm * (1 + size) + (_most(ref[2]) if bias else 0)))
    g = qd.norm_bwd(x, w, dy, stats, rms=rms, want_dbias=bias)
    lf.close("dx", g["dx"], rg[0], k * r * gm * (1 + size) ** 2)
    kw = (200 + rows) * lf.ULP
    for name, ref_, terms in (("dweight", rg[1], (dy.double().cpu().abs() * size * (1 + size)).sum(0)), ("dbias", rg[2], dy.double().cpu().abs().sum(0))):
        assert (g[name] is None) == (ref_ is None)
        if ref_ is not None:
            lf.close(name, g[name], ref_, kw * terms)
    have = [t.requires_grad_() for t in (x, w, b) if t is not None]
    ay = qa.layer_norm(x, w, b, eps, rms=rms)
    assert torch.equal(ay, y)
    names = [m for m, t in zip(("dx", "dweight", "dbias"), (x, w, b)) if t is not None]
    for m, t, got in zip(names, have, torch.autograd.grad(ay, have, dy)):
        assert got.dtype == t.dtype and torch.equal(got, g[m].to(t.dtype)), m
