"""How convolution, scan and norm are used: beside the delta rule in a layer, on streams, in graphs, through autograd, next to other buffers."""
import threading

import pytest
import torch

import gpu_util as gu
import layer_forms as lf

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _n(*s, seed=0, std=1.0, to=BF):
    return (torch.randn(*s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + sum(s))) * std).to(to)


def _scan(B=2, T=70, D=40, N=16, G=1, to=BF, seed=0):
    return dict(u=_n(B, T, D, seed=seed, to=to), dt=_n(B, T, D, seed=seed + 1, to=to) - 3, A=-_n(D, N, seed=seed + 2, to=F32).exp(),
                Bm=_n(B, T, G, N, seed=seed + 3, to=to), Cm=_n(B, T, G, N, seed=seed + 4, to=to), D=_n(D, seed=seed, to=F32),
                z=_n(B, T, D, seed=seed + 5, to=to), dt_bias=_n(D, seed=seed + 6, to=F32))


# ---- a layer: norm -> convolution of q, k, v -> delta rule -> norm of the read-out per head ------------------------------------
def _layer(p, x, states=None):
    """x [B,T,D] -> output, states; one call serves a prompt and what follows it."""
    from paper_2606_08804_b200 import autograd as qa
    B, T, D = x.shape
    H, d = p["H"], 128
    n = qa.layer_norm(x, p["nw"], p["nb"])
    qkv = n @ p["wqkv"]
    c, conv = qa.short_conv(qkv, p["cw"], p["cb"], states[0] if states else None, silu=True)
    q, k, v = (t.reshape(B, T, H, d) for t in c.split(H * d, -1))
    gates = [(n @ p[w]).reshape(B, T, H) for w in ("wb", "wa", "wl")]
    o, hT = qa.qdelta_chunk(q, k, v, *gates, states[1] if states else None, logits=True, norm_qk=True)
    o = qa.layer_norm(o, p["ow"], None, rms=True).reshape(B, T, H * d)
    return o @ p["wo"], (conv, hT)


def _step(p, x, states):
    """One token, states updated in place."""
    from paper_2606_08804_b200 import binding as qd
    B, S, D = x.shape
    H, d = p["H"], 128
    n, _ = qd.norm_fwd(x, p["nw"], p["nb"], want_stats=False)
    c = qd.conv_steps(n @ p["wqkv"], p["cw"], p["cb"], states[0], silu=True)
    q, k, v = (t.reshape(B, S, H, d).contiguous() for t in c.split(H * d, -1))
    gates = [(n @ p[w]).reshape(B, S, H) for w in ("wb", "wa", "wl")]
    o = qd.recurrent_steps(q, k, v, *gates, states[1], logits=True, norm_qk=True)
    o, _ = qd.norm_fwd(o, p["ow"], None, rms=True, want_stats=False)
    return o.reshape(B, S, H * d) @ p["wo"]


def _layer_params(D=64, H=2, to=BF):
    m = lambda *s, seed: _n(*s, seed=seed, std=s[0] ** -0.5, to=to)  # noqa: E731
    return dict(H=H, nw=1 + _n(D, seed=1, std=.1, to=to), nb=_n(D, seed=2, std=.1, to=to), wqkv=m(D, 3 * H * 128, seed=3), cw=_n(3 * H * 128, 4, seed=4, std=.5, to=to),
                cb=_n(3 * H * 128, seed=5, std=.1, to=to), wb=m(D, H, seed=6), wa=m(D, H, seed=7), wl=m(D, H, seed=8), ow=1 + _n(128, seed=9, std=.1, to=to),
                wo=m(H * 128, D, seed=10))


def test_layer_prompt_then_tokens():
    """A prompt and tokens after it against one call over everything: two orders of the same sums, each within the bf16 bar of the delta rule."""
    p, x = _layer_params(), _n(2, 100, 64)
    with torch.no_grad():
        want, (conv, hT) = _layer(p, x)
        y, (c0, h0) = _layer(p, x[:, :90])
        states = (c0.clone(), h0.clone())
        got = torch.cat([y] + [_step(p, x[:, t:t + 1].contiguous(), states) for t in range(90, 100)], 1)
    assert gu.rel_err(got, want.double().cpu().numpy()) < gu.TOL["bf16"]
    assert gu.rel_err(states[1], hT.double().cpu().numpy()) < gu.TOL["bf16"]
    assert torch.equal(states[0], conv)


def test_layer_gradients_reach_every_parameter():
    p, x = _layer_params(to=F32), _n(2, 40, 64, to=F32).requires_grad_()
    leaves = [x] + [t.requires_grad_() for t in p.values() if torch.is_tensor(t)]
    dy = _n(2, 40, 64, seed=9, to=F32)
    y, _ = _layer(p, x)
    g = torch.autograd.grad(y, leaves, dy)
    # along a random direction of all of them: fp32 differences of a sum S of 5120 terms are good to about 2^-24 sqrt(5120) S / step
    way = [_n(*t.shape, seed=77 + i, to=F32) * t.detach().std().clamp(min=0.05) for i, t in enumerate(leaves)]
    h = 3e-3
    def along(e):
        with torch.no_grad():
            q = {n: (t + e * way[1 + [i for i, u in enumerate(v for v in p.values() if torch.is_tensor(v)) if u is t][0]]) if torch.is_tensor(t) else t
                 for n, t in p.items()}
            return float((_layer(q, x + e * way[0])[0].double() * dy.double()).sum())
    want = (along(h) - along(-h)) / (2 * h)
    got = sum(float((a.double() * b.double()).sum()) for a, b in zip(g, way))
    assert abs(got - want) <= 2e-2 * abs(want) + 2.0 ** -24 * 72 * abs(along(0.0)) / h, (got, want)


def test_scan_layer_prompt_then_tokens():
    """norm -> convolution -> scan, as a prompt and then token by token."""
    from paper_2606_08804_b200 import binding as qd
    B, T, D, N = 3, 60, 96, 16
    x, cw, a = _n(B, T, D), _n(D, 4, std=.5), _scan(B, T, D, N)

    def run(lo, hi, conv, h):
        n, _ = qd.norm_fwd(x[:, lo:hi].contiguous(), rms=True)
        part = {m: t[:, lo:hi].contiguous() if m in ("dt", "Bm", "Cm", "z") else t for m, t in a.items() if m != "u"}
        if hi - lo > 4:
            u, conv = qd.conv_fwd(n, cw, None, conv, silu=True)
            y, h, _ = qd.scan_fwd(u, part["dt"], part["A"], part["Bm"], part["Cm"], part["D"], part["z"], part["dt_bias"], h, softplus=True)
        else:
            u = qd.conv_steps(n, cw, None, conv, silu=True)
            y = qd.scan_steps(u, part["dt"], part["A"], part["Bm"], part["Cm"], part["D"], part["z"], part["dt_bias"], h, softplus=True)
        return y, conv, h

    want, c1, h1 = run(0, T, None, None)
    y, c, h = run(0, 50, None, None)
    ys = [y]
    for lo, hi in ((50, 51), (51, 52), (52, 55), (55, 59), (59, 60)):
        y, c, h = run(lo, hi, c, h)
        ys.append(y)
    assert torch.equal(c, c1)
    got = torch.cat(ys, 1)
    # y is rounded to bf16 once on either side; the states are fp32 sums in the same order but for segments
    assert ((got.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 1e-3 * float(want.float().abs().max())).all()
    assert ((h - h1).abs() <= 10 * T * lf.ULP * float(h1.abs().max())).all()


# ---- streams, graphs, threads --------------------------------------------------------------------------------------------------
def _calls():
    """name -> (function of nothing, giving tensors): every entry point on small inputs of its own."""
    from paper_2606_08804_b200 import binding as qd
    x, w, b, s, dy = _n(3, 50, 72), _n(72, 4), _n(72), _n(3, 3, 72), _n(3, 50, 72, seed=1)
    a = _scan()
    g = _n(2, 70, 40, seed=4)
    nx, nw, nb, nd = _n(300, 256), _n(256), _n(256, seed=1), _n(300, 256, seed=2)
    h = _n(2, 40, 16, to=F32)

    def scan():
        y, hT, ws = qd.scan_fwd(**a, h0=h, softplus=True, save_for_bwd=True)
        return [y, hT] + list(qd.scan_bwd(**a, h0=h, dy=g, dhT=h, workspace=ws, reuse_fwd=True, softplus=True).values())

    def scan_long():          # cut into segments
        y, hT, _ = qd.scan_fwd(**long, softplus=True)
        return [y, hT]
    long = _scan(1, 1500, 24)

    def steps():
        s1, h1 = s.clone(), h.clone()
        one = {n: t[:, :2].contiguous() if t.dim() > 2 else t for n, t in a.items()}
        return [qd.conv_steps(x[:, :3].contiguous(), w, b, s1, silu=True), s1, qd.scan_steps(**one, state=h1, softplus=True), h1]

    def norm():
        y, st = qd.norm_fwd(nx, nw, nb)
        return [y, st] + list(qd.norm_bwd(nx, nw, nd, st).values())

    def conv():
        return list(qd.conv_fwd(x, w, b, s, silu=True)) + list(qd.conv_bwd(x, w, b, s, dy, s, silu=True).values())
    return {"conv": conv, "scan": scan, "scan_long": scan_long, "steps": steps, "norm": norm}


@pytest.mark.parametrize("name", ["conv", "scan", "scan_long", "steps", "norm"])
def test_same_bits_again_on_another_stream_in_a_graph_and_between_others(name):
    f = _calls()[name]
    want = [t.clone() for t in f()]
    others = _calls()
    for _ in range(3):
        for o in others.values():
            o()
        assert all(torch.equal(a, b) for a, b in zip(f(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = f()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = f()
    with torch.cuda.graph(second):
        more = f()
    for t in got + more:
        t.zero_()
    for k in range(3):                                    # the two at once, on a stream each
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        second.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(more, want)), k


def test_two_threads_on_two_streams():
    want = {n: [t.clone() for t in f()] for n, f in _calls().items()}
    torch.cuda.synchronize()
    bad = []

    def work():
        calls = _calls()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(5):
                got = {n: f() for n, f in calls.items()}
                s.synchronize()
                bad.extend(n for n in got if not all(torch.equal(a, b) for a, b in zip(got[n], want[n])))
    ts = [threading.Thread(target=work) for _ in range(2)]
    [t.start() for t in ts]
    [t.join() for t in ts]
    assert not bad, bad


def test_training_step_in_a_graph():
    """Captured forward and backward through autograd.  (No eager autograd graph of the same leaves may live meanwhile: torch's engine would
    wait for the stream of its AccumulateGrad nodes, which ends a capture, whatever operators the step is made of.)"""
    from paper_2606_08804_b200 import autograd as qa
    x, w, cw = _n(2, 40, 64).requires_grad_(), (1 + _n(64)).detach().requires_grad_(), _n(64, 4).requires_grad_()
    a = {n: t.detach().requires_grad_() for n, t in _scan(2, 40, 64).items() if n != "u"}
    leaves = [x, w, cw] + list(a.values())
    dy = _n(2, 40, 64, seed=5)

    def step():
        u, _ = qa.short_conv(qa.layer_norm(x, w), cw, silu=True)
        y, _ = qa.selective_scan(u, **a, softplus=True)
        return torch.autograd.grad(y, leaves, dy)
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


# ---- autograd --------------------------------------------------------------------------------------------------------------------
def test_inputs_of_any_stride_and_place():
    """Slices, transposed, expanded and odd-placed inputs and gradients give what their dense copies give."""
    from paper_2606_08804_b200 import autograd as qa
    big, w = _n(2, 30, 3 * 24, to=F32), _n(24, 4, to=F32)
    x = big[:, :, 24:48].detach().requires_grad_()
    dense = x.detach().clone().requires_grad_()
    up = _n(1, 1, 24, to=F32).expand(2, 30, 24)
    y, _ = qa.short_conv(x, w)
    yd, _ = qa.short_conv(dense, w)
    assert torch.equal(y, yd) and torch.equal(torch.autograd.grad(y, x, up)[0], torch.autograd.grad(yd, dense, up.contiguous())[0])
    flat = _n(1 + 64 * 8, to=F32)
    off = flat[1:].view(64, 8).detach().requires_grad_()                # dense, 4 bytes past a boundary
    yo, yc = qa.layer_norm(off), qa.layer_norm(off.detach().clone())
    assert off.data_ptr() % 16 == 4 and torch.equal(yo, yc)
    t = _n(30, 2, 24).transpose(0, 1)
    assert torch.equal(qa.short_conv(t, _n(24, 3))[0], qa.short_conv(t.contiguous(), _n(24, 3))[0])


def test_only_wanted_gradients_and_unused_outputs():
    from paper_2606_08804_b200 import autograd as qa
    x, w, b = _n(20, 64).requires_grad_(), (1 + _n(64)).detach(), _n(64).requires_grad_()
    y = qa.layer_norm(x, w, b)
    dy = _n(20, 64, seed=3)
    gx, gb = torch.autograd.grad(y, (x, b), dy)
    assert torch.equal(gb, dy.float().sum(0).to(BF)) or (gb.float() - dy.float().sum(0)).abs().max() <= 2.0 ** -8 * dy.float().sum(0).abs().max() + 1e-5
    a = {n: t.detach().requires_grad_() for n, t in _scan().items()}
    y, hT = qa.selective_scan(**a, softplus=True)
    # of the state alone: u, dt, B, A have gradients, C, D, z none
    g = torch.autograd.grad(hT, list(a.values()), torch.ones_like(hT))
    zero = {n: float(t.abs().max()) == 0 for n, t in zip(a, g)}
    assert zero == {"u": False, "dt": False, "A": False, "Bm": False, "Cm": True, "D": True, "z": True, "dt_bias": False}
    with torch.no_grad():
        y2, _ = qa.selective_scan(**a, softplus=True)
    assert not y2.requires_grad and gu.rel_err(y2, y.detach().double().cpu().numpy()) < 2e-2


def test_second_derivatives_are_refused_when_asked_for():
    from paper_2606_08804_b200 import autograd as qa
    x = _n(4, 64, to=F32).requires_grad_()
    g, = torch.autograd.grad(qa.layer_norm(x).square().sum(), x, create_graph=True)
    assert g.requires_grad
    with pytest.raises(RuntimeError, match="second derivatives"):
        g.sum().backward()


def test_checkpoint_and_saved_tensors_on_the_host():
    from torch.utils.checkpoint import checkpoint
    from paper_2606_08804_b200 import autograd as qa
    a = {n: t.detach().requires_grad_() for n, t in _scan().items()}
    x, w = _n(2, 70, 40).requires_grad_(), _n(40, 4).requires_grad_()

    def f(*t):
        u, _ = qa.short_conv(t[0], t[1], silu=True)
        return qa.layer_norm(qa.selective_scan(u, *t[2:], softplus=True)[0])
    t = [x, w] + [a[n] for n in a if n != "u"]
    up = _n(2, 70, 40, seed=8)
    want = torch.autograd.grad(f(*t), t, up)
    assert all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(checkpoint(f, *t, use_reentrant=False), t, up), want))
    with torch.autograd.graph.save_on_cpu():
        y = f(*t)
    assert all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(y, t, up), want))


@pytest.mark.parametrize("change,says", [(lambda v: v.cpu(), "contiguous CUDA tensor"), (lambda v: v.double() if v.is_floating_point() else v, "dtype"),
                                         (lambda v: v[:-1].contiguous(), "shape|workspace|WORKSPACE|must be")])
def test_saved_tensors_that_come_back_changed_are_refused(change, says):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    a = {n: t.detach().requires_grad_() for n, t in _scan().items()}
    x, w = _n(2, 70, 40).requires_grad_(), _n(40, 4).requires_grad_()
    for make in (lambda: qa.selective_scan(**a, softplus=True)[0], lambda: qa.short_conv(x, w)[0], lambda: qa.layer_norm(x, w[:, 0].contiguous())):
        with torch.autograd.graph.saved_tensors_hooks(lambda v: v, change):
            y = make()
        with pytest.raises(qd.QdeltaError, match=says):
            y.float().sum().backward()
    torch.cuda.synchronize()


def test_wrong_arguments_are_named():
    from paper_2606_08804_b200 import binding as qd
    x, w = _n(2, 8, 16), _n(16, 4)
    for call, says in ((lambda: qd.conv_fwd(x, w.float()), "w must have dtype"), (lambda: qd.conv_fwd(x[0], w), "x must be"),
                       (lambda: qd.conv_fwd(x, w, None, _n(2, 2, 16)), "state must have shape"), (lambda: qd.conv_fwd(x, _n(16, 5)), "UNSUPPORTED"),
                       (lambda: qd.conv_fwd(x.transpose(0, 1), w), "contiguous"), (lambda: qd.conv_fwd(x.half(), w.half()), "unsupported dtype"),
                       (lambda: qd.conv_fwd(x[:, :0].contiguous(), w), "INVALID_ARG"), (lambda: qd.norm_fwd(_n(4, 8), _n(9)), "weight must have shape"),
                       (lambda: qd.norm_fwd(torch.tensor(1.0, device="cuda")), "last dimension"), (lambda: qd.norm_fwd(_n(4, 16500)), "UNSUPPORTED"),
                       (lambda: qd.norm_bwd(_n(4, 8), None, _n(4, 8), torch.zeros(2, 3, device="cuda")), "stats must have shape"),
                       (lambda: qd.scan_fwd(**dict(_scan(), A=_n(40, 16))), "A must have dtype"), (lambda: qd.scan_fwd(**dict(_scan(), z=_n(2, 70, 39))), "z must have shape"),
                       (lambda: qd.scan_fwd(**_scan(N=65)), "UNSUPPORTED"), (lambda: qd.scan_fwd(**_scan(G=3)), "UNSUPPORTED"),
                       (lambda: qd.scan_fwd(**_scan(), save_for_bwd=True, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), "WORKSPACE"),
                       (lambda: qd.scan_steps(**_scan(), state=_n(2, 40, 16)), "state must have dtype")):
        with pytest.raises(qd.QdeltaError, match=says):
            call()
    torch.cuda.synchronize()


def test_out_of_memory_can_be_caught_as_such():
    from paper_2606_08804_b200 import binding as qd
    torch.cuda.empty_cache()                               # so that x takes a block of its own, with no room beside it
    x, w = torch.zeros(8, 4096, 512, dtype=BF, device="cuda"), torch.zeros(512, 4, dtype=BF, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    limit = torch.cuda.memory_reserved() + (2 << 20)
    torch.cuda.set_per_process_memory_fraction(limit / torch.cuda.get_device_properties(0).total_memory)
    try:
        with pytest.raises(torch.OutOfMemoryError):
            qd.conv_fwd(x, w)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    qd.conv_fwd(x, w)
    torch.cuda.synchronize()


# ---- memory ------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D,T,N,to", [(40, 33, 16, BF), (7, 9, 3, BF), (130, 260, 33, F32), (24, 700, 5, F32)])
def test_nothing_is_written_beside_the_outputs(D, T, N, to):
    """Through the C ABI, every output and workspace between two bands of a fixed pattern."""
    import ctypes

    from paper_2606_08804_b200 import binding as qd
    lib, code, B, W = qd.load(), 1 if to == BF else 0, 2, 4
    G = lambda *s, t=to, fill=None: gu.Guarded(s, t, fill)  # noqa: E731
    x, w, s, dy = _n(B, T, D, to=to), _n(D, W, to=to), _n(B, W - 1, D, to=to), _n(B, T, D, seed=1, to=to)
    a = _scan(B, T, D, N, to=to)
    nx = _n(T, D, to=to)
    p = lambda t: None if t is None else (t.t if isinstance(t, gu.Guarded) else t).data_ptr()  # noqa: E731
    stream = torch.cuda.current_stream().cuda_stream
    u8 = torch.uint8
    n = lib.qdelta_conv_workspace_bytes(B, T, D, W, code)
    cy, cl, cdx, cdw, cdb, cds, cws = G(B, T, D), G(B, W - 1, D), G(B, T, D), G(D, W, t=F32), G(D, t=F32), G(B, W - 1, D), G(n, t=u8)
    bias = _n(D, to=to)
    cst = G(B, W - 1, D, fill=s)
    assert lib.qdelta_conv_fwd(B, T, D, W, code, p(x), p(w), p(bias), p(s), p(cy), p(cl), 32, stream) == 0
    assert lib.qdelta_conv_bwd(B, T, D, W, code, p(x), p(w), p(bias), p(s), p(dy), p(s), p(cdx), p(cdw), p(cdb), p(cds), p(cws), n, 32, stream) == 0
    cy2 = G(B, T, D)
    assert lib.qdelta_conv_steps(B, T, D, W, code, p(x), p(w), p(bias), p(cst), p(cy2), 32, stream) == 0
    sh = qd.QdScanShape(B, T, D, N, 1, code)
    r = ctypes.byref(sh)
    m = lib.qdelta_scan_workspace_bytes(r, 1)
    f = lib.qdelta_scan_workspace_bytes(r, 0)
    ws, wf = G(m, t=u8), G(max(f, 16), t=u8)
    h0 = _n(B, D, N, to=F32)
    ins = [p(a[k]) for k in ("u", "dt", "A", "Bm", "Cm", "D", "z", "dt_bias")]
    y, hT = G(B, T, D), G(B, D, N, t=F32)
    assert lib.qdelta_scan_fwd(r, *ins, p(h0), p(y), p(hT), p(wf), f, 64, stream) == 0
    assert lib.qdelta_scan_fwd(r, *ins, p(h0), p(y), p(hT), p(ws), m, 64 | 1, stream) == 0
    g = [G(B, T, D), G(B, T, D), G(D, N, t=F32), G(B, T, 1, N), G(B, T, 1, N), G(D, t=F32), G(B, T, D), G(D, t=F32), G(B, D, N, t=F32)]
    assert lib.qdelta_scan_bwd(r, *ins, p(h0), p(dy), p(h0), *[p(t) for t in g], p(ws), m, 64 | 2, stream) == 0
    assert lib.qdelta_scan_bwd(r, *ins, p(h0), p(dy), p(h0), *[p(t) for t in g], p(ws), m, 64, stream) == 0
    st, sy = G(B, D, N, t=F32, fill=h0), G(B, T, D)
    assert lib.qdelta_scan_steps(r, *ins, p(st), p(sy), 64, stream) == 0
    k = lib.qdelta_norm_workspace_bytes(T, D, code)
    ny, nst, ndx, ndw, ndb, nws = G(T, D), G(2, T, t=F32), G(T, D), G(D, t=F32), G(D, t=F32), G(k, t=u8)
    assert lib.qdelta_norm_fwd(T, D, code, p(nx), p(bias), p(bias), p(ny), p(nst), 1e-5, 0, stream) == 0
    assert lib.qdelta_norm_bwd(T, D, code, p(nx), p(bias), p(nx), p(nst), p(ndx), p(ndw), p(ndb), p(nws), k, 0, stream) == 0
    torch.cuda.synchronize()
    for i, t in enumerate([cy, cl, cdx, cdw, cdb, cds, cws, cst, cy2, ws, wf, y, hT, *g, st, sy, ny, nst, ndx, ndw, ndb, nws]):
        assert t.intact(), i
    assert torch.equal(cy.t, cy2.t) and torch.equal(cl.t, cst.t)
    for i, t in enumerate([cy, cdx, y, hT, *g, st, sy, ny, ndx, ndw]):
        assert gu.all_finite(t.t), i


def test_sequences_and_rows_do_not_see_each_other():
    """NaN and infinities in one sequence, row or group leave the others' bits alone."""
    from paper_2606_08804_b200 import binding as qd
    x, w = _n(3, 40, 72), _n(72, 4)
    y, last = qd.conv_fwd(x, w, silu=True)
    g = qd.conv_bwd(x, w, None, None, x, silu=True)
    x2 = x.clone()
    x2[1] = float("nan")
    x2[1, 5] = float("inf")
    y2, last2 = qd.conv_fwd(x2, w, silu=True)
    g2 = qd.conv_bwd(x2, w, None, None, x, silu=True)
    for a, b in ((y, y2), (last, last2), (g["dx"], g2["dx"])):
        assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])
    a = _scan(3, 70, 40, 16, 2)
    b = {n: t.clone() for n, t in a.items()}
    b["u"][1, 3] = float("nan")
    b["Bm"][2, :, 1] = float("inf")                       # the second group's channels of the last sequence
    up = _n(3, 70, 40, seed=3)
    r = [qd.scan_fwd(**t, softplus=True, save_for_bwd=True) for t in (a, b)]
    gs = [qd.scan_bwd(**t, h0=None, dy=up, workspace=q[2], reuse_fwd=True, softplus=True) for t, q in zip((a, b), r)]
    for p, q in ((r[0][0], r[1][0]), (gs[0]["du"], gs[1]["du"]), (gs[0]["ddt"], gs[1]["ddt"])):
        assert torch.equal(p[0], q[0]) and torch.equal(p[2, :, :20], q[2, :, :20])
    n, m = _n(9, 300), _n(9, 300)
    m = n.clone()
    m[4] = float("nan")
    p, q = qd.norm_fwd(n)[0], qd.norm_fwd(m)[0]
    keep = [i for i in range(9) if i != 4]
    assert torch.equal(p[keep], q[keep]) and q[4].isnan().all()


def test_offsets_past_32_bits():
    """Tensors of more than 2^32 elements: the last rows are what a call on them alone gives."""
    from paper_2606_08804_b200 import binding as qd
    D = 4096
    T = (1 << 20) + 40
    x = torch.empty(1, T, D, dtype=BF, device="cuda")
    x[:, -200:] = _n(1, 200, D)
    x[:, :-200].zero_()
    w = _n(D, 4)
    y, last = qd.conv_fwd(x, w, silu=True)
    tail = x[:, -100:].contiguous()
    want, _ = qd.conv_fwd(tail, w, None, x[:, -103:-100].contiguous(), silu=True)
    assert torch.equal(y[:, -100:], want) and torch.equal(last, x[:, -3:])
    del y
    ny, st = qd.norm_fwd(x[0])
    ty, _ = qd.norm_fwd(tail[0])
    assert torch.equal(ny[-100:], ty)
    g = qd.norm_bwd(x[0], None, x[0], st)
    tg = qd.norm_bwd(tail[0], None, tail[0], qd.norm_fwd(tail[0])[1])
    assert torch.equal(g["dx"][-100:], tg["dx"])
    del ny, g, tg
    torch.cuda.empty_cache()
    # steps of 0 keep the state: the scan's last tokens from a zero state
    a = _scan(1, 100, D, 4)
    Bm, Cm = torch.zeros(1, T, 1, 4, dtype=BF, device="cuda"), torch.zeros(1, T, 1, 4, dtype=BF, device="cuda")
    Bm[:, -100:], Cm[:, -100:] = a["Bm"], a["Cm"]
    dt = torch.zeros(1, T, D, dtype=BF, device="cuda")
    dt[:, -100:] = (a["dt"].float().exp()).to(BF)
    y, hT, _ = qd.scan_fwd(x, dt, a["A"], Bm, Cm)
    ty, th, _ = qd.scan_fwd(tail, dt[:, -100:].contiguous(), a["A"], a["Bm"], a["Cm"])
    lf.close("y", y[:, -100:], ty.double().cpu(), 2.0 ** -8 * ty.double().cpu().abs() + 1e-4 * float(ty.float().abs().max()))
    lf.close("hT", hT, th.double().cpu(), 1e-4 * float(th.abs().max()))
