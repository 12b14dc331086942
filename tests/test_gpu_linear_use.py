"""How linear attention, the norms with a gate and behind a residual sum, and rotary positions are used: in a layer, on streams, in graphs,
through autograd, next to other buffers, in tensors past 2^32 elements."""
import ctypes
import math
import threading

import pytest
import torch

import gpu_util as gu
import layer_forms as lf
import linear_forms as f

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _n(*s, seed=0, std=1.0, to=BF):
    return (torch.randn(*s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + sum(s))) * std).to(to)


def _decay(H, slow=0.003):
    return -torch.linspace(slow, 0.9, H, device="cuda")


# ---- a layer: norm -> q, k, v, gate -> rotary -> linear attention -> gated norm -> product -> residual sum and norm ------------------
def _params(D=64, H=2, to=BF):
    m = lambda *s, seed: _n(*s, seed=seed, std=s[0] ** -0.5, to=to)  # noqa: E731
    return dict(H=H, nw=1 + _n(D, seed=1, std=.1, to=to), wqkv=m(D, 3 * H * 64, seed=3), wg=m(D, H * 64, seed=4), ow=1 + _n(64, seed=9, std=.1, to=to),
                wo=m(H * 64, D, seed=10), rs=_n(D, seed=11, std=.2, to=to) + 0.5, fw=1 + _n(D, seed=12, std=.1, to=to), fb=_n(D, seed=13, std=.1, to=to))


def _split(p, n):
    B, T, _ = n.shape
    q, k, v = ((n @ p["wqkv"]).reshape(B, T, 3, p["H"], 64).unbind(2))
    return q, k, v, (n @ p["wg"]).reshape(B, T, p["H"], 64)


def _layer(p, x, turns, decay, h=None, start=0):
    from paper_2606_08804_b200 import autograd as qa
    B, T, D = x.shape
    q, k, v, z = _split(p, qa.layer_norm(x, p["nw"], rms=True))
    q, k = qa.rotary(q, k, turns, start=start)
    o, h = qa.linear_attention(q, k, v, decay, h, scale=0.125)
    o = qa.gated_norm(o, z, p["ow"], rms=True).reshape(B, T, -1)
    y, total = qa.add_norm(o @ p["wo"], x, p["rs"], p["fw"], p["fb"])
    return y, total, h


def _step(p, x, turns, decay, h, at):
    """One token of every sequence, at positions of its own; the state in place."""
    from paper_2606_08804_b200 import binding as qd
    B, S, D = x.shape
    n, _ = qd.norm_fwd(x, p["nw"], rms=True, want_stats=False)
    q, k, v, z = (t.contiguous() for t in _split(p, n))
    q, k = qd.rotary(q, k, turns, positions=at, out=(q, k))
    o = qd.linear_steps(q, k, v, decay, h, scale=0.125)
    o, _ = qd.gated_norm_fwd(o, z, p["ow"], rms=True, want_stats=False)
    y, total, _ = qd.add_norm_fwd(o.reshape(B, S, -1) @ p["wo"], x, p["rs"], p["fw"], p["fb"], want_stats=False)
    return y, total


def test_layer_prompt_then_tokens():
    from paper_2606_08804_b200 import binding as qd
    p, x, turns, decay = _params(), _n(3, 200, 64), qd.rotary_turns(24), _decay(2)
    with torch.no_grad():
        want, wt, wh = _layer(p, x, turns, decay)
        y, t, h = _layer(p, x[:, :190], turns, decay)
        ys, ts, h = [y], [t], h.clone()
        for i in range(190, 200):
            y, t = _step(p, x[:, i:i + 1].contiguous(), turns, decay, h, torch.full((3, 1), i, device="cuda"))
            ys.append(y)
            ts.append(t)
        # the prompt in two pieces
        y0, _, h0 = _layer(p, x[:, :130], turns, decay)
        y1, _, h1 = _layer(p, x[:, 130:], turns, decay, h0, start=130)
    for got, ref in ((torch.cat(ys, 1), want), (torch.cat(ts, 1), wt), (h, wh), (torch.cat((y0, y1), 1), want), (h1, wh)):
        assert gu.rel_err(got, ref.double().cpu().numpy()) < gu.TOL["bf16"]


def test_layer_gradients_reach_every_parameter():
    from paper_2606_08804_b200 import binding as qd
    p, x, turns, decay = _params(to=F32), _n(2, 70, 64, to=F32).requires_grad_(), qd.rotary_turns(24), _decay(2)
    names = [n for n in p if torch.is_tensor(p[n])]
    leaves = [x] + [p[n].requires_grad_() for n in names]
    ups = [_n(2, 70, 64, seed=s, to=F32) for s in (9, 10)]
    y, total, _ = _layer(p, x, turns, decay)
    g = torch.autograd.grad((y, total), leaves, ups)
    # along a random direction of all of them: fp32 differences of a sum S of 17920 terms are good to about 2^-24 sqrt(17920) S / step
    way = [_n(*t.shape, seed=77 + i, to=F32) * t.detach().std().clamp(min=0.05) for i, t in enumerate(leaves)]
    h = 3e-3

    def along(e):
        with torch.no_grad():
            q = dict(p, **{n: p[n] + e * w for n, w in zip(names, way[1:])})
            a = _layer(q, x + e * way[0], turns, decay)
            return sum(float((o.double() * u.double()).sum()) for o, u in zip(a, ups))
    want = (along(h) - along(-h)) / (2 * h)
    got = sum(float((a.double() * b.double()).sum()) for a, b in zip(g, way))
    assert abs(got - want) <= 2e-2 * abs(want) + 2.0 ** -24 * 134 * abs(along(0.0)) / h, (got, want)
    assert all(float(t.abs().max()) > 0 for t in g)


# ---- streams, graphs, threads --------------------------------------------------------------------------------------------------
def _calls():
    """name -> function of nothing, giving tensors: every entry point on small inputs of its own."""
    from paper_2606_08804_b200 import binding as qd

    def attention(B, T, H, dk, dv, to):
        q, k, v, dO = _n(B, T, H, dk, std=.1, to=to), _n(B, T, H, dk, std=.1, seed=1, to=to), _n(B, T, H, dv, seed=2, to=to), _n(B, T, H, dv, seed=3, to=to)
        g, h, dh = _decay(H), _n(B, H, dk, dv, to=F32), _n(B, H, dk, dv, seed=1, to=F32)

        def f():
            o, hT, _ = qd.linear_fwd(q, k, v, g, h, 0.5)
            return [o, hT] + list(qd.linear_bwd(q, k, v, g, h, dO, dh, 0.5).values())
        return f
    q, k, v, g, h = _n(3, 4, 5, 64), _n(3, 4, 5, 64, seed=1), _n(3, 4, 5, 128), _decay(5), _n(3, 5, 64, 128, to=F32)

    def steps():
        s = h.clone()
        return [qd.linear_steps(q, k, v, g, s), s]

    def norms(rows, width, to=BF):
        x, z, e, dy, dt = (_n(rows, width, seed=i, to=to) for i in range(5))
        w, b, c = _n(width, to=to), _n(width, seed=1, to=to), _n(width, seed=2, to=to)

        def f():
            y, s = qd.gated_norm_fwd(x, z, w, b)
            y2, t, s2 = qd.add_norm_fwd(x, e, c, w, b)
            return [y, s, y2, t, s2] + list(qd.gated_norm_bwd(x, z, w, b, dy, s).values()) + \
                list(qd.add_norm_bwd(x, e, c, w, dy, dt, s2, want_dbias=True).values())
        return f
    turns = qd.rotary_turns(20)
    return {"attention": attention(2, 150, 3, 64, 64, BF), "segments": attention(1, 1500, 2, 128, 128, BF), "unequal": attention(1, 300, 2, 64, 128, BF),
            "fp32": attention(1, 500, 2, 64, 64, F32), "steps": steps, "norms": norms(300, 256), "odd": norms(70, 301), "wide": norms(9, 9000),
            "rotary": lambda: list(qd.rotary(q, k, turns, start=7)) + list(qd.rotary(q, k, turns, interleaved=True, inverse=True))}


NAMES = ["attention", "segments", "unequal", "fp32", "steps", "norms", "odd", "wide", "rotary"]


@pytest.mark.parametrize("name", NAMES)
def test_same_bits_again_on_another_stream_in_a_graph_and_between_others(name):
    others = _calls()
    f = others[name]
    want = [t.clone() for t in f()]
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
    """Captured forward and backward through autograd, with no eager graph of the same leaves alive (see test_gpu_layer_use.py)."""
    from paper_2606_08804_b200 import binding as qd
    p, x, turns, decay = _params(), _n(2, 140, 64).requires_grad_(), qd.rotary_turns(24), _decay(2)
    leaves = [x] + [t.requires_grad_() for t in p.values() if torch.is_tensor(t)]
    dy = _n(2, 140, 64, seed=5)

    def step():
        return torch.autograd.grad(_layer(p, x, turns, decay)[0], leaves, dy)
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
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- autograd --------------------------------------------------------------------------------------------------------------------
def test_inputs_of_any_stride_and_place():
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    qkv = _n(2, 70, 3, 2, 64, to=F32)
    q, k, v = (t.detach().requires_grad_() for t in qkv.unbind(2))
    dense = [t.detach().contiguous().requires_grad_() for t in (q, k, v)]
    g, up = _decay(2), _n(1, 1, 1, 64, to=F32).expand(2, 70, 2, 64)
    turns = qd.rotary_turns(32)
    for a, b in zip(qa.rotary(q, k, turns), qa.rotary(dense[0], dense[1], turns)):
        assert torch.equal(a, b)
    o, od = qa.linear_attention(q, k, v, g)[0], qa.linear_attention(*dense, g)[0]
    assert torch.equal(o, od)
    for a, b in zip(torch.autograd.grad(o, (q, k, v), up), torch.autograd.grad(od, dense, up.contiguous())):
        assert torch.equal(a, b)
    flat = _n(1 + 64 * 8, to=F32)
    off = flat[1:].view(64, 8)                                          # dense, 4 bytes past a boundary
    assert off.data_ptr() % 16 == 4
    assert torch.equal(qa.gated_norm(off, off), qa.gated_norm(off.clone(), off.clone()))
    assert torch.equal(qa.add_norm(off, off)[0], qa.add_norm(off.clone(), off.clone())[0])


def test_unused_outputs_and_one_tensor_twice():
    from paper_2606_08804_b200 import autograd as qa
    x, z = _n(20, 64, to=F32).requires_grad_(), _n(20, 64, seed=1, to=F32).requires_grad_()
    dy = _n(20, 64, seed=3, to=F32)
    y, total = qa.add_norm(x, z)
    gx, gz = torch.autograd.grad(total, (x, z), dy)
    assert torch.equal(gx, dy) and torch.equal(gz, dy)
    # a residual that is the block's own input, and a gate that is its own norm's
    y, _ = qa.add_norm(x, x)
    a, = torch.autograd.grad(y, x, dy)
    y, _ = qa.add_norm(x, x.detach())
    b, = torch.autograd.grad(y, x, dy)
    assert torch.equal(a, 2 * b)
    both, = torch.autograd.grad(qa.gated_norm(x, x), x, dy)
    one, = torch.autograd.grad(qa.gated_norm(x, x.detach()), x, dy)
    two, = torch.autograd.grad(qa.gated_norm(x.detach(), x), x, dy)
    assert torch.equal(both, one + two)
    q, g = _n(1, 40, 2, 64, to=F32).requires_grad_(), _decay(2)
    o, hT = qa.linear_attention(q, q, q, g)
    u = _n(*o.shape, seed=4, to=F32)
    whole = torch.autograd.grad(o, q, u, retain_graph=True)[0]
    each = [torch.autograd.grad(qa.linear_attention(*[t if i == j else t.detach() for j, t in enumerate((q, q, q))], g)[0], q, u)[0] for i in range(3)]
    # three summands in any order: two roundings of at most their sizes' sum
    assert ((whole - sum(each)).abs() <= 4 * lf.ULP * sum(t.abs() for t in each)).all()
    gq = torch.autograd.grad(hT, q, torch.ones_like(hT))[0]             # of the state alone
    assert float(gq.abs().max()) > 0


def test_what_is_refused():
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    q, k, v, g, h = _n(2, 8, 2, 64), _n(2, 8, 2, 64), _n(2, 8, 2, 64), _decay(2), _n(2, 2, 64, 64, to=F32)
    x, turns = _n(4, 8), qd.rotary_turns(16)
    for call, says in ((lambda: qd.linear_fwd(q, k, v.float(), g), "v must have dtype"), (lambda: qd.linear_fwd(q[0], k, v, g), "q must be"),
                       (lambda: qd.linear_fwd(q, k[:, :4].contiguous(), v, g), "k must have shape"), (lambda: qd.linear_fwd(q, k, v, g.double()), "log_decay must have dtype"),
                       (lambda: qd.linear_fwd(q, k, v, g[:1].contiguous()), "log_decay must have shape"), (lambda: qd.linear_fwd(q, k, v, g.cpu()), "log_decay must be"),
                       (lambda: qd.linear_fwd(q, k, v, g, h.bfloat16()), "h0 must have dtype"), (lambda: qd.linear_fwd(q.transpose(0, 1), k, v, g), "contiguous"),
                       (lambda: qd.linear_fwd(q.half(), k.half(), v.half(), g), "unsupported dtype"), (lambda: qd.linear_fwd(_n(1, 2, 1, 32), _n(1, 2, 1, 32), _n(1, 2, 1, 32), g[:1]), "unsupported"),
                       (lambda: qd.linear_fwd(q, k, v, g, scale=float("inf")), "INVALID_ARG"), (lambda: qd.linear_fwd(q[:, :0], k[:, :0], v[:, :0], g), "unsupported or invalid|contiguous"),
                       (lambda: qd.linear_fwd(q, k, v, g, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), "WORKSPACE"),
                       (lambda: qd.linear_bwd(q, k, v, g, None, v[:1].contiguous()), "dO must have shape"), (lambda: qd.linear_steps(q, k, v, g, h.bfloat16()), "state must have dtype"),
                       (lambda: qd.linear_steps(q, k, v, g, h, o=q), "INVALID_ARG"),
                       (lambda: qd.gated_norm_fwd(x, _n(4, 9)), "gate must have shape"), (lambda: qd.gated_norm_fwd(x, x, _n(9)), "weight must have shape"),
                       (lambda: qd.gated_norm_fwd(_n(2, 16500), _n(2, 16500)), "UNSUPPORTED"), (lambda: qd.gated_norm_bwd(x, x, None, None, x, torch.zeros(2, 3, device="cuda")), "stats must have shape"),
                       (lambda: qd.add_norm_fwd(x, x.float()), "residual must have dtype"), (lambda: qd.add_norm_fwd(x, x, _n(7)), "scale must have shape"),
                       (lambda: qd.add_norm_fwd(torch.tensor(1.0, device="cuda"), x), "last dimension"),
                       (lambda: qd.rotary(q, k, turns.int()), "turns must have dtype"), (lambda: qd.rotary(q, k, turns, torch.zeros(2, 7, dtype=torch.int64, device="cuda")), "positions must have shape"),
                       (lambda: qd.rotary(q, k, turns, torch.zeros(2, 8, dtype=torch.int32, device="cuda")), "positions must have dtype"), (lambda: qd.rotary(q, _n(2, 8, 2, 32), turns), "k must have shape"),
                       (lambda: qd.rotary(q, k, qd.rotary_turns(33)), "UNSUPPORTED"), (lambda: qd.rotary(q, k, turns, out=(q, q)), "INVALID_ARG"),
                       (lambda: qd.rotary(q, None, turns, out=(q, k)), "needs k"),
                       (lambda: qa.linear_attention(q, k, v, g.clone().requires_grad_()), "log_decay is a constant")):
        with pytest.raises(qd.QdeltaError, match=says):
            call()
    torch.cuda.synchronize()
    for f in (lambda t: qa.linear_attention(t, k.float(), v.float(), g)[0], lambda t: qa.gated_norm(t, t), lambda t: qa.add_norm(t, t)[0], lambda t: qa.rotary(t, None, turns)[0]):
        t = q.float().requires_grad_()
        d, = torch.autograd.grad(f(t).square().sum(), t, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            d.sum().backward()


def test_what_was_saved_may_not_be_written():
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    q, k, v, g, h = _n(2, 8, 2, 64), _n(2, 8, 2, 64, seed=1), _n(2, 8, 2, 64, seed=2), _decay(2), _n(2, 2, 64, 64, to=F32)
    q.requires_grad_()
    o, _ = qa.linear_attention(q, k, v, g, h)
    qd.linear_steps(q.detach(), k, v, g, h)                              # the initial state, in place
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.float().sum().backward()
    turns = qd.rotary_turns(32)
    x, w = _n(2, 8, 2, 64, seed=3), _n(64).requires_grad_()
    y = qa.gated_norm(x, x, w)
    qd.rotary(x, None, turns, out=(x, None))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()


def test_checkpoint_and_saved_tensors_that_come_back():
    from torch.utils.checkpoint import checkpoint
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    p, x, turns, decay = _params(), _n(2, 70, 64).requires_grad_(), qd.rotary_turns(24), _decay(2)
    f = lambda t: _layer(p, t, turns, decay)[0]  # noqa: E731
    up = _n(2, 70, 64, seed=8)
    want = torch.autograd.grad(f(x), x, up)[0]
    assert torch.equal(torch.autograd.grad(checkpoint(f, x, use_reentrant=False), x, up)[0], want)
    with torch.autograd.graph.save_on_cpu():
        y = f(x)
    assert torch.equal(torch.autograd.grad(y, x, up)[0], want)
    q = _n(2, 70, 2, 64).requires_grad_()
    for change, says in ((lambda t: t.cpu(), "contiguous CUDA tensor"), (lambda t: t.double() if t.is_floating_point() else t, "dtype")):
        for make in (lambda: qa.linear_attention(q, q, q, decay)[0], lambda: qa.gated_norm(q, q), lambda: qa.add_norm(q, q)[0]):
            with torch.autograd.graph.saved_tensors_hooks(lambda t: t, change):
                y = make()
            with pytest.raises(qd.QdeltaError, match=says):
                y.float().sum().backward()
    torch.cuda.synchronize()


# ---- memory ------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,H,dk,dv,to", [(1, 1, 64, 64, F32), (130, 2, 128, 64, BF), (700, 1, 64, 128, BF), (333, 2, 64, 64, F32), (1400, 2, 128, 128, BF)])
def test_attention_writes_nothing_beside_its_outputs(T, H, dk, dv, to):
    from paper_2606_08804_b200 import binding as qd
    lib, B = qd.load(), 2
    G = lambda *s, t=to, fill=None: gu.Guarded(s, t, fill)  # noqa: E731
    p = lambda t: None if t is None else (t.t if isinstance(t, gu.Guarded) else t).data_ptr()  # noqa: E731
    q, k, v, dO, g, h = _n(B, T, H, dk, to=to), _n(B, T, H, dk, to=to), _n(B, T, H, dv, to=to), _n(B, T, H, dv, to=to), _decay(H), _n(B, H, dk, dv, to=F32)
    s = qd.QdLinearShape(B, T, H, dk, dv, 1 if to == BF else 0)
    r, stream = ctypes.byref(s), torch.cuda.current_stream().cuda_stream
    nf, nb = lib.qdelta_linear_workspace_bytes(r, 0), lib.qdelta_linear_workspace_bytes(r, 1)
    wf, wb, o, hT, st, so = G(nf, t=torch.uint8), G(nb, t=torch.uint8), G(B, T, H, dv), G(B, H, dk, dv, t=F32), G(B, H, dk, dv, t=F32, fill=h), G(B, T, H, dv)
    dq, dk_, dv_, dh = G(B, T, H, dk), G(B, T, H, dk), G(B, T, H, dv), G(B, H, dk, dv, t=F32)
    assert lib.qdelta_linear_fwd(r, p(q), p(k), p(v), p(g), p(h), p(o), p(hT), 1.0, p(wf), nf, 0, stream) == 0
    assert lib.qdelta_linear_bwd(r, p(q), p(k), p(v), p(g), p(h), p(dO), p(h), p(dq), p(dk_), p(dv_), p(dh), 1.0, p(wb), nb, 0, stream) == 0
    assert lib.qdelta_linear_steps(r, p(q), p(k), p(v), p(g), p(st), p(so), 1.0, 0, stream) == 0
    torch.cuda.synchronize()
    for i, t in enumerate([wf, wb, o, hT, st, so, dq, dk_, dv_, dh]):
        assert t.intact(), i
    for i, t in enumerate([o, hT, st, so, dq, dk_, dv_, dh]):
        assert gu.all_finite(t.t), i


@pytest.mark.parametrize("rows,width,to", [(1, 1, BF), (5, 7, BF), (300, 129, BF), (40, 1001, BF), (40, 1002, BF), (7, 5001, BF), (3, 16383, BF), (3, 16384, BF),
                                           (33, 9, F32), (9, 1023, F32), (5, 4097, F32), (3, 16384, F32), (1000, 128, BF), (70, 4096, F32)])
def test_norms_and_rotary_write_nothing_beside_their_outputs(rows, width, to):
    from paper_2606_08804_b200 import binding as qd
    lib, code, stream = qd.load(), 1 if to == BF else 0, torch.cuda.current_stream().cuda_stream
    G = lambda *s, t=to, fill=None: gu.Guarded(s, t, fill)  # noqa: E731
    p = lambda t: (t.t if isinstance(t, gu.Guarded) else t).data_ptr()  # noqa: E731
    x, z, dy, w = _n(rows, width, to=to), _n(rows, width, seed=1, to=to), _n(rows, width, seed=2, to=to), _n(width, to=to)
    n = lib.qdelta_fused_norm_workspace_bytes(rows, width, code)
    y, st, dx, dz, dw, db, ws = G(rows, width), G(2, rows, t=F32), G(rows, width), G(rows, width), G(width, t=F32), G(width, t=F32), G(n, t=torch.uint8)
    assert lib.qdelta_gated_norm_fwd(rows, width, code, p(x), p(z), p(w), p(w), p(y), p(st), 1e-5, 32, stream) == 0
    assert lib.qdelta_gated_norm_bwd(rows, width, code, p(x), p(z), p(w), p(w), p(dy), p(st), p(dx), p(dz), p(dw), p(db), p(ws), n, 32, stream) == 0
    y2, t2, st2, dx2, dr, ds, dw2, db2 = G(rows, width), G(rows, width), G(2, rows, t=F32), G(rows, width), G(rows, width), G(width, t=F32), G(width, t=F32), G(width, t=F32)
    assert lib.qdelta_add_norm_fwd(rows, width, code, p(x), p(z), p(w), p(w), p(w), p(t2), p(y2), p(st2), 1e-5, 0, stream) == 0
    assert lib.qdelta_add_norm_bwd(rows, width, code, p(x), p(z), p(w), p(w), p(dy), p(dy), p(st2), p(dx2), p(dr), p(ds), p(dw2), p(db2), p(ws), n, 0, stream) == 0
    outs = [y, st, dx, dz, dw, db, ws, y2, t2, st2, dx2, dr, ds, dw2, db2]
    if 2 <= width <= 1024:
        turns, q = qd.rotary_turns(max(1, width // 3)), G(1, rows, 1, width)
        assert lib.qdelta_rotary(1, rows, 1, 0, width, len(turns), code, p(x), None, p(turns), None, 5, p(q), None, 1.0, 0, stream) == 0
        outs.append(q)
    torch.cuda.synchronize()
    for i, t in enumerate(outs):
        assert t.intact(), i
        assert t is ws or gu.all_finite(t.t), i
    # in place: the stream's buffer becomes the sum
    e = z.clone()
    assert lib.qdelta_add_norm_fwd(rows, width, code, p(x), p(e), p(w), p(w), p(w), p(e), p(y), None, 1e-5, 0, stream) == 0
    assert torch.equal(e, t2.t) and torch.equal(y.t, y2.t)


def test_every_width_has_a_kernel():
    """Around every power of two, where plans change, and between: all calls run and agree with torch's formulas in fp32 within bf16 steps."""
    from paper_2606_08804_b200 import binding as qd
    widths = sorted({w for k in range(15) for w in (2 ** k - 1, 2 ** k, 2 ** k + 1, 2 ** k + 2, 3 * 2 ** k + 16, 5 * 2 ** k + 4, 7 * 2 ** k + 3) if 1 <= w <= 16384})
    for to in (BF, F32):
        for width in widths:
            x, z, dy = _n(3, width, to=to), _n(3, width, seed=1, to=to), _n(3, width, seed=2, to=to)
            y, s = qd.gated_norm_fwd(x, z, rms=True)
            g = qd.gated_norm_bwd(x, z, None, None, dy, s, rms=True, want_dweight=True)
            y2, t, s2 = qd.add_norm_fwd(x, z, rms=True)
            g2 = qd.add_norm_bwd(x, z, None, None, dy, dy, s2, rms=True, want_dweight=True)
            xf, zf, df = x.float(), z.float(), dy.float()
            f = torch.nn.functional.silu(zf)
            xh, th = (v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-5) for v in (xf, xf + zf))
            for name, got, ref in (("y", y, xh * f), ("y2", y2, th), ("total", t, xf + zf), ("dweight", g["dweight"], (df * f * xh).sum(0)), ("dweight2", g2["dweight"], (df * th).sum(0))):
                assert gu.rel_err(got, ref.double().cpu().numpy()) < 1e-2, (width, to, name)
            assert gu.all_finite(g["dx"], g["dgate"], g2["dresidual"]), (width, to)


def test_sequences_heads_and_rows_do_not_see_each_other():
    """NaN and infinities in one sequence, head or row leave the others' bits alone, and in the attention the chunks before them."""
    from paper_2606_08804_b200 import binding as qd
    for to, chunk in ((BF, 128), (F32, 64)):
        a = [_n(3, 300, 2, 64, seed=i, to=to) for i in range(4)]
        b = [t.clone() for t in a]
        b[1][1, 200, 1] = float("nan")
        b[2][1, 210, 1, 3] = float("inf")
        g = _decay(2)
        r = [qd.linear_fwd(t[0], t[1], t[2], g) for t in (a, b)]
        d = [qd.linear_bwd(t[0], t[1], t[2], g, None, t[3]) for t in (a, b)]
        for p, q in [(r[0][0], r[1][0])] + [(d[0][n], d[1][n]) for n in ("dq", "dk", "dv")]:
            assert torch.equal(p[0], q[0]) and torch.equal(p[2], q[2]) and torch.equal(p[1, :, 0], q[1, :, 0])
        first = 200 // chunk * chunk
        assert torch.equal(r[0][0][1, :first], r[1][0][1, :first]) and torch.equal(d[0]["dq"][1, :first], d[1]["dq"][1, :first])
        assert torch.equal(r[0][1][[0, 2]], r[1][1][[0, 2]]) and torch.equal(r[0][1][1, 0], r[1][1][1, 0])
    for width in (300, 301, 9001):
        x, z = _n(9, width), _n(9, width, seed=1)
        m = x.clone()
        m[4] = float("nan")
        keep = [i for i in range(9) if i != 4]
        for f in (lambda t: qd.gated_norm_fwd(t, z), lambda t: qd.add_norm_fwd(t, z)):
            p, q = f(x)[0], f(m)[0]
            assert torch.equal(p[keep], q[keep]) and q[4].isnan().all()
        s = qd.gated_norm_fwd(x, z)[1]
        assert torch.equal(qd.gated_norm_bwd(x, z, None, None, x, s)["dx"][keep], qd.gated_norm_bwd(m, z, None, None, x, s)["dx"][keep])


def test_offsets_past_32_bits():
    """Tensors of more than 2^32 elements: the last rows are what a call on them alone gives."""
    from paper_2606_08804_b200 import binding as qd
    T, H, d = (1 << 18) + 300, 128, 128
    g = torch.full((H,), -1.0, device="cuda")                            # what is 512 tokens away has become 0
    a = [torch.zeros(1, T, H, d, dtype=BF, device="cuda") for _ in range(4)]
    for i, t in enumerate(a):
        t[:, -1500:] = _n(1, 1500, H, d, seed=i, std=.3)
    cut = T // 128 * 128 - 1024
    tail = [t[:, cut:].contiguous() for t in a]
    (o, hT, _), (to, th, _) = qd.linear_fwd(*a[:3], g), qd.linear_fwd(*tail[:3], g)
    assert torch.equal(o[:, -300:], to[:, -300:]) and torch.equal(hT, th)
    del o, to
    w, tw = qd.linear_bwd(*a[:3], g, None, a[3]), qd.linear_bwd(*tail[:3], g, None, tail[3])
    for n in ("dq", "dk", "dv"):
        assert torch.equal(w[n][:, -300:], tw[n][:, -300:]), n
    del w, tw, a, tail
    torch.cuda.empty_cache()
    D = 4096
    rows = (1 << 20) + 40
    x = torch.zeros(rows, D, dtype=BF, device="cuda")
    x[-200:] = _n(200, D)
    t = x[-100:].contiguous()
    y, s = qd.gated_norm_fwd(x, x)
    ty, ts = qd.gated_norm_fwd(t, t)
    assert torch.equal(y[-100:], ty) and torch.equal(s[:, -100:], ts)
    del y
    gx, gt = qd.gated_norm_bwd(x, x, None, None, x, s), qd.gated_norm_bwd(t, t, None, None, t, ts)
    assert torch.equal(gx["dx"][-100:], gt["dx"]) and torch.equal(gx["dgate"][-100:], gt["dgate"])
    del gx, gt
    q = x.view(1, rows, 32, 128)
    turns = qd.rotary_turns(64)
    r = qd.rotary(q, None, turns)[0]
    assert torch.equal(r[:, -100:], qd.rotary(q[:, -100:].contiguous(), None, turns, start=rows - 100)[0])
    del r, q, x
    torch.cuda.empty_cache()
    B = (1 << 18) // 16 + 1
    state = torch.zeros(B, 16, 128, 128, device="cuda")
    state[-1] = 1.0
    q, k, v = (_n(B, 1, 16, 128, seed=i) for i in range(3))
    o = qd.linear_steps(q, k, v, g[:16], state)
    one = torch.ones(1, 16, 128, 128, device="cuda")
    lone = qd.linear_steps(q[-1:].contiguous(), k[-1:].contiguous(), v[-1:].contiguous(), g[:16], one)
    lf.close("o", o[-1:], lone.double().cpu(), 2.0 ** -7 * lone.double().cpu().abs())        # fewer states: other columns to a CTA, another order
    assert torch.equal(state[-1:], one)


# ---- infinite and NaN -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,at", [(1, 0), (40, 17), (128, 127), (200, 128), (333, 70), (1500, 1290)])
@pytest.mark.parametrize("dk,dv,dtype", [(128, 128, torch.bfloat16), (64, 64, torch.bfloat16), (64, 128, torch.bfloat16), (128, 64, torch.bfloat16),
                                         (64, 64, torch.float32), (128, 128, torch.float32)])
@pytest.mark.parametrize("what", ["q", "k", "v", "dO"])
def test_a_token_that_is_not_finite_reaches_what_follows_it(T, at, dk, dv, dtype, what):
    """What comes before it, in the order of each walk, has the bits that it has without it; so have, of what comes after it, the columns that do
    not take anything of it; the others are not finite."""
    from paper_2606_08804_b200 import binding as qd
    H, col = 4, 5
    gen = torch.Generator(device="cuda").manual_seed(T + at)
    n = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(dtype)  # noqa: E731
    t = {"q": n(1, T, H, dk), "k": n(1, T, H, dk), "v": n(1, T, H, dv), "dO": n(1, T, H, dv)}
    g = torch.tensor([-0.02, -0.9, 0.0, -0.5], device="cuda")
    h0, dhT = n(1, H, dk, dv).float(), n(1, H, dk, dv).float()

    def run(state):
        o, hT, ws = qd.linear_fwd(t["q"], t["k"], t["v"], g, h0 if state else None)
        gr = qd.linear_bwd(t["q"], t["k"], t["v"], g, h0, t["dO"], dhT if state else None)
        assert qd.workspace_status(ws) == 0
        return dict(o=o, hT=hT, dq=gr["dq"], dk=gr["dk"], dv=gr["dv"], dh0=gr["dh0"])
    heads = (0, 1, 3)                                                          # of all but the third
    for state in (True, False):
        clean = run(state)
        keep = t[what].clone()
        for e, h in enumerate(heads):
            t[what][0, at, h, col] = (math.inf, -math.inf, math.nan)[e]
        got = run(state)
        t[what] = keep
        for name in ("o", "dq", "dk", "dv"):
            a, b = got[name][0], clean[name][0]
            assert torch.equal(a[:, 2], b[:, 2]), name                         # another head
            behind = name in ("o", "dq")                                       # these take what is before them, dk and dv what is behind
            apart = slice(0, at) if behind else slice(at + 1, T)
            own = slice(at, T) if behind else slice(0, at + 1)
            # rows' own factors, by which a token reaches its own row alone: of o q, of dq dO, of dk v, of dv k
            if {"o": "q", "dq": "dO", "dk": "v", "dv": "k"}[name] == what:
                rest = torch.ones(T, dtype=torch.bool, device="cuda")
                rest[at] = False
                assert torch.equal(a[rest], b[rest]), name
                assert not a[at, list(heads)].isfinite().any(), name
            elif {"o": "dO", "dq": "q", "dk": "k", "dv": "v"}[name] == what:
                assert torch.equal(a, b), name                                 # takes nothing of it
            else:
                assert torch.equal(a[apart], b[apart]), name
                # the columns' factors: of o v, of dq k, of dk q, of dv dO, one column; else all of them
                if {"o": "v", "dq": "k", "dk": "q", "dv": "dO"}[name] == what:
                    hit = torch.zeros(a.shape[-1], dtype=torch.bool, device="cuda")
                    hit[col] = True
                    assert torch.equal(a[own][:, :, ~hit], b[own][:, :, ~hit]), name
                    assert not a[own][:, list(heads)][..., hit].isfinite().any(), name
                else:
                    assert not a[own][:, list(heads)].isfinite().any(), name
        for name, by in (("hT", "kv"), ("dh0", ("q", "dO"))):
            a, b = got[name][0], clean[name][0]
            assert torch.equal(a[2], b[2]), name
            if what not in by:
                assert torch.equal(a, b), name
            else:
                assert not (a[list(heads), col] if what in "kq" else a[list(heads), :, col]).isfinite().any(), name


@pytest.mark.parametrize("width,dtype", [(127, BF), (128, BF), (130, BF), (1001, F32), (2048, BF), (5001, BF), (9, F32), (16383, BF)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_row_that_is_not_finite_stays_alone(width, dtype, value):
    from paper_2606_08804_b200 import binding as qd
    rows, bad = 67, [0, 5, 31, 66]
    good = [r for r in range(rows) if r not in bad]
    t = {n: _n(rows, width, seed=i, to=dtype) for i, n in enumerate(("x", "gate", "dy", "dt"))}
    w, b, c = (_n(width, seed=9 + i, to=dtype) for i in range(3))

    def run():
        y, st = qd.gated_norm_fwd(t["x"], t["gate"], w, b)
        g = qd.gated_norm_bwd(t["x"], t["gate"], w, b, t["dy"], st)
        z, total, sa = qd.add_norm_fwd(t["x"], t["gate"], c, w, b)
        a = qd.add_norm_bwd(t["x"], t["gate"], c, w, t["dy"], t["dt"], sa)
        return dict(y=y, dx=g["dx"], dgate=g["dgate"], z=z, total=total, ax=a["dx"], ar=a["dresidual"], s=st.t(), sa=sa.t())
    clean = run()
    t["x"][bad, ::3] = value
    got = run()
    for name in clean:
        assert torch.equal(got[name][good], clean[name][good]), name
        assert not got[name][bad].isfinite().all(1).any(), name


@pytest.mark.parametrize("T", [1, 40, 80])
@pytest.mark.parametrize("dk,dv,dtype", [(128, 128, BF), (64, 64, F32), (64, 128, BF)])
def test_states_that_grow(T, dk, dv, dtype):
    """Up to e^(|g| T) = e^80, just inside fp32: chunks that are not full form no factor beyond it.  Exponents cost 2 half steps of their size."""
    from paper_2606_08804_b200 import autograd as qa
    g = torch.tensor([1.0, 0.71, 0.3], device="cuda")
    q, k = (_n(2, T, 3, dk, seed=i, std=dk ** -0.5, to=dtype).requires_grad_() for i in range(2))
    v, h0 = _n(2, T, 3, dv, seed=3, to=dtype).requires_grad_(), _n(2, 3, dk, dv, seed=4, to=F32).requires_grad_()
    o, hT = qa.linear_attention(q, k, v, g, h0)
    leaves = (q, k, v, h0)
    up = (_n(2, T, 3, dv, seed=5, to=dtype), _n(2, 3, dk, dv, seed=6, to=F32))
    got = torch.autograd.grad((o, hT), leaves, up)
    ref = [lf.f64(t) for t in leaves]
    ro = f.linear(*ref[:3], g.double().cpu(), ref[3])
    rg = lf.grads(ro, [u.double().cpu() for u in up], ref)
    for name, a, r in zip(("o", "hT", "dq", "dk", "dv", "dh0"), (o, hT) + got, tuple(ro) + tuple(rg)):
        a, r = a.detach().double().cpu(), r.detach()
        for h in range(3):
            x, y = (a[:, :, h], r[:, :, h]) if name not in ("hT", "dh0") else (a[:, h], r[:, h])
            assert x.isfinite().all(), (name, h)
            # length of the difference: sums of up to 128 products that partly cancel, and for bf16 two roundings a term
            off = float((x - y).norm() / y.norm())
            assert off < (2.0 ** -6 if dtype == BF and name not in ("hT", "dh0") else (2 * 80 + 128) * 2.0 ** -24), (name, h, off)
