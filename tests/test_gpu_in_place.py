"""What the calls write into tensors of their caller is seen by autograd, as torch's own operations in place are."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
SAYS = "modified by an inplace operation"


def _n(*s, seed=0, std=1.0, to=F32):
    return (torch.randn(*s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + sum(s))) * std).to(to)


def _heads(T, seed=0):
    """q, k, v, beta, alpha, lam of one sequence and two heads; T None: a single token."""
    t = [1] if T is None else [1, T]
    return [_n(*t, 2, 64, seed=seed + i, std=.1) for i in range(3)] + [torch.sigmoid(_n(*t, 2, seed=seed + 3 + i)) for i in range(3)]


def test_convolution_state_that_a_graph_saved():
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    x, w, s = _n(2, 20, 16).requires_grad_(), _n(16, 4).requires_grad_(), _n(2, 3, 16)
    want = torch.autograd.grad(qa.short_conv(x, w, None, s, silu=True)[0].sum(), (x, w))
    y, _ = qa.short_conv(x, w, None, s, silu=True)
    keep = s.clone()
    qd.conv_steps(_n(2, 1, 16), w.detach(), None, s, silu=True)
    assert not torch.equal(s, keep)
    with pytest.raises(RuntimeError, match=SAYS):
        torch.autograd.grad(y.sum(), (x, w))
    # a copy handed on instead: the gradients of before
    y, _ = qa.short_conv(x, w, None, keep, silu=True)
    qd.conv_steps(_n(2, 1, 16), w.detach(), None, keep.clone(), silu=True)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y.sum(), (x, w)), want))


def test_outputs_that_the_caller_gave():
    from paper_2606_08804_b200 import binding as qd
    one = dict(u=_n(2, 1, 16), dt=_n(2, 1, 16), A=-_n(16, 4).exp(), Bm=_n(2, 1, 1, 4), Cm=_n(2, 1, 1, 4), D=None, z=None, dt_bias=None)
    w, x = _n(16, 4), _n(2, 1, 16)
    for call in (lambda y: qd.conv_steps(x, w, None, _n(2, 3, 16), y=y), lambda y: qd.scan_steps(**one, state=_n(2, 16, 4), y=y, softplus=True)):
        y, up = torch.zeros(2, 1, 16, device="cuda"), torch.ones(16, device="cuda", requires_grad=True)
        z = y * up                                             # saves y
        assert call(y) is y and float(y.abs().max()) > 0
        with pytest.raises(RuntimeError, match=SAYS):
            z.sum().backward()


@pytest.mark.parametrize("kind", ["step", "steps", "chunk_fwd", "chunk_fwd_static", "chunk_bwd", "scan_steps", "conv_steps"])
def test_versions_count(kind):
    """Every tensor that is written in place counts once a call, those that are read do not, and refused calls write nothing."""
    from paper_2606_08804_b200 import binding as qd
    state = _n(1, 2, 64, 64)
    if kind == "step":
        ins, o = _heads(None), torch.empty(1, 2, 64, device="cuda")
        call, out = lambda: qd.recurrent_step(*ins, state, o), [state, o]
        refused = lambda: qd.recurrent_step(*ins, state, o[:, :1])  # noqa: E731
    elif kind == "steps":
        ins, o = _heads(3), torch.empty(1, 3, 2, 64, device="cuda")
        call, out = lambda: qd.recurrent_steps(*ins, state, o), [state, o]
        refused = lambda: qd.recurrent_steps(*ins, state, o[:, :1])  # noqa: E731
    elif kind == "chunk_fwd":
        ins, o, hT = _heads(70), torch.empty(1, 70, 2, 64, device="cuda"), torch.empty_like(state)
        ins.append(state)
        call, out = lambda: qd.chunk_fwd(*ins, o=o, hT=hT), [o, hT]
        refused = lambda: qd.chunk_fwd(*ins, o=o, hT=hT[:, :1])  # noqa: E731
    elif kind == "chunk_fwd_static":
        ins, o, hT = _heads(70), torch.empty(1, 70, 2, 64, device="cuda"), torch.empty_like(state)
        ins.append(state)
        call, out = lambda: qd.chunk_fwd_static(*ins, o, hT), [o, hT]
        refused = lambda: qd.chunk_fwd_static(*ins, o, hT[:, :1])  # noqa: E731
    elif kind == "chunk_bwd":
        ins = _heads(70)
        ins += [state, _n(1, 70, 2, 64)]
        dq = torch.empty(1, 70, 2, 64, device="cuda")
        call, out = lambda: qd.chunk_bwd(*ins, out={"dq": dq}), [dq]
        refused = lambda: qd.chunk_bwd(*ins, out={"dq": dq[:, :1]})  # noqa: E731
    elif kind == "scan_steps":
        ins = [_n(2, 1, 16), _n(2, 1, 16), -_n(16, 4).exp(), _n(2, 1, 1, 4), _n(2, 1, 1, 4)]
        st, y = _n(2, 16, 4), torch.empty(2, 1, 16, device="cuda")
        call, out = lambda: qd.scan_steps(*ins, None, None, None, st, y, softplus=True), [st, y]
        refused = lambda: qd.scan_steps(*ins, None, None, None, st, y[:1], softplus=True)  # noqa: E731
    else:
        ins = [_n(2, 1, 16), _n(16, 4)]
        st, y = _n(2, 3, 16), torch.empty(2, 1, 16, device="cuda")
        call, out = lambda: qd.conv_steps(*ins, None, st, y), [st, y]
        refused = lambda: qd.conv_steps(*ins, None, st, y[:1])  # noqa: E731
    ins = [t for t in ins if torch.is_tensor(t)]
    before = [t._version for t in out], [t._version for t in ins]
    call()
    assert [t._version for t in out] == [v + 1 for v in before[0]] and [t._version for t in ins] == before[1]
    with pytest.raises(qd.QdeltaError):
        refused()
    assert [t._version for t in out] == [v + 1 for v in before[0]]


def test_inference_tensors_have_no_version_and_are_served():
    from paper_2606_08804_b200 import binding as qd
    with torch.inference_mode():
        s, x, w = _n(2, 3, 16), _n(2, 1, 16), _n(16, 4)
        want = s.clone()
        qd.conv_steps(x, w, None, s)
        assert torch.equal(s[:, 2], x[:, 0]) and torch.equal(s[:, :2], want[:, 1:])
    qd.conv_steps(x.clone(), w.clone(), None, s)               # and outside, as the kernel does not need it
    assert torch.equal(s[:, 2], x[:, 0])


@pytest.mark.parametrize("which", ["scan", "delta"])
def test_initial_state_is_not_needed_for_the_backward(which):
    """Its owner goes on with it in place between forward and backward: the gradients are those of the state as it was."""
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    if which == "scan":
        ins = [_n(2, 40, 16), _n(2, 40, 16), -_n(16, 4).exp(), _n(2, 40, 1, 4), _n(2, 40, 1, 4)]
        f = lambda h: qa.selective_scan(*ins, h0=h, softplus=True)[0]  # noqa: E731
        go_on = lambda h: qd.scan_steps(*[t[:, :1].contiguous().detach() if t.dim() > 2 else t.detach() for t in ins], None, None, None, h, softplus=True)  # noqa: E731
        h0 = _n(2, 16, 4)
    else:
        ins, token = _heads(70), _heads(1, seed=9)
        f = lambda h: qa.qdelta_chunk(*ins, h)[0]  # noqa: E731
        go_on = lambda h: qd.recurrent_steps(*token, h)  # noqa: E731
        h0 = _n(1, 2, 64, 64)
    ins = [t.requires_grad_() for t in ins]
    leaf = h0.clone().requires_grad_()
    want = torch.autograd.grad(f(leaf).sum(), ins + [leaf])
    state = h0.clone()
    y = f(state)
    go_on(state)
    assert not torch.equal(state, h0)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y.sum(), ins), want))
    again = h0.clone().requires_grad_()
    assert torch.equal(torch.autograd.grad(f(again).sum(), again)[0], want[-1])
