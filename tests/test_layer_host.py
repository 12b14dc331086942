"""Refusals of the operators around the delta rule, before anything is enqueued: no GPU is needed."""
import ctypes

import pytest
import torch

FAKE = 0x1000            # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    from paper_2606_08804_b200 import binding, build
    build.build()
    return binding.load()


def _conv(lib, B=2, T=8, D=64, W=4, dtype=1, x=FAKE, w=FAKE, bias=None, state=None, y=2 * FAKE, last=None, flags=0):
    return lib.qdelta_conv_fwd(B, T, D, W, dtype, x, w, bias, state, y, last, flags, None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), 1), (dict(T=0), 1), (dict(D=-1), 1), (dict(W=0), 1), (dict(W=1), 2), (dict(W=5), 2), (dict(dtype=7), 2),
    (dict(T=(1 << 30) + 1), 2), (dict(D=(1 << 20) + 1), 2), (dict(B=1 << 20, T=1 << 20), 2), (dict(x=None), 1), (dict(w=None), 1), (dict(y=None), 1),
    (dict(y=FAKE), 1), (dict(x=FAKE + 2), 1), (dict(bias=FAKE + 8), 1), (dict(state=FAKE + 4), 1), (dict(state=FAKE, last=FAKE), 1),
    (dict(flags=1), 1), (dict(flags=64), 1)])
def test_convolution_forward(lib, change, code):
    assert _conv(lib, **change) == code


def test_convolution_steps_and_backward(lib):
    step = lambda *a: lib.qdelta_conv_steps(2, 1, 64, 4, 1, *a, 0, None)  # noqa: E731
    assert step(FAKE, FAKE, None, None, 2 * FAKE) == 1 and step(FAKE, FAKE, None, FAKE, FAKE) == 1 and step(FAKE, FAKE, None, FAKE + 2, 2 * FAKE) == 1
    back = lambda bias, dbias, dx, ws, n: lib.qdelta_conv_bwd(  # noqa: E731
        2, 8, 64, 4, 1, FAKE, FAKE, bias, None, 3 * FAKE, None, dx, FAKE, dbias, None, ws, n, 0, None)
    need = lib.qdelta_conv_workspace_bytes(2, 8, 64, 4, 1)
    assert need > 0 and lib.qdelta_conv_workspace_bytes(2, 8, 64, 5, 1) == 0
    assert back(FAKE, None, 2 * FAKE, FAKE, need) == 1                 # bias without dbias
    assert back(None, None, FAKE, FAKE, need) == 1                     # dx over x
    assert back(None, None, 3 * FAKE, FAKE, need) == 1                 # dx over dy
    state = lambda dlast, dstate: lib.qdelta_conv_bwd(  # noqa: E731
        2, 8, 64, 4, 1, FAKE, FAKE, None, None, 3 * FAKE, dlast, 2 * FAKE, FAKE, None, dstate, None, 0, 0, None)
    assert state(4 * FAKE, 4 * FAKE) == 1 and state(4 * FAKE, 5 * FAKE) == 3        # one buffer for both; no workspace
    assert back(None, None, 2 * FAKE, FAKE, need - 1) == 3 and back(None, None, 2 * FAKE, None, need) == 3


def _shape(**change):
    from paper_2606_08804_b200.binding import QdScanShape
    a = dict(B=2, T=64, D=128, N=16, G=1, dtype=1)
    a.update(change)
    return QdScanShape(*[a[n] for n in ("B", "T", "D", "N", "G", "dtype")])


@pytest.mark.parametrize("change,code", [
    (dict(B=0), 1), (dict(T=0), 1), (dict(N=0), 1), (dict(G=0), 1), (dict(N=65), 2), (dict(G=3), 2), (dict(dtype=2), 2), (dict(T=(1 << 30) + 1), 2),
    (dict(D=(1 << 20) + 1), 2), (dict(B=1 << 20, D=1 << 11), 2)])
def test_scan_shapes(lib, change, code):
    s = _shape(**change)
    r = ctypes.byref(s)
    assert lib.qdelta_scan_fwd(r, *[FAKE] * 5, None, None, None, None, FAKE, None, FAKE, 1 << 40, 0, None) == code
    assert lib.qdelta_scan_bwd(r, *[FAKE] * 5, None, None, None, None, FAKE, None, *[FAKE] * 5, None, None, None, None, FAKE, 1 << 40, 0, None) == code
    assert lib.qdelta_scan_steps(r, *[FAKE] * 5, None, None, None, FAKE, FAKE, 0, None) == code
    assert lib.qdelta_scan_workspace_bytes(r, 1) == 0


def test_scan_arguments(lib):
    s = _shape()
    r = ctypes.byref(s)
    need = lib.qdelta_scan_workspace_bytes(r, 1)
    fwd = lambda u=FAKE, y=FAKE, h0=None, ws=FAKE, n=need, flags=1: lib.qdelta_scan_fwd(  # noqa: E731
        r, u, FAKE, FAKE, FAKE, FAKE, None, None, None, h0, y, None, ws, n, flags, None)
    assert need > lib.qdelta_scan_workspace_bytes(r, 0)
    assert fwd(u=None) == 1 and fwd(y=None) == 1 and fwd(h0=FAKE + 4) == 1 and fwd(flags=1 | 32) == 1 and fwd(flags=2) == 1
    assert fwd(n=need - 1) == 3 and fwd(ws=None) == 3
    bwd = lambda D=None, dD=None, z=None, dz=None, b=None, db=None, ws=FAKE, n=need: lib.qdelta_scan_bwd(  # noqa: E731
        r, FAKE, FAKE, FAKE, FAKE, FAKE, D, z, b, None, FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE, dD, dz, db, None, ws, n, 2, None)
    assert bwd(D=FAKE) == 1 and bwd(z=FAKE) == 1 and bwd(b=FAKE) == 1 and bwd(n=need - 1) == 3 and bwd(ws=None) == 3
    # one buffer for the states before and after, and for their gradients; with two it is the workspace that is missing
    states = lambda h0, hT: lib.qdelta_scan_fwd(r, *[FAKE] * 5, None, None, None, h0, FAKE, hT, None, 0, 1, None)  # noqa: E731
    assert states(FAKE, FAKE) == 1 and states(FAKE, 2 * FAKE) == 3
    grads = lambda dhT, dh0: lib.qdelta_scan_bwd(  # noqa: E731
        r, *[FAKE] * 5, None, None, None, FAKE, FAKE, dhT, *[FAKE] * 5, None, None, None, dh0, None, 0, 0, None)
    assert grads(FAKE, FAKE) == 1 and grads(FAKE, 2 * FAKE) == 3
    # a forward of many channels needs no workspace, one of few long sequences does
    assert lib.qdelta_scan_workspace_bytes(ctypes.byref(_shape(B=64, D=2048)), 0) == 0
    assert lib.qdelta_scan_workspace_bytes(ctypes.byref(_shape(B=1, T=4096, D=128)), 0) > 0


@pytest.mark.parametrize("rows,width,dtype,code", [(0, 64, 1, 1), (4, 0, 1, 1), (4, 16385, 1, 2), (4, 64, 9, 2), (1 << 36, 1, 0, 2), (1 << 28, 1024, 1, 2)])
def test_norm_shapes(lib, rows, width, dtype, code):
    assert lib.qdelta_norm_fwd(rows, width, dtype, FAKE, None, None, FAKE, None, 1e-5, 0, None) == code
    assert lib.qdelta_norm_bwd(rows, width, dtype, FAKE, None, FAKE, FAKE, FAKE, None, None, None, 0, 0, None) == code
    assert lib.qdelta_norm_workspace_bytes(rows, width, dtype) == 0


def test_norm_arguments(lib):
    fwd = lambda x=FAKE, y=FAKE, eps=1e-5, flags=0, w=None: lib.qdelta_norm_fwd(4, 64, 1, x, w, None, y, None, eps, flags, None)  # noqa: E731
    assert fwd(x=None) == 1 and fwd(y=None) == 1 and fwd(eps=-1e-5) == 1 and fwd(eps=float("nan")) == 1 and fwd(eps=float("inf")) == 1
    assert fwd(flags=1) == 1 and fwd(w=FAKE + 8) == 1
    need = lib.qdelta_norm_workspace_bytes(4, 64, 1)
    bwd = lambda dw, ws, n, stats=FAKE: lib.qdelta_norm_bwd(4, 64, 1, FAKE, None, FAKE, stats, FAKE, dw, None, ws, n, 0, None)  # noqa: E731
    assert bwd(FAKE, None, 0) == 3 and bwd(FAKE, FAKE, need - 1) == 3 and bwd(None, None, 0, stats=None) == 1


def test_binding_refuses_what_no_kernel_could_read():
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    z = torch.zeros
    for call in (lambda: qd.conv_fwd(z(1, 4, 8), z(8, 4)), lambda: qd.conv_steps(z(1, 1, 8), z(8, 4), None, z(1, 3, 8)),
                 lambda: qd.scan_fwd(z(1, 4, 8), z(1, 4, 8), z(8, 2), z(1, 4, 1, 2), z(1, 4, 1, 2)), lambda: qd.norm_fwd(z(4, 8)),
                 lambda: qa.short_conv(z(1, 4, 8), z(8, 4)), lambda: qa.layer_norm(z(4, 8, requires_grad=True)),
                 lambda: qa.selective_scan(z(1, 4, 8), z(1, 4, 8), z(8, 2), z(1, 4, 1, 2), z(1, 4, 1, 2))):
        with pytest.raises(qd.QdeltaError, match="CUDA"):
            call()
    with pytest.raises(qd.QdeltaError, match="workspace"):
        qd.scan_bwd(*[None] * 10, reuse_fwd=True)
    with pytest.raises(TypeError, match="w must be a tensor"):
        qd.conv_fwd(z(1, 4, 8), None)
    with pytest.raises(TypeError, match="tensor"):
        qd.norm_fwd([1.0])
