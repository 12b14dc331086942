"""Refusals of the linear attention layer's operators, before anything is enqueued: no GPU is needed."""
import ctypes

import pytest

FAKE = 0x1000            # never dereferenced: validation fails first
INF = float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_2606_08804_b200 import binding, build
    build.build()
    return binding.load()


def _shape(**change):
    from paper_2606_08804_b200.binding import QdLinearShape
    a = dict(B=2, T=64, H=2, dk=128, dv=64, dtype=1)
    a.update(change)
    return ctypes.byref(QdLinearShape(*[a[n] for n in ("B", "T", "H", "dk", "dv", "dtype")]))


def _fwd(lib, shape=None, q=FAKE, k=2 * FAKE, v=3 * FAKE, g=FAKE, h0=None, o=4 * FAKE, hT=None, scale=1.0, ws=FAKE, n=1 << 40, flags=0):
    return lib.qdelta_linear_fwd(shape or _shape(), q, k, v, g, h0, o, hT, scale, ws, n, flags, None)


def _bwd(lib, shape=None, q=FAKE, k=2 * FAKE, v=3 * FAKE, g=FAKE, h0=None, dO=4 * FAKE, dhT=None, dq=5 * FAKE, dk=6 * FAKE, dv=7 * FAKE, dh0=None,
         scale=1.0, ws=FAKE, n=1 << 40, flags=0):
    return lib.qdelta_linear_bwd(shape or _shape(), q, k, v, g, h0, dO, dhT, dq, dk, dv, dh0, scale, ws, n, flags, None)


def _steps(lib, shape=None, q=FAKE, k=2 * FAKE, v=3 * FAKE, g=FAKE, state=4 * FAKE, o=5 * FAKE, scale=1.0, flags=0):
    return lib.qdelta_linear_steps(shape or _shape(), q, k, v, g, state, o, scale, flags, None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), 1), (dict(T=0), 1), (dict(H=-1), 1), (dict(dk=0), 1), (dict(dk=96), 2), (dict(dv=256), 2), (dict(dtype=2), 2),
    (dict(T=(1 << 30) + 1), 2), (dict(H=(1 << 20) + 1), 2), (dict(B=1 << 13, H=1 << 11), 2), (dict(B=1 << 12, T=1 << 20, H=8), 2)])
def test_shapes(lib, change, code):
    s = _shape(**change)
    assert _fwd(lib, s) == code and _bwd(lib, s) == code and _steps(lib, s) == code
    assert lib.qdelta_linear_workspace_bytes(s, 0) == 0 and lib.qdelta_linear_workspace_bytes(s, 1) == 0


def test_attention_arguments(lib):
    need = lib.qdelta_linear_workspace_bytes(_shape(), 0)
    assert need >= 256 and lib.qdelta_linear_workspace_bytes(_shape(), 1) >= 256
    for change, code in ((dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(g=None), 1), (dict(o=None), 1), (dict(o=FAKE), 1),
                         (dict(o=3 * FAKE), 1), (dict(h0=FAKE, hT=FAKE), 1), (dict(scale=INF), 1), (dict(scale=float("nan")), 1), (dict(flags=1), 1),
                         (dict(q=FAKE + 8), 1), (dict(g=FAKE + 2), 1), (dict(hT=FAKE + 4), 1), (dict(ws=None), 3), (dict(n=need - 1), 3)):
        assert _fwd(lib, **change) == code, change
    for change, code in ((dict(dO=None), 1), (dict(dq=None), 1), (dict(dk=None), 1), (dict(dv=None), 1), (dict(dq=FAKE), 1), (dict(dk=4 * FAKE), 1),
                         (dict(dv=6 * FAKE), 1), (dict(dhT=8 * FAKE, dh0=8 * FAKE), 1), (dict(scale=INF), 1), (dict(flags=2), 1),
                         (dict(dv=7 * FAKE + 2), 1), (dict(ws=None), 3), (dict(n=16), 3)):
        assert _bwd(lib, **change) == code, change
    for change in (dict(q=None), dict(state=None), dict(o=None), dict(o=2 * FAKE), dict(state=FAKE + 4), dict(scale=INF), dict(flags=32)):
        assert _steps(lib, **change) == 1, change


def _gated(lib, rows=4, width=64, dtype=1, x=FAKE, gate=FAKE, w=None, b=None, y=FAKE, stats=None, eps=1e-5, flags=0):
    return lib.qdelta_gated_norm_fwd(rows, width, dtype, x, gate, w, b, y, stats, eps, flags, None)


def _added(lib, rows=4, width=64, dtype=1, x=FAKE, res=FAKE, scale=None, w=None, b=None, total=FAKE, y=2 * FAKE, stats=None, eps=1e-5, flags=0):
    return lib.qdelta_add_norm_fwd(rows, width, dtype, x, res, scale, w, b, total, y, stats, eps, flags, None)


@pytest.mark.parametrize("change,code", [
    (dict(rows=0), 1), (dict(width=0), 1), (dict(width=16385), 2), (dict(dtype=3), 2), (dict(rows=1 << 36), 2), (dict(x=None), 1), (dict(y=None), 1),
    (dict(w=FAKE + 8), 1), (dict(eps=-1.0), 1), (dict(eps=INF), 1), (dict(flags=64), 1), (dict(stats=FAKE + 4), 1)])
def test_norms_forward(lib, change, code):
    assert _gated(lib, **change) == code and _added(lib, **change) == code


def test_norms_backward(lib):
    n = lib.qdelta_fused_norm_workspace_bytes(4, 64, 1)
    assert n > 0 and lib.qdelta_fused_norm_workspace_bytes(4, 16385, 1) == 0 and _gated(lib, gate=None) == 1
    assert _added(lib, res=None) == 1 and _added(lib, total=None) == 1 and _added(lib, total=2 * FAKE) == 1 and _added(lib, flags=32) == 1

    def gated(dy=FAKE, stats=FAKE, dx=FAKE, dz=2 * FAKE, dw=None, ws=None, size=0, flags=0):
        return lib.qdelta_gated_norm_bwd(4, 64, 1, FAKE, FAKE, None, None, dy, stats, dx, dz, dw, None, ws, size, flags, None)
    for change, code in ((dict(dy=None), 1), (dict(stats=None), 1), (dict(dx=None), 1), (dict(dz=None), 1), (dict(dz=FAKE), 1), (dict(flags=64), 1),
                         (dict(dw=FAKE), 3), (dict(dw=FAKE, ws=FAKE, size=n - 1), 3)):
        assert gated(**change) == code, change

    def added(x=FAKE, res=FAKE, scale=None, dy=FAKE, dt=None, stats=FAKE, dx=None, dres=3 * FAKE, ds=None, ws=None, size=0, flags=0):
        return lib.qdelta_add_norm_bwd(4, 64, 1, x, res, scale, None, dy, dt, stats, dx, dres, ds, None, None, ws, size, flags, None)
    for change, code in ((dict(res=None), 1), (dict(dy=None), 1), (dict(stats=None), 1), (dict(dres=None), 1), (dict(scale=FAKE), 1),
                         (dict(dx=3 * FAKE), 1), (dict(x=None), 1), (dict(ds=FAKE), 3), (dict(flags=32), 1)):
        assert added(**change) == code, change


@pytest.mark.parametrize("change,code", [
    (dict(B=0), 1), (dict(T=0), 1), (dict(Hq=0), 1), (dict(Hk=-1), 1), (dict(d=0), 1), (dict(pairs=0), 1), (dict(pairs=33), 2), (dict(d=1025), 2),
    (dict(dtype=2), 2), (dict(Hq=(1 << 16) + 1), 2), (dict(B=1 << 16, T=1 << 16), 2), (dict(q=None), 1), (dict(qo=None), 1), (dict(turns=None), 1),
    (dict(k=None), 1), (dict(ko=None), 1), (dict(qo=2 * FAKE), 1), (dict(ko=FAKE), 1), (dict(ko=3 * FAKE), 1), (dict(q=FAKE + 8), 1),
    (dict(turns=FAKE + 4), 1), (dict(positions=FAKE + 4), 1), (dict(scale=INF), 1), (dict(flags=1), 1)])
def test_rotary(lib, change, code):
    a = dict(B=2, T=8, Hq=4, Hk=2, d=64, pairs=32, dtype=1, q=FAKE, k=2 * FAKE, turns=FAKE, positions=None, start=0, qo=3 * FAKE, ko=4 * FAKE, scale=1.0,
             flags=0)
    a.update(change)
    assert lib.qdelta_rotary(*a.values(), None) == code
