"""The layer norm at every shape of a row (lanes, groups of columns) and over many rows to a CTA, element by element against 64 bits.

Bounds to first order in e = 2^-24.  A row: 64 terms in a thread at most, a tree of 10 and the products around them are below 200 roundings, of
values as large as |x| before the mean is taken off, times r.  The weights' gradients: a thread adds up the rows that it takes, then the threads of
a CTA that share columns (256 at most) in a row, then the CTAs' parts, of which 32 threads take every 32nd.
"""
import pytest
import torch

from scan_exact import E, close, told

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
K = 200

CASES = [  # rows, width, dtype, rms: a lane's groups of columns 8 at a time (bf16), 4 (fp32) or single
    # a warp a row with eight groups to a lane: rows enough, 129 to 256 groups
    (2400, 2048, BF, False), (5000, 1504, BF, True), (2400, 1000, F32, False), (2500, 131, BF, False), (2401, 1032, BF, True),
    (2999, 255, F32, True),
    # 65 to 128 groups: four to a lane, forward and backward
    (3001, 1024, BF, False), (700, 520, BF, True), (3000, 400, F32, False), (1777, 512, F32, True), (2000, 101, BF, False), (5000, 127, F32, False),
    # every number of lanes, and rows for three passes of the staying CTAs and a part of one
    (460001, 1, F32, True), (460001, 3, BF, True), (230001, 16, BF, False), (150001, 32, BF, False), (120001, 64, BF, False), (120001, 60, F32, True),
    (60007, 128, BF, True), (60007, 128, F32, False), (30011, 256, BF, False), (30011, 33, F32, False), (15001, 512, BF, False), (15001, 63, BF, True),
    # a CTA a row, several rows to each
    (1000, 4096, BF, False), (800, 3004, F32, False), (700, 300, BF, False), (900, 999, F32, True), (500, 8192, BF, True), (400, 5120, F32, False),
    (300, 16384, BF, False), (300, 16384, F32, True), (310, 5001, BF, False), (299, 16383, F32, False)]


@pytest.mark.parametrize("rows,width,dt,rms", CASES)
def test_every_element(rows, width, dt, rms):
    from paper_2606_08804_b200 import binding as qd
    g = torch.Generator(device="cuda").manual_seed(rows + width)
    n = lambda *s, std=1.0: torch.randn(*s, device="cuda", generator=g) * std  # noqa: E731
    x = (n(rows, width) * n(rows, 1, std=0.5).exp() + 0.3).to(dt)
    w, b, dy, eps = (1 + n(width, std=0.2)).to(dt), n(width, std=0.2).to(dt), n(rows, width).to(dt), 1e-3
    y, stats = qd.norm_fwd(x, w, b, eps, rms=rms)
    got = dict(qd.norm_bwd(x, w, dy, stats, rms=rms), y=y)
    ctas = qd.load().qdelta_norm_workspace_bytes(rows, width, 1 if dt == BF else 0) // (8 * width)
    xd, wd, bd, up = x.double(), w.double(), b.double(), dy.double()
    mean = 0 * xd[:, :1] if rms else xd.mean(-1, keepdim=True)
    r = 1 / torch.sqrt((xd - mean).square().mean(-1, keepdim=True) + eps)
    xh = (xd - mean) * r
    size = xd.abs().amax(-1, keepdim=True) * r
    close("y", y, xh * wd + bd, K * E * (size * float(wd.abs().max()) * (1 + size) + float(bd.abs().max())))
    close("mean", stats[0], mean[:, 0], K * E * xd.abs().amax(-1))
    close("r", stats[1], r[:, 0], K * E * (r * (1 + size ** 2))[:, 0])
    gr = up * wd
    dx = r * (gr - xh * (gr * xh).mean(-1, keepdim=True) - (0 if rms else gr.mean(-1, keepdim=True)))
    bound = K * E * r * gr.abs().amax(-1, keepdim=True) * (1 + size) ** 2
    close("dx", got["dx"], dx, bound)
    adds = rows // max(ctas, 1) + 1 + 256 + ctas // 32 + 6
    for name, v, terms in (("dweight", (up * xh).sum(0), ((up * xh).abs() * adds + up.abs() * size * (1 + size) * K).sum(0)),
                           ("dbias", up.sum(0), up.abs().sum(0) * adds)):
        close(name, got[name], v, E * terms)
        if width > 1:
            assert told(name, v, E * terms) > 0.8, name
    # without what is optional, the same bits
    y2, none = qd.norm_fwd(x, w, b, eps, rms=rms, want_stats=False)
    assert none is None and torch.equal(y2, y)
    only = qd.norm_bwd(x, w, dy, stats, rms=rms, want_dweight=False, want_dbias=False)
    assert only["dweight"] is None and only["dbias"] is None and torch.equal(only["dx"], got["dx"])
