"""The selective scan and its gradients in 64 bits, written out (no autograd), and for every element how far 32-bit arithmetic may be off.

The bounds follow the kernels' operations to first order in e = 2^-24, half a step of fp32:
  * a special function (2^x, 1 / x) is within 2 steps, 4 e; an argument of size s that is rounded k times costs s k e;
  * a decay a_t = 2^(dt A log2 e) is off by (|A| of dt's error + e (3 |dt A| + 4.24)) a_t: three roundings of the argument, 2^x, and the
    2e-8 (0.24 e) by which the argument is shifted; a power below 2^-126, the smallest that is not denormal, comes out 0; where a segment's decay is one power of the sum of its steps, n e |dt A| more, n the
    tokens of the longest segment (a sum of n terms);
  * an error of the state decays as the state does: E_t = a_t E_{t-1} + what token t adds, per state and not for the largest of them.
Second-order terms are taken in by the factor SECOND.
"""
import torch

E = 2.0 ** -24
SECOND = 1.05
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}          # half a step of the type, relative to the value


def _d(t):
    return None if t is None else t.detach().double()


def scan(u, dt, A, Bm, Cm, D=None, z=None, dt_bias=None, h0=None, softplus=False, dy=None, dhT=None, cut=(0, 0)):
    """-> {name: (value, bound)} of y, hT and, with dy, the gradients.  cut: tokens of the longest segment of the forward and of the
    backward, 0 where a sequence is one segment."""
    u, dt, A, Bm, Cm, D, z, bias, h0, dy, dhT = (_d(t) for t in (u, dt, A, Bm, Cm, D, z, dt_bias, h0, dy, dhT))
    B, T, C = u.shape
    N, G = A.shape[1], Bm.shape[2]
    K = C // G
    grouped = lambda m: m.repeat_interleave(K, 2)  # noqa: E731                  [B, T, C, N]
    v = dt if bias is None else dt + bias
    if softplus:
        low = torch.log1p(torch.exp(-v.abs()))
        dt = low + torch.clamp(v, min=0)
        slope = torch.sigmoid(v)
        e_dt = E * (v.abs() * slope + low * (2 * v.abs() + 14) + 2 * dt)
    else:
        dt, slope, e_dt = v, None, E * v.abs()
    x = dt * u
    e_x = e_dt * u.abs() + E * x.abs()
    arg = dt[..., None] * A
    a = torch.exp(arg)
    known = A.abs() * e_dt[..., None]
    ra = a * (known + E * (3 * arg.abs() + 4.24)) + torch.clamp(a, max=2.0 ** -126)          # error of a decay
    ra_f, ra_b = (ra + a * E * n * arg.abs() for n in cut)
    BB, CC = grouped(Bm), grouped(Cm)
    xB = x[..., None] * BB
    add = e_x[..., None] * BB.abs() + E * xB.abs()
    h = h0 if h0 is not None else u.new_zeros(B, C, N)
    e = torch.zeros_like(h)
    hs, es = [h], [e]
    for t in range(T):
        n = a[:, t] * h + xB[:, t]
        e = a[:, t] * e + ra_f[:, t] * h.abs() + add[:, t] + E * n.abs()
        h = n
        hs.append(h)
        es.append(e)
    hs, es = torch.stack(hs, 1), torch.stack(es, 1)
    before, e_before, after, e_after = hs[:, :-1], es[:, :-1], hs[:, 1:], es[:, 1:]
    raw = (CC * after).sum(-1)
    e_raw = (CC.abs() * e_after).sum(-1) + 10 * E * (CC * after).abs().sum(-1)
    if D is not None:
        e_raw = e_raw + 2 * E * ((D * u).abs() + raw.abs())
        raw = raw + D * u
    y, e_y = raw, e_raw
    if z is not None:
        sig = torch.sigmoid(z)
        silu = z * sig
        y = raw * silu
        e_y = e_raw * silu.abs() + y.abs() * (2 * z.abs() + 14) * E
    out = {"y": (y, e_y), "hT": (h, e)}
    if dy is not None:
        gy, e_gy = dy, 0 * dy
        if z is not None:
            gy = dy * silu
            e_gy = E * gy.abs() * (2 * z.abs() + 14)
            gate = sig * (1 + z * (1 - sig))
            e_gate = E * (1 + z.abs()) * (2 * z.abs() + 16)
            out["dz"] = dy * gate * raw, dy.abs() * (e_gate * raw.abs() + gate.abs() * e_raw) + 2 * E * (dy * gate * raw).abs()
        ga = dhT if dhT is not None else torch.zeros_like(h)
        e_ga = torch.zeros_like(ga)
        gts, e_gts, gas, e_gas = [None] * T, [None] * T, [None] * T, [None] * T
        for t in reversed(range(T)):
            c = gy[:, t, :, None] * CC[:, t]
            gt = c + ga
            e_gt = e_gy[:, t, :, None] * CC[:, t].abs() + e_ga + E * gt.abs()
            ga = gt * a[:, t]
            e_ga = a[:, t] * e_gt + ra_b[:, t] * gt.abs() + E * ga.abs()
            gts[t], e_gts[t], gas[t], e_gas[t] = gt, e_gt, ga, e_ga
        gt, e_gt, gas, e_gas = (torch.stack(m, 1) for m in (gts, e_gts, gas, e_gas))
        del gts, e_gts
        out["dh0"] = ga, e_ga
        gp = gas * before
        e_gp = e_gas * before.abs() + gas.abs() * e_before + E * gp.abs()
        del gas, e_gas, before, e_before
        gB = (gt * BB).sum(-1)
        e_gB = (e_gt * BB.abs()).sum(-1) + 10 * E * (gt * BB).abs().sum(-1)
        gA = (gp * A).sum(-1)
        e_gA = (e_gp * A.abs()).sum(-1) + 14 * E * (gp * A).abs().sum(-1)
        du = gB * dt + (0 if D is None else D * gy)
        e_du = e_gB * dt.abs() + gB.abs() * e_dt + 2 * E * (gB * dt).abs() + E * du.abs()
        out["du"] = du, e_du + (0 if D is None else D.abs() * e_gy + 2 * E * (D * gy).abs())
        ddt = gB * u + gA
        e_ddt = e_gB * u.abs() + e_gA + 2 * E * ((gB * u).abs() + gA.abs())
        if softplus:
            e_ddt = slope * e_ddt + (ddt * slope).abs() * (3 * v.abs() + 16) * E
            ddt = ddt * slope
        out["ddt"] = ddt, e_ddt
        # a thread adds a tile of 8 tokens after the other, 8 threads share a channel; then the sequences' and segments' parts, one by one up
        # to 32 of them, else by 32 threads
        most = T / 8 + 48 + B * T / 1024
        out["ddt_bias"] = ddt.sum((0, 1)), e_ddt.sum((0, 1)) + most * E * ddt.abs().sum((0, 1))
        out["dD"] = (gy * u).sum((0, 1)), (e_gy * u.abs()).sum((0, 1)) + most * E * (gy * u).abs().sum((0, 1))
        step, e_step = dt[..., None], e_dt[..., None]
        out["dA"] = (step * gp).sum((0, 1)), (step.abs() * e_gp + e_step * gp.abs()).sum((0, 1)) + (most + 8) * E * (step * gp).abs().sum((0, 1))
        wide = 14 + K / 16                                      # channels: two in a lane, 8 lanes, 4 warps, one CTA after the other
        groups = lambda m: m.reshape(B, T, G, K, N).sum(3)  # noqa: E731
        out["dBm"] = groups(gt * x[..., None]), groups(e_gt * x[..., None].abs() + gt.abs() * e_x[..., None] + wide * E * (gt * x[..., None]).abs())
        gh = gy[..., None] * after
        out["dCm"] = groups(gh), groups(e_gy[..., None] * after.abs() + gy[..., None].abs() * e_after + wide * E * gh.abs())
    return {n: (r, SECOND * b) for n, (r, b) in out.items()}


def told(name, r, bound):
    """Share of the elements whose value is above the bound: of which the bound would notice that they are missing."""
    return float((r.abs() > bound).double().mean())


def close(name, got, ref, bound):
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    off = (got.detach().double() - ref).abs()
    most = HALF[got.dtype] * ref.abs() + bound
    bad = ~(off <= most)
    assert not bad.any(), "%s: %d of %d off, worst %.3g times the allowed, at %s" % (
        name, int(bad.sum()), bad.numel(), float((off / most)[bad].nan_to_num(float("inf")).max()), bad.nonzero()[0].tolist())
