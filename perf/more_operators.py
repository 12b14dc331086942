"""The operators of a layer of linear attention, as cases that can be timed and compared: the rotation of queries and keys before
it, linear attention with a decay for each head, the gated norm of its read-out, and the norm after the residual sum.

A case is one pass through one operator: a training step (forward and backward), a prompt (forward that also returns the
state) or decode steps (state updated in place).  `run` computes it in elementary torch operations in fp32, or, where `own`
is true, through the library's public entry points.  `exact` computes the definition in fp64.

    linear      S_t = e^g S_{t-1} + k_t v_t^T ,  o_t = scale S_t^T q_t     per head, g = log_decay of the head
    gated norm  y = ((x - mean) rstd w + b) f(gate) over the last dimension, f = SiLU or the logistic function; rms: mean = 0
    add norm    total = residual + scale x ,  y = norm(total)     scale per channel or absent
    rotary      the pairs (x_j, x_{j+R}), or (x_2j, x_2j+1), j < R, turned by position * frequency_j and scaled; the rest as it is
"""
import math

import torch

own = False

EPS = 1e-5
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases --------------------------------------------------------------------------------------------------------
# kind  "train"    forward and backward through the two calls that a training loop of its own makes
#       "autograd" the same pair through torch.autograd
#       "prefill"  forward only, state handed on
#       "steps"    T tokens per sequence, state updated in place

def _linear(kind, B, T, H, dk=128, dv=128, dtype="bf16", state=False):
    return {"op": "linear", "kind": kind, "B": B, "T": T, "H": H, "dk": dk, "dv": dv, "dtype": dtype, "state": state}


def _gated(kind, rows, width, dtype="bf16", rms=True, silu=True, weight=True, bias=False):
    return {"op": "gated", "kind": kind, "rows": rows, "width": width, "dtype": dtype, "rms": rms, "silu": silu, "weight": weight, "bias": bias}


def _added(kind, rows, width, dtype="bf16", rms=False, scale=True, weight=True, bias=False):
    return {"op": "added", "kind": kind, "rows": rows, "width": width, "dtype": dtype, "rms": rms, "scale": scale, "weight": weight, "bias": bias}


def _rotary(kind, B, T, Hq, Hk, d=128, pairs=64, dtype="bf16", interleaved=False, positions="count", stretch=1.0, scale=1.0):
    return {"op": "rotary", "kind": kind, "B": B, "T": T, "Hq": Hq, "Hk": Hk, "d": d, "pairs": pairs, "dtype": dtype,
            "interleaved": interleaved, "positions": positions, "stretch": stretch, "scale": scale}


def listed():
    c = [
        # the headline layer's heads (16 of 128): training step of 16384 tokens (the largest case)
        ("linear train lm", _linear("train", 8, 2048, 16)),
        # a small full-precision layer through torch.autograd, ragged length, initial state
        ("linear autograd ragged f32", _linear("autograd", 2, 1000, 4, 64, 64, "f32", True)),
        # a context of 32768 tokens, one sequence of 16 heads: few heads, many tokens
        ("linear prefill long", _linear("prefill", 1, 32768, 16)),
        # one user's prompt of odd length, going on from a cached state
        ("linear prefill one ragged", _linear("prefill", 1, 777, 16, state=True)),
        # one token for each of 256 sequences
        ("linear decode 256", _linear("steps", 256, 1, 16, state=True)),
        # read-out of the headline layer per head, gated: 16384 tokens x 16 heads of 128
        ("gated norm train heads", _gated("train", 262144, 128)),
        # the same while decoding 256 sequences
        ("gated norm decode 256", _gated("prefill", 4096, 128)),
        # residual sum and norm before the next layer, 16384 tokens
        ("add norm train lm", _added("train", 16384, 2048, rms=True)),
        # the same with mean and bias, full precision, odd width, through torch.autograd
        ("add norm autograd odd f32", _added("autograd", 1018, 1001, "f32", scale=False, bias=True)),
        # the same norm for one token of each of 256 sequences
        ("add norm decode 256", _added("prefill", 256, 2048, rms=True, scale=False)),
        # queries and keys of the headline layer, 16384 tokens, forward and backward
        ("rotary train lm", _rotary("train", 8, 2048, 16, 16)),
        # one token for each of 256 sequences at far positions: half of the head, interleaved, four key heads, a stretched context
        ("rotary decode 256 far", _rotary("prefill", 256, 1, 16, 4, 128, 32, interleaved=True, positions="far", stretch=8.0, scale=1.2)),
    ]
    return [dict(d, name=n) for n, d in c]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _even(rng, n, m):
    """n as drawn, or near it a multiple of m."""
    return max(m, n // m * m) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["linear", "linear", "gated", "added", "rotary"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    flag = lambda p: rng.random() < p  # noqa: E731
    if op in ("gated", "added"):
        width = _even(rng, _log_int(rng, 1, 16384), 64)
        rows = _log_int(rng, 1, max(1, min(262144, (1 << (25 if dtype == "bf16" else 24)) // width)))
        kind = rng.choice(["train", "train", "autograd", "prefill"])
        make = _gated if op == "gated" else _added
        return make(kind, rows, width, dtype, flag(0.5), flag(0.6), flag(0.9), flag(0.4))
    if op == "rotary":
        d = 2 * _even(rng, _log_int(rng, 1, 128), 8)
        pairs = d // 2 if flag(0.6) else rng.randint(1, d // 2)
        Hq = _log_int(rng, 1, 24)
        Hk = rng.choice([Hq, max(1, Hq // 4), 0])
        T = min(rng.choice([1, _even(rng, _log_int(rng, 1, 16384), 64)]), (1 << 24) // (d * (Hq + Hk)))
        B = min(_log_int(rng, 1, 256), max(1, (1 << (25 if dtype == "bf16" else 24)) // (T * d * (Hq + Hk))))
        return _rotary(rng.choice(["train", "autograd", "prefill"]), B, T, Hq, Hk, d, pairs, dtype, flag(0.5), rng.choice(["count", "start", "far"]),
                       rng.choice([1.0, 4.0]), rng.choice([1.0, 1.0, 0.5]))
    dk, dv, H = rng.choice([64, 128]), rng.choice([64, 128]), _log_int(rng, 1, 32)
    if flag(0.25):
        return _linear("steps", _log_int(rng, 1, max(1, 3600 // H)), rng.randint(1, 8), H, dk, dv, dtype, True)
    T = _even(rng, _log_int(rng, 1, 32768), 64)
    most = 1 << (18 if dtype == "bf16" else 16)
    H = min(H, max(1, most // T))
    B = min(_log_int(rng, 1, 32), max(1, (most - most // 16) // ((T + 128) * H)))
    return _linear(rng.choice(["train", "autograd", "prefill"]), B, T, H, dk, dv, dtype, flag(0.4))


# ---- inputs -----------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = _DT[case["dtype"]]

    def normal(*dims, std=1.0, to=dt):
        return (torch.randn(*dims, device="cuda", generator=gen) * std).to(to)

    def uniform(*dims):
        return torch.rand(*dims, device="cuda", generator=gen)

    s, kind = {"case": case}, case["kind"]
    train = kind in ("train", "autograd")
    if case["op"] in ("gated", "added"):
        rows, width = case["rows"], case["width"]
        # activations: rows of different scale, a few channels that stand out
        x = normal(rows, width, to=torch.float32) * normal(rows, 1, std=0.5, to=torch.float32).exp()
        x = (x * (1.0 + 4.0 * (uniform(width) < 0.01)) + 0.3).to(dt)
        s["weight"] = (1.0 + normal(width, std=0.2, to=torch.float32)).to(dt) if case["weight"] else None
        s["bias"] = normal(width, std=0.2) if case["bias"] else None
        s["dy"] = normal(rows, width) if train else None
        if case["op"] == "gated":
            s["x"], s["gate"] = x, normal(rows, width, std=1.5)
            wanted = ("x", "gate", "weight", "bias")
        else:
            # what a block adds to the stream, scaled by a trained factor per channel
            s["x"], s["residual"] = normal(rows, width), x
            s["scale"] = (uniform(width) + 0.1).to(dt) if case["scale"] else None
            s["dtotal"] = normal(rows, width) if train else None
            wanted = ("x", "residual", "scale", "weight", "bias")
    elif case["op"] == "rotary":
        B, T, d = case["B"], case["T"], case["d"]
        s["q"] = normal(B, T, case["Hq"], d)
        s["k"] = normal(B, T, case["Hk"], d) if case["Hk"] else None
        s["start"], s["positions"] = 0, None
        if case["positions"] == "start":
            s["start"] = 1000 + seed % 1000
        elif case["positions"] == "far":
            s["positions"] = torch.randint(0, 1 << 20, (B, 1), device="cuda", generator=gen) + torch.arange(T, device="cuda")
        s["dq"] = normal(B, T, case["Hq"], d) if train else None
        s["dk"] = normal(B, T, case["Hk"], d) if train and case["Hk"] else None
        if own:
            from paper_2606_08804_b200 import binding as qd
            s["turns"] = qd.rotary_turns(case["pairs"], base=10000.0, factor=case["stretch"], device="cuda")
        wanted = ("q", "k")
    else:
        B, T, H, dk, dv = (case[n] for n in ("B", "T", "H", "dk", "dv"))
        unit = lambda x: (x / x.square().sum(-1, keepdim=True).sqrt()).to(dt)  # noqa: E731
        s["q"] = unit(normal(B, T, H, dk, to=torch.float32) + 0.3)
        s["k"] = unit(normal(B, T, H, dk, to=torch.float32) + 0.3)
        s["v"] = normal(B, T, H, dv)
        # what heads remember: from 2 tokens to a few hundred
        s["log_decay"] = torch.log1p(-torch.exp2(-1.0 - 7.0 * (torch.arange(H, device="cuda") + uniform(H)) / H))
        s["h0"] = normal(B, H, dk, dv, std=0.2, to=torch.float32) if case["state"] else None
        s["scale"] = 1.0 if case["state"] else 1.0 / math.sqrt(dk)
        if train:
            s["do"] = normal(B, T, H, dv)
            s["dhT"] = normal(B, H, dk, dv, std=0.2, to=torch.float32) if case["state"] else None
        wanted = ("q", "k", "v", "h0")
    if kind == "autograd":
        s["wanted"] = {n: s[n].requires_grad_() for n in wanted if s[n] is not None}
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _own(s)
    with torch.no_grad():
        return {"linear": _plain_linear, "gated": _plain_gated, "added": _plain_added, "rotary": _plain_rotary}[s["case"]["op"]](s)


def _own(s):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    case = s["case"]
    kind = case["kind"]
    if case["op"] == "gated":
        args, how = (s["x"], s["gate"], s["weight"], s["bias"]), {"rms": case["rms"], "silu": case["silu"]}
        if kind == "autograd":
            y = qa.gated_norm(*args, EPS, **how)
            return {"y": y.detach(), **_grads(s, (y,), (s["dy"],))}
        y, stats = qd.gated_norm_fwd(*args, EPS, **how)
        return {"y": y} if kind == "prefill" else {"y": y, **_kept(qd.gated_norm_bwd(*args, s["dy"], stats, **how))}
    if case["op"] == "added":
        args, rms = (s["x"], s["residual"], s["scale"], s["weight"], s["bias"]), case["rms"]
        if kind == "autograd":
            y, total = qa.add_norm(*args, EPS, rms=rms)
            return {"y": y.detach(), "total": total.detach(), **_grads(s, (y, total), (s["dy"], s["dtotal"]))}
        y, total, stats = qd.add_norm_fwd(*args, EPS, rms=rms)
        if kind == "prefill":
            return {"y": y, "total": total}
        g = qd.add_norm_bwd(s["x"], s["residual"], s["scale"], s["weight"], s["dy"], s["dtotal"], stats, rms=rms, want_dbias=case["bias"])
        return {"y": y, "total": total, **_kept(g)}
    if case["op"] == "rotary":
        how = {"positions": s["positions"], "start": s["start"], "interleaved": case["interleaved"], "scale": case["scale"]}
        if kind == "autograd":
            y = [t for t in qa.rotary(s["q"], s["k"], s["turns"], **how) if t is not None]
            return {**{n: t.detach() for n, t in zip(("q", "k"), y)}, **_grads(s, y, [s[n] for n in ("dq", "dk") if s[n] is not None])}
        q, k = qd.rotary(s["q"], s["k"], s["turns"], **how)
        out = {"q": q, "k": k}
        if kind == "train":
            dq, dk = qd.rotary(s["dq"], s["dk"], s["turns"], inverse=True, **how)
            out["grads"] = {"dq": dq, "dk": dk}
        return _present(out)
    args, scale = (s["q"], s["k"], s["v"], s["log_decay"]), s["scale"]
    if kind == "steps":
        return {"o": qd.linear_steps(*args, s["h0"], scale=scale), "state": s["h0"]}
    if kind == "autograd":
        o, hT = qa.linear_attention(*args, s["h0"], scale=scale)
        outs, ups = ((o, hT), (s["do"], s["dhT"])) if s["dhT"] is not None else ((o,), (s["do"],))
        return {"o": o.detach(), "hT": hT.detach(), **_grads(s, outs, ups)}
    o, hT, _ = qd.linear_fwd(*args, s["h0"], scale=scale)
    if kind == "prefill":
        return {"o": o, "hT": hT}
    return {"o": o, "hT": hT, **_kept(qd.linear_bwd(*args, s["h0"], s["do"], s["dhT"], scale=scale))}


def _grads(s, outs, ups):
    g = torch.autograd.grad(outs, list(s["wanted"].values()), ups)
    return {"grads": {"d" + n: x for n, x in zip(s["wanted"], g)}}


def _kept(g):
    return {"grads": {n: x for n, x in g.items() if x is not None}}


def _present(out):
    return {n: _present(x) if isinstance(x, dict) else x for n, x in out.items() if x is not None}


def _named(s, g):
    """Gradients under the names and in the types of the entry points: those of parameters are fp32 in a training loop of its
    own, and of the parameter's type through torch.autograd."""
    auto = s["case"]["kind"] == "autograd"
    out = {}
    for n, x in g.items():
        like = s[n[1:]]
        if like is not None:
            out[n] = x.reshape(like.shape).to(torch.float32 if n in ("dscale", "dweight", "dbias") and not auto else like.dtype)
    return {"grads": out}


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _wide(x):
    return x.float() if x is not None else None


def _normed(x, rms):
    c = x if rms else x - x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
    return c * rstd, rstd


def _norm_slope(xh, rstd, g, rms):
    dx = g - xh * (g * xh).mean(-1, keepdim=True)
    return (dx if rms else dx - g.mean(-1, keepdim=True)) * rstd


def _plain_gated(s):
    case, dt = s["case"], s["x"].dtype
    w, b, z = _wide(s["weight"]), _wide(s["bias"]), s["gate"].float()
    xh, rstd = _normed(s["x"].float(), case["rms"])
    n = xh if w is None else xh * w
    n = n if b is None else n + b
    sig = _sigmoid(z)
    f = z * sig if case["silu"] else sig
    y = (n * f).to(dt)
    if case["kind"] == "prefill":
        return {"y": y}
    dy = s["dy"].float()
    dn = dy * f
    dgate = dy * n * (sig * (1.0 + z * (1.0 - sig)) if case["silu"] else sig * (1.0 - sig))
    dx = _norm_slope(xh, rstd, dn if w is None else dn * w, case["rms"])
    return {"y": y, **_named(s, {"dx": dx, "dgate": dgate, "dweight": (dn * xh).sum(0), "dbias": dn.sum(0)})}


def _plain_added(s):
    case, dt = s["case"], s["x"].dtype
    w, b, c, x = _wide(s["weight"]), _wide(s["bias"]), _wide(s["scale"]), s["x"].float()
    total = s["residual"].float() + (x if c is None else x * c)
    xh, rstd = _normed(total, case["rms"])
    y = xh if w is None else xh * w
    out = {"y": (y if b is None else y + b).to(dt), "total": total.to(dt)}
    if case["kind"] == "prefill":
        return out
    dy = s["dy"].float()
    d = _norm_slope(xh, rstd, dy if w is None else dy * w, case["rms"]) + s["dtotal"].float()
    return {**out, **_named(s, {"dx": d if c is None else d * c, "dresidual": d, "dscale": (d * x).sum(0), "dweight": (dy * xh).sum(0), "dbias": dy.sum(0)})}


def _plain_rotary(s):
    case = s["case"]
    R = case["pairs"]
    at = s["positions"] if s["positions"] is not None else s["start"] + torch.arange(case["T"], device="cuda").expand(case["B"], -1)
    freq = torch.exp(torch.arange(R, device="cuda", dtype=torch.float64) * (-math.log(10000.0) / R)) / case["stretch"]
    angle = at.double()[..., None] * freq                                           # far positions: fp32 would lose the angle
    c, n = ((f(angle) * case["scale"]).float()[:, :, None] for f in (torch.cos, torch.sin))

    def turn(x, n):
        if x is None:
            return None
        y = x.float().clone()
        a, b = (y[..., 0:2 * R:2], y[..., 1:2 * R:2]) if case["interleaved"] else (y[..., :R], y[..., R:2 * R])
        a2, b2 = a * c - b * n, a * n + b * c
        a.copy_(a2)
        b.copy_(b2)
        return y.to(x.dtype)

    out = {"q": turn(s["q"], n), "k": turn(s["k"], n)}
    if case["kind"] != "prefill":
        out["grads"] = {"dq": turn(s["dq"], -n), "dk": turn(s["dk"], -n)}
    return _present(out)


def _plain_linear(s):
    """Chunks of 64 tokens: products within a chunk, states between them."""
    case, io = s["case"], s["q"].dtype
    B, T, H, dk, dv = (case[n] for n in ("B", "T", "H", "dk", "dv"))
    g, scale = s["log_decay"], s["scale"]
    h = s["h0"] if s["h0"] is not None else g.new_zeros(B, H, dk, dv)
    if case["kind"] == "steps":
        o = []
        for t in range(T):
            h = torch.exp(g)[:, None, None] * h + s["k"][:, t].float()[..., None] * s["v"][:, t].float()[..., None, :]
            o.append((h * s["q"][:, t].float()[..., None]).sum(-2) * scale)
        s["h0"].copy_(h)
        return {"o": torch.stack(o, 1).to(io), "state": s["h0"]}
    C = 64
    N = (T + C - 1) // C

    def cut(x):                                                                     # [B, T, H, d] -> [N, B, H, C, d]
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, N * C - T))
        return x.reshape(B, N, C, H, -1).permute(1, 0, 3, 2, 4).contiguous()

    def whole(x):
        return x.permute(1, 0, 3, 2, 4).reshape(B, N * C, H, -1)[:, :T].to(io)

    q, k, v = cut(s["q"]), cut(s["k"]), cut(s["v"])
    r = torch.arange(C, device="cuda")
    last = torch.full((N,), C, device="cuda")                                       # tokens of every chunk
    last[-1] = T - (N - 1) * C
    reach = (r[:, None] - r[None, :])
    D = torch.where(reach >= 0, torch.exp(g[:, None, None] * reach.clamp(min=0)), torch.zeros((), device="cuda")) * scale      # [H, C, C]
    rise = (torch.exp(g[:, None] * (r + 1)) * scale)[..., None]                      # [H, C, 1]
    fall = torch.exp(g[:, None] * (last[:, None, None] - 1 - r).clamp(min=0))[:, None, ..., None]     # [N, 1, H, C, 1]
    keep = torch.exp(g * last[:, None])[:, None, :, None, None]                      # [N, 1, H, 1, 1]
    add = (k * fall).transpose(-1, -2) @ v
    before = torch.empty_like(add)
    for n in range(N):
        before[n] = h
        h = keep[n] * h + add[n]
    P = (q @ k.transpose(-1, -2)) * D
    out = {"o": whole(P @ v + (q * rise) @ before), "hT": h}
    if case["kind"] == "prefill":
        return out
    do = cut(s["do"])
    add = (q * rise).transpose(-1, -2) @ do
    dh = s["dhT"] if s["dhT"] is not None else g.new_zeros(B, H, dk, dv)
    after = torch.empty_like(add)
    for n in reversed(range(N)):
        after[n] = dh
        dh = keep[n] * dh + add[n]
    dS = (do @ v.transpose(-1, -2)) * D
    dq = dS @ k + (do @ before.transpose(-1, -2)) * rise
    dk_ = dS.transpose(-1, -2) @ q + (v @ after.transpose(-1, -2)) * fall
    dv_ = P.transpose(-1, -2) @ do + (k @ after) * fall
    return {**out, **_named(s, {"dq": whole(dq), "dk": whole(dk_), "dv": whole(dv_), "dh0": dh})}


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------
def work(case):
    io = 2 if case["dtype"] == "bf16" else 4
    train = case["kind"] in ("train", "autograd")
    if case["op"] == "gated":
        n, p = case["rows"] * case["width"], case["width"] * (int(case["weight"]) + int(case["bias"]))
        # read x, gate (and dy), write y (and dx, dgate)
        return {"bytes": float(io * (n * (6 if train else 3) + p) + (4 * p if train else 0)), "flops": n * (40.0 if train else 14.0)}
    if case["op"] == "added":
        n, p = case["rows"] * case["width"], case["width"] * (int(case["weight"]) + int(case["bias"]) + int(case["scale"]))
        # read x, residual (and dy, dtotal), write total, y (and dresidual, dx)
        return {"bytes": float(io * (n * ((7 + int(case["scale"])) if train else 4) + p) + (4 * p if train else 0)), "flops": n * (30.0 if train else 10.0)}
    if case["op"] == "rotary":
        n = case["B"] * case["T"] * (case["Hq"] + case["Hk"])
        return {"bytes": float(n * case["d"] * io * (4 if train else 2) + case["pairs"] * 8 + (8 * case["B"] * case["T"] if case["positions"] == "far" else 0)),
                "flops": n * case["pairs"] * (16.0 if train else 8.0)}
    B, T, H, dk, dv = (case[n] for n in ("B", "T", "H", "dk", "dv"))
    n, st = B * T * H, B * H * dk * dv
    states = 1 + int(case["state"])
    nbytes = io * n * 2 * (dk + dv) + 4 * states * st
    flops = 4.0 * n * dk * dv                   # the recurrence: the state and the read-out, one product each
    if train:
        nbytes += io * n * (2 * dk + 2 * dv) + (8 * st if case["state"] else 0)
        flops += 10.0 * n * dk * dv             # three products with states, two sums of states
    return {"bytes": float(nbytes), "flops": flops}


# ---- the definition in fp64 -------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        return _exact_linear(case, s)
    if case["op"] == "rotary":
        return _exact_rotary(case, s)
    train = case["kind"] in ("train", "autograd")
    names = ("x", "gate", "weight", "bias") if case["op"] == "gated" else ("x", "residual", "scale", "weight", "bias")
    d = {n: s[n].detach().double().requires_grad_(train) for n in names if s[n] is not None}
    with torch.set_grad_enabled(train):
        x = d["x"] if case["op"] == "gated" else d["residual"] + d.get("scale", 1.0) * d["x"]
        if case["rms"]:
            y = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * d.get("weight", 1.0) + d.get("bias", 0.0)
        else:
            y = torch.nn.functional.layer_norm(x, x.shape[-1:], d.get("weight"), d.get("bias"), EPS)
        if case["op"] == "gated":
            y = y * (torch.nn.functional.silu(d["gate"]) if case["silu"] else torch.sigmoid(d["gate"]))
    outs = {"y": y.detach()} if case["op"] == "gated" else {"y": y.detach(), "total": x.detach()}
    if not train:
        return outs
    pairs = [(y, s["dy"].double())] + ([] if case["op"] == "gated" else [(x, s["dtotal"].double())])
    g = torch.autograd.grad([o for o, _ in pairs], list(d.values()), [u for _, u in pairs])
    return {**outs, "grads": {"d" + n: x for n, x in zip(d, g)}}


def _exact_rotary(case, s):
    R = case["pairs"]
    at = s["positions"] if s["positions"] is not None else torch.arange(s["start"], s["start"] + case["T"], device="cuda")[None].expand(case["B"], case["T"])
    freq = 10000.0 ** (-torch.arange(R, device="cuda", dtype=torch.float64) / R) / case["stretch"]
    phase = torch.polar(torch.full((), float(case["scale"]), device="cuda", dtype=torch.float64), at.double()[..., None] * freq)[:, :, None]

    def turn(x, phase):
        if x is None:
            return None
        x = x.detach().double()
        a, b = (x[..., 0:2 * R:2], x[..., 1:2 * R:2]) if case["interleaved"] else x[..., :2 * R].split(R, -1)
        z = torch.complex(a, b) * phase
        pair = torch.stack((z.real, z.imag), -1).flatten(-2) if case["interleaved"] else torch.cat((z.real, z.imag), -1)
        return torch.cat((pair, x[..., 2 * R:]), -1)

    out = {"q": turn(s["q"], phase), "k": turn(s["k"], phase)}
    if case["kind"] != "prefill":
        out["grads"] = {"dq": turn(s["dq"], phase.conj()), "dk": turn(s["dk"], phase.conj())}
    return _present(out)


def _exact_linear(case, s):
    """Every output as a sum over all tokens, head by head, in blocks of rows."""
    B, T, H, dk, dv = (case[n] for n in ("B", "T", "H", "dk", "dv"))
    if case["kind"] == "steps":
        h, o = s["h0"].double(), []
        for t in range(T):
            h = torch.exp(s["log_decay"].double())[:, None, None] * h + torch.einsum("bhk,bhv->bhkv", s["k"][:, t].double(), s["v"][:, t].double())
            o.append(torch.einsum("bhkv,bhk->bhv", h, s["q"][:, t].double()) * s["scale"])
        return {"o": torch.stack(o, 1), "state": h}
    train = case["kind"] in ("train", "autograd")
    new = lambda *dims: torch.zeros(*dims, dtype=torch.float64, device="cuda")  # noqa: E731
    o, hT = new(B, T, H, dv), new(B, H, dk, dv)
    g = {"dq": new(B, T, H, dk), "dk": new(B, T, H, dk), "dv": new(B, T, H, dv), "dh0": new(B, H, dk, dv)}
    t = torch.arange(T, device="cuda", dtype=torch.float64)
    block = max(1, min(T, (1 << 26) // T))
    for h in range(H):
        a = s["log_decay"][h].double()
        power = torch.exp(a * t)                                                    # e^(a n), n tokens later
        for b in range(B):
            q, k, v = (s[n][b, :, h].detach().double() for n in ("q", "k", "v"))
            h0 = s["h0"][b, h].detach().double() if s["h0"] is not None else new(dk, dv)
            rise, fall = (power * torch.exp(a))[:, None], power.flip(0)[:, None]
            hT[b, h] = k.mT @ (fall * v) + torch.exp(a * T) * h0
            if train:
                do = s["do"][b, :, h].double() * s["scale"]
                dhT = s["dhT"][b, h].double() if s["dhT"] is not None else new(dk, dv)
                g["dh0"][b, h] = q.mT @ (rise * do) + torch.exp(a * T) * dhT
                g["dk"][b, :, h], g["dv"][b, :, h] = fall * (v @ dhT.mT), fall * (k @ dhT)
            for i in range(0, T, block):
                rows = slice(i, min(T, i + block))
                n = t[rows, None] - t[None, :rows.stop]
                W = torch.where(n >= 0, torch.exp(a * n.clamp(min=0)), torch.zeros_like(n))
                A = q[rows] @ k[:rows.stop].mT * W
                o[b, rows, h] = (A @ v[:rows.stop] + rise[rows] * (q[rows] @ h0)) * s["scale"]
                if train:
                    dA = do[rows] @ v[:rows.stop].mT * W
                    g["dq"][b, rows, h] = dA @ k[:rows.stop] + rise[rows] * (do[rows] @ h0.mT)
                    g["dk"][b, :rows.stop, h] += dA.mT @ q[rows]
                    g["dv"][b, :rows.stop, h] += A.mT @ do[rows]
    out = {"o": o, "hT": hT}
    if train:
        out["grads"] = {n: x for n, x in g.items() if n != "dh0" or s["h0"] is not None}
    return out
