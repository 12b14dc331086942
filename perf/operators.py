"""The operators that stand around the delta rule in a recurrent layer, as cases that can be timed and compared: the short
causal convolution before it, the selective state space scan beside it, the layer norm after it.

A case is one pass through one operator: a training step (forward and backward), a prompt (forward that also returns the
state) or decode steps (state updated in place).  `run` computes it in elementary torch operations in fp32, or, where `own`
is true, through the library's public entry points.  `exact` computes the definition in fp64.

    convolution  y_t = f(b + sum_j w_j x_{t-W+1+j}) per channel, f = SiLU or nothing; the W - 1 tokens before the first come
                 from `state`, the last W - 1 are the state after the call
    scan         h_t = exp(dt_t A) h_{t-1} + dt_t u_t B_t ;  y_t = (<C_t, h_t> + D u_t) SiLU(z_t)     per channel, h in R^N;
                 dt = softplus(dt + dt_bias) with `softplus`; groups of D / G channels share B_t and C_t
    norm         y = (x - mean) rstd w + b over the last dimension; rms: mean = 0, rstd = 1 / sqrt(mean(x^2) + eps)
"""
import math

import torch

own = False

EPS = 1e-5
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases --------------------------------------------------------------------------------------------------------
# kind  "train"    forward and backward through the two calls that a training loop of its own makes
#       "autograd" the same pair through torch.autograd
#       "prefill"  forward only, state handed on (norm: forward only)
#       "steps"    T tokens per sequence, state updated in place

def _conv(kind, B, T, D, W=4, dtype="bf16", silu=True, bias=True, state=False):
    return {"op": "conv", "kind": kind, "B": B, "T": T, "D": D, "W": W, "dtype": dtype, "silu": silu, "bias": bias, "state": state}


def _scan(kind, B, T, D, N=16, G=1, dtype="bf16", softplus=True, gate=True, skip=True, state=False):
    return {"op": "scan", "kind": kind, "B": B, "T": T, "D": D, "N": N, "G": G, "dtype": dtype, "softplus": softplus,
            "gate": gate, "skip": skip, "state": state}


def _norm(kind, rows, width, dtype="bf16", rms=False, weight=True, bias=True):
    return {"op": "norm", "kind": kind, "rows": rows, "width": width, "dtype": dtype, "rms": rms, "weight": weight, "bias": bias}


def listed():
    c = [
        # q, k and v of the headline layer (16 heads of 128) in one convolution: training step of 16384 tokens
        ("conv train lm", _conv("train", 8, 2048, 6144)),
        # the same layer's prompt of one user, odd length, going on from a cached state
        ("conv prefill one ragged", _conv("prefill", 1, 777, 6144, bias=False, state=True)),
        # full precision, odd number of channels and of tokens, truncated back-propagation through the state
        ("conv train odd f32", _conv("train", 2, 509, 1001, W=3, dtype="f32", silu=False, state=True)),
        # one token for each of 256 sequences
        ("conv decode 256", _conv("steps", 256, 1, 6144, bias=False)),
        # a selective layer as wide as the headline layer's heads together: training step of 16384 tokens (the largest case)
        ("scan train lm", _scan("train", 8, 2048, 2048)),
        # a small full-precision layer through torch.autograd, ragged length, initial state, two groups
        ("scan autograd ragged f32", _scan("autograd", 2, 1000, 512, G=2, dtype="f32", state=True)),
        # a context of 32768 tokens, one sequence: few channels, many tokens
        ("scan prefill long", _scan("prefill", 1, 32768, 2048)),
        # one user's prompt of odd length
        ("scan prefill one ragged", _scan("prefill", 1, 777, 2048, state=True)),
        # one token for each of 256 sequences
        ("scan decode 256", _scan("steps", 256, 1, 2048, state=True)),
        # read-out of the headline layer normalised per head: 16384 tokens x 16 heads of 128, no mean, no bias
        ("norm train heads", _norm("train", 262144, 128, rms=True, bias=False)),
        # the norm before a layer, 16384 tokens, through torch.autograd
        ("norm autograd lm", _norm("autograd", 16384, 2048)),
        # the same norm while decoding
        ("norm decode 256", _norm("prefill", 256, 2048)),
    ]
    return [dict(d, name=n) for n, d in c]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _even(rng, n, m):
    """n as drawn, or near it a multiple of m."""
    return max(m, n // m * m) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["conv", "scan", "scan", "norm"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        width = _even(rng, _log_int(rng, 1, 16384), 64)
        rows = _log_int(rng, 1, max(1, min(262144, (1 << 25) // width)))
        return _norm(rng.choice(["train", "train", "autograd", "prefill"]), rows, width, dtype, rng.random() < 0.4,
                     rng.random() < 0.9, rng.random() < 0.6)
    flag = lambda p: rng.random() < p  # noqa: E731
    steps = flag(0.25)
    if op == "conv":
        D, W = _even(rng, _log_int(rng, 1, 8192), 64), rng.choice([2, 3, 4, 4])
        if steps:
            return _conv("steps", _log_int(rng, 1, 512), rng.randint(1, 8), D, W, dtype, flag(0.8), flag(0.5))
        T = _even(rng, _log_int(rng, 1, 32768), 64)
        B = min(_log_int(rng, 1, 32), max(1, (1 << 26) // (T * D)))
        return _conv(rng.choice(["train", "autograd", "prefill"]), B, T, D, W, dtype, flag(0.8), flag(0.5), flag(0.4))
    G = rng.choice([1, 1, 1, 2, 4])
    D = G * _even(rng, _log_int(rng, 1, 4096 // G), 32)
    N = rng.choice([16, 16, 16, 8, 64, rng.randint(1, 64)])
    if steps:
        return _scan("steps", _log_int(rng, 1, max(1, min(512, (1 << 25) // (D * N)))), rng.randint(1, 8), D, N, G, dtype,
                     flag(0.8), flag(0.6), flag(0.8), True)
    kind = rng.choice(["train", "autograd", "prefill"])
    T = _even(rng, _log_int(rng, 1, 16384 if kind == "prefill" else 4096), 64)
    D = max(G, min(D, (1 << 28) // (T * N)) // G * G)
    B = min(_log_int(rng, 1, 16), max(1, (1 << 28) // (T * D * N)))
    return _scan(kind, B, T, D, N, G, dtype, flag(0.8), flag(0.6), flag(0.8), flag(0.4))


# ---- inputs -----------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = _DT[case["dtype"]]

    def normal(*dims, std=1.0, to=dt):
        return (torch.randn(*dims, device="cuda", generator=gen) * std).to(to)

    def uniform(*dims):
        return torch.rand(*dims, device="cuda", generator=gen)

    s = {"case": case}
    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        # activations of a residual stream: rows of different scale, a few channels that stand out
        x = normal(rows, width, to=torch.float32) * (normal(rows, 1, std=0.5, to=torch.float32).exp())
        s["x"] = (x * (1.0 + 4.0 * (uniform(width) < 0.01)) + 0.3).to(dt)
        s["weight"] = (1.0 + normal(width, std=0.2, to=torch.float32)).to(dt) if case["weight"] else None
        s["bias"] = normal(width, std=0.2) if case["bias"] else None
        s["dy"] = normal(rows, width) if case["kind"] != "prefill" else None
        wanted = ("x", "weight", "bias")
    elif case["op"] == "conv":
        B, T, D, W = (case[n] for n in ("B", "T", "D", "W"))
        s["x"], s["w"] = normal(B, T, D), normal(D, W, std=0.5)
        s["bias"] = normal(D, std=0.2) if case["bias"] else None
        s["state"] = normal(B, W - 1, D) if case["state"] or case["kind"] == "steps" else None
        if case["kind"] in ("train", "autograd"):
            s["dy"], s["dstate"] = normal(B, T, D), normal(B, W - 1, D) if case["state"] else None
        wanted = ("x", "w", "bias", "state")
    else:
        B, T, D, N, G = (case[n] for n in ("B", "T", "D", "N", "G"))
        s["u"], s["Bm"], s["Cm"] = normal(B, T, D), normal(B, T, G, N), normal(B, T, G, N)
        # steps of a trained layer: 0.001 to 0.1 per channel, varied by the token
        step = torch.exp(uniform(D) * math.log(100.0) + math.log(1e-3))
        s["dt_bias"] = torch.log(torch.expm1(step)) if case["softplus"] else None
        wave = normal(B, T, D, std=0.7, to=torch.float32)
        s["dt"] = (wave if case["softplus"] else step * wave.exp()).to(dt)
        s["A"] = -(torch.arange(1, N + 1, device="cuda").float() * normal(D, N, std=0.2, to=torch.float32).exp())
        s["D"] = 1.0 + normal(D, std=0.2, to=torch.float32) if case["skip"] else None
        s["z"] = normal(B, T, D) if case["gate"] else None
        s["h0"] = normal(B, D, N, std=0.5, to=torch.float32) if case["state"] else None
        if case["kind"] in ("train", "autograd"):
            s["dy"] = normal(B, T, D)
            s["dhT"] = normal(B, D, N, std=0.5, to=torch.float32) if case["state"] else None
        wanted = ("u", "dt", "A", "Bm", "Cm", "D", "z", "dt_bias", "h0")
    if case["kind"] == "autograd":
        s["wanted"] = {n: s[n].requires_grad_() for n in wanted if s[n] is not None}
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _own(s)
    with torch.no_grad():
        return {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm}[s["case"]["op"]](s)


def _own(s):
    from paper_2606_08804_b200 import autograd as qa
    from paper_2606_08804_b200 import binding as qd
    case = s["case"]
    kind = case["kind"]
    if case["op"] == "norm":
        x, w, b = s["x"], s["weight"], s["bias"]
        if kind == "autograd":
            y = qa.layer_norm(x, w, b, EPS, rms=case["rms"])
            return {"y": y.detach(), **_grads(s, (y,), (s["dy"],))}
        y, stats = qd.norm_fwd(x, w, b, EPS, rms=case["rms"])
        if kind == "prefill":
            return {"y": y}
        return {"y": y, **_kept(qd.norm_bwd(x, w, s["dy"], stats, rms=case["rms"], want_dbias=case["bias"]))}
    if case["op"] == "conv":
        x, w, b, state, silu = s["x"], s["w"], s["bias"], s["state"], case["silu"]
        if kind == "steps":
            return {"y": qd.conv_steps(x, w, b, state, silu=silu), "state": state}
        if kind == "autograd":
            y, last = qa.short_conv(x, w, b, state, silu=silu)
            outs, ups = ((y, last), (s["dy"], s["dstate"])) if s["dstate"] is not None else ((y,), (s["dy"],))
            return {"y": y.detach(), "last": last.detach(), **_grads(s, outs, ups)}
        y, last = qd.conv_fwd(x, w, b, state, silu=silu)
        if kind == "prefill":
            return {"y": y, "last": last}
        return {"y": y, "last": last, **_kept(qd.conv_bwd(x, w, b, state, s["dy"], s["dstate"], silu=silu))}
    args = [s[n] for n in ("u", "dt", "A", "Bm", "Cm", "D", "z", "dt_bias")]
    if kind == "steps":
        return {"y": qd.scan_steps(*args, s["h0"], softplus=case["softplus"]), "state": s["h0"]}
    if kind == "autograd":
        y, hT = qa.selective_scan(*args, s["h0"], softplus=case["softplus"])
        outs, ups = ((y, hT), (s["dy"], s["dhT"])) if s["dhT"] is not None else ((y,), (s["dy"],))
        return {"y": y.detach(), "hT": hT.detach(), **_grads(s, outs, ups)}
    y, hT, ws = qd.scan_fwd(*args, s["h0"], softplus=case["softplus"], save_for_bwd=kind == "train")
    if kind == "prefill":
        return {"y": y, "hT": hT}
    g = qd.scan_bwd(*args, s["h0"], s["dy"], s["dhT"], workspace=ws, reuse_fwd=True, softplus=case["softplus"])
    return {"y": y, "hT": hT, **_kept(g)}


def _grads(s, outs, ups):
    g = torch.autograd.grad(outs, list(s["wanted"].values()), ups)
    return {"grads": {"d" + n: x for n, x in zip(s["wanted"], g)}}


def _kept(g):
    return {"grads": {n: x for n, x in g.items() if x is not None}}


def _named(s, g):
    """Gradients under the names and in the types of the entry points: those of parameters are fp32 in a training loop of its
    own, and of the parameter's type through torch.autograd."""
    auto = s["case"]["kind"] == "autograd"
    tokens = ("dx", "du", "ddt", "dBm", "dCm", "dz", "dstate")
    out = {}
    for n, x in g.items():
        like = s[n[1:]]
        if like is None:
            continue
        out[n] = x.reshape(like.shape).to(like.dtype if auto or n in tokens else torch.float32)
    return {"grads": out}


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _plain_norm(s):
    case, x, dt = s["case"], s["x"].float(), s["x"].dtype
    w = s["weight"].float() if s["weight"] is not None else None
    if not case["rms"]:
        x = x - x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    xh = x * rstd
    y = xh if w is None else xh * w
    y = y if s["bias"] is None else y + s["bias"].float()
    if s["dy"] is None:
        return {"y": y.to(dt)}
    dy = s["dy"].float()
    g = dy if w is None else dy * w
    dx = g - xh * (g * xh).mean(-1, keepdim=True)
    if not case["rms"]:
        dx = dx - g.mean(-1, keepdim=True)
    return {"y": y.to(dt), **_named(s, {"dx": dx * rstd, "dweight": (dy * xh).sum(0), "dbias": dy.sum(0)})}


def _plain_conv(s):
    case, x, dt = s["case"], s["x"].float(), s["x"].dtype
    B, T, D, W = (case[n] for n in ("B", "T", "D", "W"))
    w = s["w"].float()
    before = s["state"].float() if s["state"] is not None else x.new_zeros(B, W - 1, D)
    xp = torch.cat([before, x], 1)
    win = xp.unfold(1, W, 1)                                             # [B, T, D, W]
    pre = (win * w).sum(-1)
    pre = pre if s["bias"] is None else pre + s["bias"].float()
    sig = _sigmoid(pre) if case["silu"] else None
    y = pre * sig if case["silu"] else pre
    last = xp[:, T:].to(dt)
    if case["kind"] == "steps":
        s["state"].copy_(last)
        return {"y": y.to(dt), "state": s["state"]}
    out = {"y": y.to(dt), "last": last}
    if case["kind"] == "prefill":
        return out
    dpre = s["dy"].float()
    if case["silu"]:
        dpre = dpre * (sig * (1.0 + pre * (1.0 - sig)))
    rim = dpre.new_zeros(B, W - 1, D)
    dxp = (torch.cat([rim, dpre, rim], 1).unfold(1, W, 1) * w.flip(-1)).sum(-1)
    if s["dstate"] is not None:
        dxp[:, T:] += s["dstate"].float()
    return {**out, **_named(s, {"dx": dxp[:, W - 1:], "dw": (win * dpre[..., None]).sum((0, 1)), "dbias": dpre.sum((0, 1)),
                                "dstate": dxp[:, :W - 1]})}


def _prefix(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1 from h = 0: a parallel prefix, the reach doubled each time."""
    reach = 1
    while reach < b.shape[1]:
        b = torch.cat([b[:, :reach], b[:, reach:] + a[:, reach:] * b[:, :-reach]], 1)
        a = torch.cat([a[:, :reach], a[:, reach:] * a[:, :-reach]], 1)
        reach *= 2
    return b


def _plain_scan(s):
    case, io = s["case"], s["u"].dtype
    B, T, D, N, G = (case[n] for n in ("B", "T", "D", "N", "G"))
    K = D // G
    split = lambda x: None if x is None else x.float().reshape(*x.shape[:-1], G, K)  # noqa: E731
    u, raw, z, skip = split(s["u"]), split(s["dt"]), split(s["z"]), split(s["D"])
    A = s["A"].reshape(G, K, N)
    Bm, Cm = s["Bm"].float()[:, :, :, None], s["Cm"].float()[:, :, :, None]          # [B, T, G, 1, N]
    h0 = s["h0"].reshape(B, G, K, N) if s["h0"] is not None else A.new_zeros(B, G, K, N)
    raw = raw if s["dt_bias"] is None else raw + split(s["dt_bias"])
    dt = torch.clamp(raw, min=0) + torch.log1p(torch.exp(-raw.abs())) if case["softplus"] else raw
    a = torch.exp(dt[..., None] * A)                                               # [B, T, G, K, N]
    b = (dt * u)[..., None] * Bm
    b[:, 0] += a[:, 0] * h0
    h = _prefix(a, b)
    del b
    yr = (h * Cm).sum(-1)
    yr = yr if skip is None else yr + skip * u
    sig = None if z is None else _sigmoid(z)
    y = (yr if z is None else yr * (z * sig)).reshape(B, T, D).to(io)
    hT = h[:, -1].reshape(B, D, N)
    if case["kind"] == "steps":
        s["h0"].copy_(hT)
        return {"y": y, "state": s["h0"]}
    out = {"y": y, "hT": hT.clone()}
    if case["kind"] == "prefill":
        return out
    g = {}
    dy = split(s["dy"])
    if z is not None:
        g["dz"] = dy * yr * sig * (1.0 + z * (1.0 - sig))
        dy = dy * z * sig
    g["dCm"] = (h * dy[..., None]).sum(3)
    c = dy[..., None] * Cm
    if s["dhT"] is not None:
        c[:, -1] += s["dhT"].reshape(B, G, K, N)
    after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    gh = _prefix(after.flip(1), c.flip(1)).flip(1)                                   # dL/dh_t
    del c, after
    g["dBm"] = (gh * (dt * u)[..., None]).sum(3)
    gb = (gh * Bm).sum(-1)
    g["du"] = gb * dt if skip is None else gb * dt + skip * dy
    g["dh0"] = a[:, 0] * gh[:, 0]
    gh = gh * a * torch.cat([h0[:, None], h[:, :-1]], 1)                             # dL/d(dt A)
    del a, h
    ddt = gb * u + (gh * A).sum(-1)
    if case["softplus"]:
        ddt = ddt * _sigmoid(raw)
    g["ddt"], g["ddt_bias"] = ddt, ddt.sum((0, 1))
    g["dA"], g["dD"] = (gh * dt[..., None]).sum((0, 1)), (dy * u).sum((0, 1))
    return {**out, **_named(s, g)}


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------
def work(case):
    io = 2 if case["dtype"] == "bf16" else 4
    train = case["kind"] in ("train", "autograd")
    if case["op"] == "norm":
        n, p = case["rows"] * case["width"], case["width"] * (int(case["weight"]) + int(case["bias"]))
        # read x (and dy), write y (and dx): the backward's x is the forward's
        return {"bytes": float(io * (n * (4 if train else 2) + p) + (4 * p if train else 0)), "flops": n * (20.0 if train else 8.0)}
    if case["op"] == "conv":
        B, T, D, W = (case[n] for n in ("B", "T", "D", "W"))
        n, st = B * T * D, B * (W - 1) * D
        states = (1 if case["state"] or case["kind"] == "steps" else 0) + 1
        nbytes = io * (2 * n + states * st + D * (W + 1))
        flops = n * (2.0 * W + 6.0)
        if train:
            nbytes += io * (2 * n + (2 * st if case["state"] else 0)) + 4 * D * (W + 1)
            flops += n * (4.0 * W + 10.0)
        return {"bytes": float(nbytes), "flops": flops}
    B, T, D, N, G = (case[n] for n in ("B", "T", "D", "N", "G"))
    rows, bc, st = B * T * D, B * T * G * N, B * D * N
    tokens, states = 3 + int(case["gate"]), 1 + int(case["state"])
    nbytes = io * (tokens * rows + 2 * bc) + 4 * (states * st + D * (N + 2))
    flops = 7.0 * rows * N                      # the exponential counted as one
    if train:
        nbytes += io * ((3 + int(case["gate"])) * rows + 2 * bc) + 4 * (D * (N + 2) + (2 * st if case["state"] else 0))
        flops += 20.0 * rows * N
    return {"bytes": float(nbytes), "flops": flops}


# ---- the definition in fp64 -------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    train = case["kind"] in ("train", "autograd")
    names = {"norm": ("x", "weight", "bias"), "conv": ("x", "w", "bias", "state"),
             "scan": ("u", "dt", "A", "Bm", "Cm", "D", "z", "dt_bias", "h0")}[case["op"]]
    d = {n: s[n].detach().double().requires_grad_(train) for n in names if s[n] is not None}
    with torch.set_grad_enabled(train):
        outs = {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm}[case["op"]](case, d)
    if not train:
        return outs
    ups = {"y": s["dy"], "last": s.get("dstate"), "hT": s.get("dhT")}
    pairs = [(o, ups[n].double()) for n, o in outs.items() if ups.get(n) is not None]
    g = torch.autograd.grad([o for o, _ in pairs], list(d.values()), [u for _, u in pairs])
    return {**{n: o.detach() for n, o in outs.items()}, "grads": {"d" + n: x for n, x in zip(d, g)}}


def _exact_norm(case, d):
    x = d["x"]
    if not case["rms"]:
        return {"y": torch.nn.functional.layer_norm(x, x.shape[-1:], d.get("weight"), d.get("bias"), EPS)}
    y = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    return {"y": y * d.get("weight", 1.0) + d.get("bias", 0.0)}


def _exact_conv(case, d):
    T, W = case["T"], case["W"]
    xp = torch.nn.functional.pad(d["x"], (0, 0, W - 1, 0)) if "state" not in d else torch.cat([d["state"], d["x"]], 1)
    pre = sum(d["w"][:, j] * xp[:, j:j + T] for j in range(W)) + d.get("bias", 0.0)
    y = torch.nn.functional.silu(pre) if case["silu"] else pre
    return {"y": y, ("state" if case["kind"] == "steps" else "last"): xp[:, T:]}


def _exact_scan(case, d):
    B, T, D, N, G = (case[n] for n in ("B", "T", "D", "N", "G"))
    dt = d["dt"] + d.get("dt_bias", 0.0)
    dt = torch.logaddexp(dt, torch.zeros_like(dt)) if case["softplus"] else dt
    x = dt * d["u"]
    h = d.get("h0", torch.zeros(B, D, N, dtype=torch.float64, device="cuda"))
    ys = []
    for dt_t, x_t, B_t, C_t in zip(dt.unbind(1), x.unbind(1), d["Bm"].unbind(1), d["Cm"].unbind(1)):
        B_t, C_t = (m.repeat_interleave(D // G, 1) if G > 1 else m for m in (B_t, C_t))
        h = torch.exp(dt_t[..., None] * d["A"]) * h + x_t[..., None] * B_t
        ys.append((h * C_t).sum(-1))
    y = torch.stack(ys, 1) + d.get("D", 0.0) * d["u"]
    if "z" in d:
        y = y * torch.nn.functional.silu(d["z"])
    return {"y": y, ("state" if case["kind"] == "steps" else "hT"): h}
