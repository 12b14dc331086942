"""The operators around the delta rule, written out in 64 bits on the CPU, token by token: what the kernels are compared with.
Gradients are those of torch's autograd through these forms (test_layer_forms.py holds them against differences)."""
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}          # half a step of the type, relative to the value
ULP = 2.0 ** -24


def f64(t):
    return None if t is None else t.detach().double().cpu().requires_grad_()


def conv(x, w, bias=None, state=None, silu=False):
    B, T, D = x.shape
    W = w.shape[1]
    rows = list((state if state is not None else x.new_zeros(B, W - 1, D)).unbind(1)) + list(x.unbind(1))
    ys = []
    for t in range(T):
        s = sum(w[:, j] * rows[t + j] for j in range(W))
        s = s if bias is None else s + bias
        ys.append(s / (1 + torch.exp(-s)) if silu else s)
    return torch.stack(ys, 1), torch.stack(rows[T:], 1)


def scan(u, dt, A, Bm, Cm, D=None, z=None, dt_bias=None, h0=None, softplus=False):
    B, T, C = u.shape
    N, G = A.shape[1], Bm.shape[2]
    group = torch.arange(C) // (C // G)
    dt = dt if dt_bias is None else dt + dt_bias
    dt = torch.log1p(torch.exp(-dt.abs())) + torch.clamp(dt, min=0) if softplus else dt
    h = h0 if h0 is not None else u.new_zeros(B, C, N)
    ys = []
    for t in range(T):
        h = torch.exp(dt[:, t, :, None] * A) * h + (dt[:, t] * u[:, t])[..., None] * Bm[:, t, group]
        y = (Cm[:, t, group] * h).sum(-1)
        y = y if D is None else y + D * u[:, t]
        ys.append(y if z is None else y * z[:, t] / (1 + torch.exp(-z[:, t])))
    return torch.stack(ys, 1), h


def norm(x, weight=None, bias=None, eps=1e-5, rms=False):
    x = x if rms else x - x.mean(-1, keepdim=True)
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    y = y if weight is None else y * weight
    return y if bias is None else y + bias


def grads(outs, ups, inputs):
    """d(sum <out, up>) / d input, None for absent inputs."""
    pairs = [(o, u) for o, u in zip(outs, ups) if u is not None]
    have = [i for i in inputs if i is not None]
    g = iter(torch.autograd.grad([o for o, _ in pairs], have, [u for _, u in pairs], allow_unused=True))
    return [None if i is None else (lambda v: v if v is not None else torch.zeros_like(i))(next(g)) for i in inputs]


def close(name, got, ref, slack):
    """Every element within half a step of its type and `slack` (what 32-bit arithmetic on the way may cost)."""
    ref = ref.detach()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    off = (got.detach().double().cpu() - ref).abs()
    most = HALF[got.dtype] * ref.abs() + slack
    bad = ~(off <= most)
    assert not bad.any(), "%s: %d of %d off, worst %.3g over the %.3g allowed, at %s" % (
        name, int(bad.sum()), bad.numel(), float((off - most).max()), float(most.flatten()[(off - most).argmax()]),
        bad.nonzero()[0].tolist())
