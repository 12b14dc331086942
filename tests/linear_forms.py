"""The operators of a linear attention layer, written out in 64 bits on the CPU: what the kernels are compared with.  Gradients are those of
torch's autograd through these forms (test_linear_forms.py holds them against the recurrence and against differences)."""
import math

import torch

import layer_forms as lf


def decays(g, T):
    """W[h, t, i] = e^(g (t - i)) for i <= t, else 0; g may be minus infinity."""
    n = torch.arange(T)[:, None] - torch.arange(T)[None, :]
    e = torch.where(n == 0, torch.zeros((), dtype=torch.float64), g[:, None, None] * n.clamp(min=0))
    return torch.where(n >= 0, torch.exp(e), torch.zeros((), dtype=torch.float64))


def linear(q, k, v, g, h0=None, scale=1.0):
    """Every token's output as a sum over all tokens before it."""
    B, T, H, dk = q.shape
    W = decays(g, T)
    up = torch.exp(g[:, None] * (torch.arange(T) + 1))                                  # [H, T]
    A = torch.einsum("bthd,bihd->bhti", q, k) * W
    o = torch.einsum("bhti,bihv->bthv", A, v)
    h = torch.einsum("hi,bihd,bihv->bhdv", W[:, T - 1], k, v)
    if h0 is not None:
        o = o + torch.einsum("bthd,ht,bhdv->bthv", q, up, h0)
        h = h + torch.exp(g * T)[:, None, None] * h0
    return o * scale, h


def linear_recurrence(q, k, v, g, h0=None, scale=1.0):
    B, T, H, dk = q.shape
    h = h0 if h0 is not None else q.new_zeros(B, H, dk, v.shape[-1])
    os = []
    for t in range(T):
        h = torch.exp(g)[:, None, None] * h + k[:, t, :, :, None] * v[:, t, :, None, :]
        os.append((h * q[:, t, :, :, None]).sum(-2) * scale)
    return torch.stack(os, 1), h


def gate(z, silu):
    s = 1 / (1 + torch.exp(-z))
    return z * s if silu else s


def gated_norm(x, z, weight=None, bias=None, eps=1e-5, rms=False, silu=True):
    return lf.norm(x, weight, bias, eps, rms) * gate(z, silu)


def add_norm(x, residual, scale=None, weight=None, bias=None, eps=1e-5, rms=False):
    total = residual + (x if scale is None else scale * x)
    return lf.norm(total, weight, bias, eps, rms), total


def angles(turns, positions):
    """Radians of every (position, pair), from the exact fraction of a turn (both lists of Python integers)."""
    return torch.tensor([[((p * t) % (1 << 64)) / 2.0 ** 64 * 2 * math.pi for t in turns] for p in positions], dtype=torch.float64)


def rotary(x, angle, interleaved=False, scale=1.0):
    """x [B, T, H, d], angle [B, T, pairs]."""
    R = angle.shape[-1]
    c, s = torch.cos(angle)[:, :, None] * scale, torch.sin(angle)[:, :, None] * scale
    if interleaved:
        a, b = x[..., 0:2 * R:2], x[..., 1:2 * R:2]
        y = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
    else:
        a, b = x[..., :R], x[..., R:2 * R]
        y = torch.cat((a * c - b * s, a * s + b * c), -1)
    return torch.cat((y, x[..., 2 * R:]), -1)
