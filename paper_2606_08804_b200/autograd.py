"""`torch.autograd` front-end of the chunkwise kernels: marshalling only.

    o, hT = qdelta_chunk(q, k, v, beta, alpha, lam, h0, logits=False, norm_qk=False)

q, k [B,T,H,dk], v [B,T,H,dv], beta/alpha/lam [B,T,H] (alpha, lam, h0 may be None), all CUDA tensors; returns the
outputs o [B,T,H,dv] and the final state hT [B,H,dk,dv] (fp32), both differentiable.  The forward runs
`qdelta_chunk_fwd` saving what the backward needs in a workspace that the autograd node keeps; the backward runs
`qdelta_chunk_bwd` on that workspace; the node itself is native (host/host.cpp).  Every number is computed by the library's CUDA kernels.

The operators around it likewise, gradients in the type of what they belong to:

    y, state = short_conv(x, w, bias, state, silu=False)                                    (binding.conv_fwd)
    y, hT = selective_scan(u, dt, A, Bm, Cm, D, z, dt_bias, h0, softplus=False)             (binding.scan_fwd)
    y = layer_norm(x, weight, bias, eps, rms=False)                                         (binding.norm_fwd)

    o, hT = linear_attention(q, k, v, log_decay, h0, scale=1.0)                             (binding.linear_fwd)
    y = gated_norm(x, gate, weight, bias, eps, rms=False, silu=True)                        (binding.gated_norm_fwd)
    y, total = add_norm(x, residual, scale, weight, bias, eps, rms=False)                   (binding.add_norm_fwd)
    q, k = rotary(q, k, turns, positions, start=0, interleaved=False, scale=1.0)            (binding.rotary)

Inputs of all of them may have any strides (they are made dense first).  Types are not converted: w, bias, state and weight have the type
of x (bf16 or fp32; pass w.to(x.dtype) where parameters are kept in fp32), A, D, dt_bias and h0 are fp32.

What is saved for the backward may not be written before it, by torch or by the single-token calls (binding.conv_steps, scan_steps,
recurrent_steps, linear_steps), which update a state in place: the backward then raises.  The initial states h0 of the delta rule and the
scan are not saved; linear_attention saves its own, as its backward walks the sequence again from there.
"""
from . import binding as qd


def qdelta_chunk(q, k, v, beta, alpha=None, lam=None, h0=None, logits=False, norm_qk=False):
    """Differentiable chunkwise Q-Delta: returns (o, hT)."""
    flags = (qd.QD_COEF_LOGITS if logits else 0) | (qd.QD_NORM_QK if norm_qk else 0)
    return qd._host().chunk_autograd(q, k, v, beta, alpha, lam, h0, flags)


def short_conv(x, w, bias=None, state=None, silu=False):
    """Differentiable short causal convolution: returns (y, state after the last token)."""
    return qd._host().conv_autograd(x, w, bias, state, qd.QD_SILU if silu else 0)


def selective_scan(u, dt, A, Bm, Cm, D=None, z=None, dt_bias=None, h0=None, softplus=False):
    """Differentiable selective state space scan: returns (y, hT)."""
    return qd._host().scan_autograd(u, dt, A, Bm, Cm, D, z, dt_bias, h0, qd.QD_SOFTPLUS if softplus else 0)


def layer_norm(x, weight=None, bias=None, eps=1e-5, rms=False):
    """Differentiable layer norm over the last dimension (rms: without the mean): returns y."""
    return qd._host().norm_autograd(x, weight, bias, eps, qd.QD_RMS if rms else 0)


def linear_attention(q, k, v, log_decay, h0=None, scale=1.0):
    """Differentiable linear attention with a decay for each head (a constant: log_decay has no gradient): returns (o, hT)."""
    return qd._host().linear_autograd(q, k, v, log_decay, h0, scale)


def gated_norm(x, gate, weight=None, bias=None, eps=1e-5, rms=False, silu=True):
    """Differentiable layer norm over the last dimension times SiLU(gate) (silu=False: sigmoid(gate)): returns y."""
    return qd._host().gated_norm_autograd(x, gate, weight, bias, eps, (qd.QD_RMS if rms else 0) | (qd.QD_SILU if silu else 0))


def add_norm(x, residual, scale=None, weight=None, bias=None, eps=1e-5, rms=False):
    """Differentiable residual + scale x and its layer norm: returns (y, total)."""
    return qd._host().add_norm_autograd(x, residual, scale, weight, bias, eps, qd.QD_RMS if rms else 0)


def rotary(q, k, turns, positions=None, start=0, interleaved=False, scale=1.0):
    """Differentiable rotary positions of q and k (or None): returns (q', k')."""
    return qd._host().rotary_autograd(q, k, turns, positions, start, scale, qd.QD_INTERLEAVED if interleaved else 0)
