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

Inputs of all of them may have any strides (they are made dense first).  Types are not converted: w, bias, state and weight have the type
of x (bf16 or fp32; pass w.to(x.dtype) where parameters are kept in fp32), A, D, dt_bias and h0 are fp32.

What is saved for the backward may not be written before it, by torch or by the single-token calls (binding.conv_steps, scan_steps,
recurrent_steps), which update a state in place: the backward then raises.  The initial states h0 are not saved.
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
