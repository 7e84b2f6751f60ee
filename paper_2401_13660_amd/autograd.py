"""The selective scan, the causal convolution and the embedding as differentiable torch
operations, for training.

The scan's forward runs ``mb_scan_fwd_ckpt`` (y in u's dtype, h_last, and the state
every 16 bytes); the backward runs ``mb_scan_bwd`` from those checkpoints.  All
arithmetic happens in the HIP library: this module only holds tensors between
the two calls.  dB and dC come back in fp32 and are handed to autograd in B's
and C's dtype.  Supported as the library's backward is: dstate 16 and L a
multiple of 16 (the library raises otherwise).  The convolution's backward is
``mb_conv1d_bwd``, which computes the forward again from x; the embedding's is
``mb_embedding_bwd``.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import _binding as _b


class _SelectiveScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, delta, A, B, C, D, dt_bias, z, h0, delta_softplus):
        y, h_last, ck = _b.scan_fwd(u, delta, A, B, C, D=D, dt_bias=dt_bias, z=z, h0=h0,
                                    delta_softplus=delta_softplus, out_dtype=u.dtype, return_last_state=True,
                                    return_ckpt=True)
        ctx.delta_softplus = delta_softplus
        ctx.save_for_backward(u, delta, A, B, C, D, dt_bias, z, h0, ck)
        return y, h_last

    @staticmethod
    def backward(ctx, dy, dh_last):
        u, delta, A, B, C, D, dt_bias, z, h0, ck = ctx.saved_tensors
        g = _b.scan_bwd(u, delta, A, B, C, dy.contiguous(), D=D, dt_bias=dt_bias, z=z, h0=h0,
                        dh_last=None if dh_last is None else dh_last.contiguous(),
                        delta_softplus=ctx.delta_softplus, ck=ck)
        dB = g["dB"] if B.dtype == torch.float32 else g["dB"].to(B.dtype)
        dC = g["dC"] if C.dtype == torch.float32 else g["dC"].to(C.dtype)
        return (g["du"], g["ddelta"], g["dA"], dB, dC, g["dD"], g["ddt_bias"], g["dz"],
                g["dh0"] if h0 is not None else None, None)


def selective_scan(u, delta, A, B, C, D=None, dt_bias=None, z=None, h0=None, *, delta_softplus=True):
    """Differentiable scan: returns (y, h_last), y in u's dtype.  Shapes and dtypes
    as for ``scan_fwd``; gradients flow to every tensor argument."""
    return _SelectiveScan.apply(u, delta, A, B, C, D, dt_bias, z, h0, delta_softplus)


class _CausalConv1d(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, state, apply_silu):
        y, state_out = _b.conv1d(x, w, bias, state, apply_silu=apply_silu, return_state=True)
        ctx.apply_silu, ctx.ytype = apply_silu, y.dtype
        ctx.set_materialize_grads(False)                # an output that the loss does not use has no gradient
        ctx.save_for_backward(x, w, bias, state)
        return y, state_out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dstate_out):
        x, w, bias, state = ctx.saved_tensors
        dy = torch.zeros_like(x, dtype=ctx.ytype) if dy is None else dy
        g = _b.conv1d_bwd(x, w, dy.contiguous(), bias, state,
                          None if dstate_out is None else dstate_out.contiguous(), apply_silu=ctx.apply_silu)
        return g["dx"], g["dw"], g["dbias"], g["dstate"] if state is not None else None, None


def causal_conv1d(x, w, bias=None, state=None, *, apply_silu=True):
    """Differentiable convolution (+ Swish): returns (y, state_out), y in x's dtype.  Shapes and dtypes as for
    ``conv1d``; gradients flow to every tensor argument, once: a second derivative raises."""
    return _CausalConv1d.apply(x, w, bias, state, apply_silu)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, weight, scale, out_dtype):
        ctx.scale, ctx.vocab, ctx.wtype = scale, weight.shape[0], weight.dtype
        ctx.save_for_backward(tokens)
        return _b.embedding_fwd(tokens, weight, scale=scale, out_dtype=out_dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        tokens, = ctx.saved_tensors
        dw = _b.embedding_bwd(tokens, dy.contiguous(), ctx.vocab, scale=ctx.scale, out_dtype=ctx.wtype)
        return None, dw, None, None


def embedding(tokens, weight, *, scale=1.0, out_dtype=None):
    """Differentiable scale * weight[tokens].  Shapes and types as for ``embedding_fwd``; the gradient flows to
    ``weight``, in its type."""
    return _Embedding.apply(tokens, weight, scale, out_dtype)
