"""The selective scan, the causal convolution, the embedding, the norm and the projection in 8 bits as
differentiable torch operations, for training.

The scan's forward runs ``mb_scan_fwd_ckpt`` (y in u's dtype, h_last, and the state
every 16 bytes); the backward runs ``mb_scan_bwd`` from those checkpoints.  All
arithmetic happens in the HIP library: this module only holds tensors between
the two calls.  dB and dC come back in fp32 and are handed to autograd in B's
and C's dtype.  Supported as the library's backward is: dstate 16 and L a
multiple of 16 (the library raises otherwise).  The convolution's backward is
``mb_conv1d_bwd``, which computes the forward again from x; the embedding's is
``mb_embedding_bwd``, the norm's ``mb_rms_norm_bwd``.  The projection's products are all
``mb_matmul_fp8``, of what ``mb_quantize_fp8`` makes of the factors as each of them needs it.
"""
from __future__ import annotations

import math

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


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps, out_dtype):
        res = _b.rms_norm_fwd(x, weight, residual, eps=eps, out_dtype=out_dtype, return_rstd=True)
        y, rstd = res[0], res[-1]
        h = x if residual is None else res[1]
        ctx.xtype, ctx.added = x.dtype, residual is not None
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(h, rstd, weight)
        return y if residual is None else (y, h)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh=None):
        h, rstd, weight = ctx.saved_tensors
        if dy is None:
            if dh is None:
                return None, None, None, None, None
            return dh.to(ctx.xtype), None if weight is None else torch.zeros_like(weight), dh, None, None
        if ctx.added and dh is None:
            dh = torch.zeros_like(h)
        g = _b.rms_norm_bwd(dy.contiguous(), h, rstd, weight, None if dh is None else dh.contiguous(), dx_dtype=ctx.xtype)
        return g["dx"], g["dweight"], g.get("dresidual"), None, None


def rms_norm(x, weight=None, residual=None, *, eps=1e-5, out_dtype=None):
    """Differentiable ``rms_norm_fwd``: y, or (y, h) with a residual.  Shapes and types as there; gradients flow to every
    tensor argument, once: a second derivative raises."""
    return _RmsNorm.apply(x, weight, residual, eps, out_dtype)


def _rows(t):
    """t's leading dimensions as one, whatever of them is 0, as a dense matrix: a copy where t is strided."""
    return t.contiguous().view(math.prod(t.shape[:-1]), t.shape[-1])


class _LinearFp8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        ctx.save_for_backward(x, weight)
        y = _b.matmul_fp8(*_b.quantize_fp8(_rows(x)), *_b.quantize_fp8(weight.contiguous(), tile=True), out_dtype=x.dtype)
        return y.view(x.shape[:-1] + (weight.shape[0],))

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        dy = _rows(dy)
        dx = dw = None
        if ctx.needs_input_grad[0]:
            dx = _b.matmul_fp8(*_b.quantize_fp8(dy), *_b.quantize_fp8(weight.contiguous(), tile=True, transpose=True),
                               out_dtype=x.dtype).view(x.shape)
        if ctx.needs_input_grad[1]:
            dw = _b.matmul_fp8(*_b.quantize_fp8(dy, transpose=True), *_b.quantize_fp8(_rows(x), transpose=True),
                               out_dtype=weight.dtype)
        return dx, dw


def linear_fp8(x, weight):
    """Differentiable projection x (..., k) by weight (n, k), each fp32 or bf16, with every product in 8 bits: (..., n) in
    x's type.  Both may be strided; they are copied for each of their products then.  x and the gradient are quantised per
    row and the weight per tile, as ``quantize_fp8`` does it; the weight's gradient is the product of both per column,
    along the rows, and in fp32 for an fp32 weight, which takes twice as long.  Gradients are those of the unrounded
    product, taken once: a second derivative raises."""
    if not isinstance(x, torch.Tensor) or x.dim() < 1:
        raise _b.MBScanError("x must be a (..., k) tensor")
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
        raise _b.MBScanError("weight must be a (n, k) tensor")
    return _LinearFp8.apply(x, weight)
