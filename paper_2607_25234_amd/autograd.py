"""torch.autograd wrappers of the WHTMix C ABI (argument marshalling only).

    y = whtmix_mix(x, gain)                                  # joint gain G[N_pad, C]
    y = whtmix_mix_separable(x, log_gain_tokens, log_gain_channels)
    y = whtmix_block(x, w_in, gain, w_out)                   # eqs. (1)-(4)
    y = whtmix_block_separable(x, w_in, log_gain_tokens, log_gain_channels, w_out)
    y, h = whtmix_norm(x, weight, residual)                  # residual's addition and norm
    y = whtmix_linear(x, w, bias, activation, residual)      # feed-forward product

The forward and backward passes both run in the HIP kernels of libwhtmix.so
(whtmix_*forward*/whtmix_*backward*); gradients flow to x and to the gains, as
when the paper trains the mixer (section IV-A).  The gradients have no gradients
of their own: a second backward pass through them raises.
"""
from __future__ import annotations

import functools

import torch

from . import whtmix


class _Gradients(torch.autograd.Function):
    """backward(ctx, *dys) as a node of the graph that a pass with create_graph=True records, with
    edges to all it depends on (dys and what ctx saved).  torch's once_differentiable has
    none to the saved tensors: a second pass that reaches them another way skips its error."""

    @staticmethod
    def forward(_, backward, ctx, count, *tensors):
        return backward(ctx, *tensors[:count])

    @staticmethod
    def backward(_, *grads):
        raise RuntimeError("libwhtmix forms first derivatives only: no second derivative goes "
                           "through its gradients")


def _first_order(backward):
    """A Function's backward whose results the kernels form."""
    @functools.wraps(backward)
    def run(ctx, *dys):
        if not torch.is_grad_enabled():
            return backward(ctx, *dys)
        return _Gradients.apply(backward, ctx, len(dys), *dys, *ctx.saved_tensors)
    return run


class WHTMixFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain):
        x = x.contiguous()
        gain = gain.contiguous()
        ctx.save_for_backward(x, gain)
        return whtmix.forward(x, gain)

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        x, gain = ctx.saved_tensors
        dx, dgain = whtmix.backward(x, dy.contiguous(), gain,
                                    want_dx=ctx.needs_input_grad[0],
                                    want_dgain=ctx.needs_input_grad[1])
        return dx, dgain


class WHTMixSeparableFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, log_gain_tokens, log_gain_channels):
        x = x.contiguous()
        gt = log_gain_tokens.contiguous()
        gc = log_gain_channels.contiguous()
        ctx.save_for_backward(x, gt, gc)
        return whtmix.forward_separable(x, gt, gc)

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        x, gt, gc = ctx.saved_tensors
        want_g = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dx, dgt, dgc = whtmix.backward_separable(x, dy.contiguous(), gt, gc,
                                                 want_dx=ctx.needs_input_grad[0],
                                                 want_dgains=want_g)
        return dx, dgt, dgc


class WHTMixBlockFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_in, gain, w_out):
        x, w_in, gain, w_out = (t.contiguous() for t in (x, w_in, gain, w_out))
        ctx.save_for_backward(x, w_in, gain, w_out)
        return whtmix.module_forward(x, w_in, gain, w_out)

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        x, w_in, gain, w_out = ctx.saved_tensors
        dx, dwi, dwo, dg = whtmix.module_backward(x, w_in, gain, w_out, dy.contiguous(),
                                                  want_dgain=ctx.needs_input_grad[2])
        return dx, dwi.to(w_in.dtype), dg, dwo.to(w_out.dtype)


class WHTMixBlockSeparableFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_in, log_gain_tokens, log_gain_channels, w_out):
        x, w_in, gt, gc, w_out = (t.contiguous() for t in
                                  (x, w_in, log_gain_tokens, log_gain_channels, w_out))
        ctx.save_for_backward(x, w_in, gt, gc, w_out)
        return whtmix.module_forward_separable(x, w_in, gt, gc, w_out)

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        x, w_in, gt, gc, w_out = ctx.saved_tensors
        want_g = ctx.needs_input_grad[2] or ctx.needs_input_grad[3]
        dx, dwi, dwo, dgt, dgc = whtmix.module_backward_separable(
            x, w_in, gt, gc, w_out, dy.contiguous(), want_dgains=want_g)
        return dx, dwi.to(w_in.dtype), dgt, dgc, dwo.to(w_out.dtype)


def _strided_rows(x):
    """x, or a copy where its rows are not contiguous or not a constant distance apart."""
    try:
        rows, width, ld = whtmix._rows(x, "x")
    except ValueError:
        return x.contiguous()
    return x if rows <= 1 or ld >= width else x.contiguous()


class WHTMixNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        x, weight = _strided_rows(x), weight.contiguous()
        y, h = whtmix.norm(x, weight, None if residual is None else residual.contiguous(), eps)
        if residual is None:      # the stream is x itself
            h = x.contiguous()
        ctx.save_for_backward(h, weight)
        ctx.eps, ctx.residual = eps, residual is not None
        return (y, h) if residual is not None else y

    @staticmethod
    @_first_order
    def backward(ctx, dy, dh=None):
        h, weight = ctx.saved_tensors
        dx, dw = whtmix.norm_backward(h, weight, dy.contiguous(),
                                      None if dh is None else dh.contiguous(), ctx.eps,
                                      want_dweight=ctx.needs_input_grad[1])
        return dx, dw, dx if ctx.residual else None, None


class WHTMixLinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, activation, residual):
        x, w = _strided_rows(x), w.contiguous()
        z = None
        # z is kept only where the activation's derivative needs it
        keep = activation != "none" and any(ctx.needs_input_grad[:3])
        y = whtmix.linear(x, w, None if bias is None else bias.contiguous(), activation,
                          None if residual is None else residual.contiguous(), want_z=keep)
        if keep:
            y, z = y
        ctx.save_for_backward(x, w, z)
        ctx.activation = activation
        return y

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        x, w, z = ctx.saved_tensors
        want = ctx.needs_input_grad
        dx = dw = db = None
        if any(want[:3]):
            dx, dw, db = whtmix.linear_backward(x, w, dy.contiguous(), z, ctx.activation,
                                                want_dx=want[0], want_dw=want[1],
                                                want_dbias=want[2])
        return dx, dw, db, None, dy if want[4] else None


def whtmix_norm(x, weight, residual=None, eps: float = 1e-6):
    """Differentiable norm with the residual's addition: (y, h), h = x + residual (x itself
    without one).  weight float32, and its gradient."""
    if residual is None:
        return WHTMixNormFunction.apply(x, weight, None, eps), x
    return WHTMixNormFunction.apply(x, weight, residual, eps)


def whtmix_linear(x, w, bias=None, activation: str = "none", residual=None):
    """Differentiable activation(x w + bias) + residual; dw in w's type, the
    bias and its gradient float32."""
    return WHTMixLinearFunction.apply(x, w, bias, activation, residual)


def whtmix_block(x, w_in, gain, w_out):
    """Differentiable block of eqs. (1)-(4): mixer(x W_in) W_out (joint gain).
    Weight gradients are computed in float32 and returned in the weights' dtype."""
    return WHTMixBlockFunction.apply(x, w_in, gain, w_out)


def whtmix_block_separable(x, w_in, log_gain_tokens, log_gain_channels, w_out):
    """Differentiable block with the paper's log-domain gains."""
    return WHTMixBlockSeparableFunction.apply(x, w_in, log_gain_tokens, log_gain_channels, w_out)


def whtmix_mix(x, gain):
    """Differentiable y = H_N (G o (H_N x H_C)) H_C."""
    return WHTMixFunction.apply(x, gain)


def whtmix_mix_separable(x, log_gain_tokens, log_gain_channels):
    """Differentiable eq. (2) then eq. (3) with log-domain gains."""
    return WHTMixSeparableFunction.apply(x, log_gain_tokens, log_gain_channels)
