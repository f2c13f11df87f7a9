"""A layer around the mixer, as a model stacks them: the block of eqs. (1)-(4), the
residual's addition with a norm, and the feed-forward sublayer.

    h = x + block(x)
    y = h + act(norm(h) W1 + b1) W2 + b2

MixerLayer trains it (every step in the library's kernels, forward and backward).
MixerLayerMx serves the state of a trained layer with its feed-forward weights in block-scaled
8 bits, laid out once: the norm writes 8-bit rows, the first product reads them
and writes 8-bit rows again, the second adds its result to the stream.

    layer = MixerLayer(tokens=4096, width=64, hidden=256, dtype=torch.float32).cuda()
    y = layer(x)                       # x [B, tokens, width]
    served = MixerLayerMx(layer)
    y = served(x)
"""
from __future__ import annotations

import torch

from . import autograd, whtmix


class MixerLayer(torch.nn.Module):
    def __init__(self, tokens: int, width: int, hidden: int, activation: str = "gelu",
                 dtype=torch.bfloat16, eps: float = 1e-6, device=None):
        super().__init__()
        n_pad = whtmix.padded_tokens(tokens)
        f32 = dict(dtype=torch.float32, device=device)

        def matrix(k, n):
            return torch.nn.Parameter(
                (torch.randn(k, n, **f32) * k ** -0.5).to(dtype))

        self.w_in, self.w_out = matrix(width, width), matrix(width, width)
        self.log_gain_tokens = torch.nn.Parameter(torch.zeros(n_pad, **f32))
        self.log_gain_channels = torch.nn.Parameter(torch.zeros(width, **f32))
        self.norm_weight = torch.nn.Parameter(torch.ones(width, **f32))
        self.w1, self.w2 = matrix(width, hidden), matrix(hidden, width)
        self.b1 = torch.nn.Parameter(torch.zeros(hidden, **f32))
        self.b2 = torch.nn.Parameter(torch.zeros(width, **f32))
        self.activation, self.eps = activation, eps

    def forward(self, x):
        m = autograd.whtmix_block_separable(x, self.w_in, self.log_gain_tokens,
                                            self.log_gain_channels, self.w_out)
        y, h = autograd.whtmix_norm(m, self.norm_weight, x, self.eps)
        u = autograd.whtmix_linear(y, self.w1, self.b1, self.activation)
        return autograd.whtmix_linear(u, self.w2, self.b2, residual=h)


class MixerLayerMx:
    """A trained MixerLayer at inference, its feed-forward weights in 8 bits.  It holds copies
    of all the layer's weights: what the layer learns afterwards does not reach it."""

    def __init__(self, layer: MixerLayer):
        with torch.no_grad():
            for name in ("w_in", "w_out", "log_gain_tokens", "log_gain_channels", "norm_weight",
                         "b1", "b2"):
                setattr(self, name, getattr(layer, name).detach().clone())
            self.w1 = whtmix.quantize_mx(layer.w1.t().contiguous())
            self.w2 = whtmix.quantize_mx(layer.w2.t().contiguous())
        self.activation, self.eps = layer.activation, layer.eps

    @torch.no_grad()
    def __call__(self, x):
        m = whtmix.module_forward_separable(x, self.w_in, self.log_gain_tokens,
                                            self.log_gain_channels, self.w_out)
        q, scales, h = whtmix.norm_mx(m, self.norm_weight, x, self.eps)
        q, scales = whtmix.linear_mx(q, scales, *self.w1, self.b1, self.activation, out_mx=True)
        return whtmix.linear_mx(q, scales, *self.w2, self.b2, residual=h)
