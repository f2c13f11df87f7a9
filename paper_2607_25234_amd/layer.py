"""A layer around the mixer, as a model stacks them: the block of eqs. (1)-(4), the
residual's addition with a norm, and the feed-forward sublayer.

    h = x + block(x)
    y = h + act(norm(h) W1 + b1) W2 + b2                        # or, gated:
    y = h + (act(norm(h) W1 + b1) * (norm(h) Wu + bu)) W2 + b2

The norm is the root mean square's ("rms") or the layer norm with its bias ("layer").

MixerLayer trains it (every step in the library's kernels, forward and backward).
MixerLayerMx serves the state of a trained layer with its feed-forward weights in block-scaled
8 bits, laid out once: the norm writes 8-bit rows, the first product (or both gated ones in a
kernel) reads them and writes 8-bit rows again, the second adds its result to the stream.

    layer = MixerLayer(tokens=4096, width=64, hidden=256, dtype=torch.float32).cuda()
    y = layer(x)                       # x [B, tokens, width]
    served = MixerLayerMx(layer)
    y = served(x)

MixerText stacks them on embedded tokens, as the sequence classification tasks of section IV-D
embed theirs; a negative id is padding, whose row is zeros.

    text = MixerText(vocab=256, tokens=4096, width=64, hidden=172, depth=4, norm="layer",
                     gated=True).cuda()
    y = text(ids)                      # ids [B, tokens] -> [B, tokens, width]
"""
from __future__ import annotations

import torch

from . import autograd, whtmix

NORMS = ("rms", "layer")


class MixerLayer(torch.nn.Module):
    def __init__(self, tokens: int, width: int, hidden: int, activation: str = "gelu",
                 dtype=torch.bfloat16, eps: float = 1e-6, device=None, norm: str = "rms",
                 gated: bool = False):
        super().__init__()
        if norm not in NORMS:
            raise ValueError(f"norm {norm!r}: one of {', '.join(NORMS)}")
        n_pad = whtmix.padded_tokens(tokens)
        f32 = dict(dtype=torch.float32, device=device)

        def matrix(k, n):
            return torch.nn.Parameter(
                (torch.randn(k, n, **f32) * k ** -0.5).to(dtype))

        def zeros(n):
            return torch.nn.Parameter(torch.zeros(n, **f32))

        self.w_in, self.w_out = matrix(width, width), matrix(width, width)
        self.log_gain_tokens = zeros(n_pad)
        self.log_gain_channels = zeros(width)
        self.norm_weight = torch.nn.Parameter(torch.ones(width, **f32))
        self.w1, self.w2 = matrix(width, hidden), matrix(hidden, width)
        self.b1 = zeros(hidden)
        self.b2 = zeros(width)
        if norm == "layer":
            self.norm_bias = zeros(width)
        if gated:
            self.w_up = matrix(width, hidden)
            self.b_up = zeros(hidden)
        self.activation, self.eps, self.norm, self.gated = activation, eps, norm, gated

    def forward(self, x):
        m = autograd.whtmix_block_separable(x, self.w_in, self.log_gain_tokens,
                                            self.log_gain_channels, self.w_out)
        if self.norm == "layer":
            y, h = autograd.whtmix_layer_norm(m, self.norm_weight, self.norm_bias, x, self.eps)
        else:
            y, h = autograd.whtmix_norm(m, self.norm_weight, x, self.eps)
        if self.gated:
            u = autograd.whtmix_gated(y, self.w1, self.w_up, self.b1, self.b_up, self.activation)
        else:
            u = autograd.whtmix_linear(y, self.w1, self.b1, self.activation)
        return autograd.whtmix_linear(u, self.w2, self.b2, residual=h)


class MixerLayerMx:
    """A trained MixerLayer at inference, its feed-forward weights in 8 bits.  It holds copies
    of all the layer's weights: what the layer learns afterwards does not reach it."""

    def __init__(self, layer: MixerLayer):
        names = ["w_in", "w_out", "log_gain_tokens", "log_gain_channels", "norm_weight", "b1", "b2"]
        if layer.norm == "layer":
            names.append("norm_bias")
        if layer.gated:
            names.append("b_up")
        with torch.no_grad():
            for name in names:
                setattr(self, name, getattr(layer, name).detach().clone())
            self.w1 = whtmix.quantize_mx(layer.w1.t().contiguous())
            self.w2 = whtmix.quantize_mx(layer.w2.t().contiguous())
            if layer.gated:
                self.w_up = whtmix.quantize_mx(layer.w_up.t().contiguous())
        self.activation, self.eps = layer.activation, layer.eps
        self.norm, self.gated = layer.norm, layer.gated

    @torch.no_grad()
    def __call__(self, x):
        m = whtmix.module_forward_separable(x, self.w_in, self.log_gain_tokens,
                                            self.log_gain_channels, self.w_out)
        if self.norm == "layer":
            q, scales, h = whtmix.layer_norm_mx(m, self.norm_weight, self.norm_bias, x, self.eps)
        else:
            q, scales, h = whtmix.norm_mx(m, self.norm_weight, x, self.eps)
        if self.gated:
            q, scales = whtmix.gated_mx(q, scales, *self.w1, *self.w_up, self.b1, self.b_up,
                                        self.activation, out_mx=True)
        else:
            q, scales = whtmix.linear_mx(q, scales, *self.w1, self.b1, self.activation,
                                         out_mx=True)
        return whtmix.linear_mx(q, scales, *self.w2, self.b2, residual=h)


class MixerText(torch.nn.Module):
    """Embedded tokens through a stack of layers, whose options MixerLayer takes."""

    def __init__(self, vocab: int, tokens: int, width: int, hidden: int, depth: int,
                 dtype=torch.bfloat16, device=None, **options):
        super().__init__()
        self.table = torch.nn.Parameter(
            (torch.randn(vocab, width, dtype=torch.float32, device=device) * width ** -0.5)
            .to(dtype))
        self.layers = torch.nn.ModuleList(
            MixerLayer(tokens, width, hidden, dtype=dtype, device=device, **options)
            for _ in range(depth))
        self.scale = width ** 0.5

    def forward(self, ids):
        x = autograd.whtmix_embedding(ids, self.table, self.scale)
        for layer in self.layers:
            x = layer(x)
        return x
