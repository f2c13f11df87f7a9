"""GPU tests of the feed-forward operators where float32's accuracy and the range of the
values are at their limits, and of what a training or serving program does around them."""
from __future__ import annotations

import math

import pytest
import torch

from tests import layer_ref as ref
from tests.gpu_util import device, say
from tests.test_gpu_layer import DTYPES, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out", ["bf16", "f32", "mx"])
@pytest.mark.parametrize("M,N", [(20, 130), (60, 200), (256, 288)])
@pytest.mark.parametrize("K", [64, 160, 256, 320, 512])
def test_mx_sums_of_few_k_are_float32(M, N, K, out):
    """Every product comes twice with opposite signs, in another order, so that each sum is 0:
    what is left is the error of the sum, which an output's rounding does not hide.  The
    bound is float32's (layer_ref); 8-bit outputs add at most an eighth to what they round."""
    from paper_2607_25234_amd import whtmix
    dev, h = device(), K // 2
    say("mx_sums", M, N, K, out)
    g = torch.Generator().manual_seed(K)

    def values(rows):
        v = torch.randn(rows, h, generator=g) * torch.exp2(torch.rand(rows, h, generator=g) * 6)
        return v.clamp(-448, 448).to(torch.float8_e4m3fn).float()

    x, w, p = values(M), values(N), torch.randperm(h, generator=g)
    x, w = torch.cat([x, x[:, p]], 1), torch.cat([w, -w[:, p]], 1)

    def rows(v):     # scales of 1
        return (v.to(torch.float8_e4m3fn).to(dev),
                torch.full((v.shape[0], K // 32), 127, dtype=torch.uint8, device=dev))

    mag = x.double().abs() @ w.double().abs().t()
    bound = ref.sum_bound(K, mag)
    if out == "mx":
        q, s = whtmix.linear_mx(*rows(x), *rows(w), out_mx=True)
        y = whtmix.dequantize_mx(q, s, N, torch.float32)
        top = torch.nn.functional.pad(bound, (0, -N % 32)).reshape(M, -1, 32).amax(-1)
        bound = 1.125 * top.repeat_interleave(32, -1)[:, :N]
    else:
        y = whtmix.linear_mx(*rows(x), *rows(w), dtype=DTYPES[out])
        bound = bound * 1.01
    ref.check("sum", y, torch.zeros_like(mag), bound)
