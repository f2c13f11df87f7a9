"""GPU tests of the feed-forward products on sizes that take the large tiles: 256 x 256 tiles of
each type and layout, float32 operands split in a pass of their own, parts of k with many partial
sums, and 8 bits on the scaled matrix instructions."""
from __future__ import annotations

import math

import pytest
import torch

from tests import layer_ref as ref
from tests.gpu_util import device, say
from tests.test_gpu_layer import DTYPES, draw

pytestmark = pytest.mark.gpu


# Square enough for 192 tiles of 256 x 256 (whole ones, and ragged edges with odd widths),
# and k of one step, of two, of an odd count of steps and elements.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(3584, 64, 3584), (3600, 128, 3700), (3585, 200, 3531),
                                   (4000, 331, 3203), (2500, 1200, 2500), (2401, 1203, 2603)])
def test_large_product(M, K, N, dtype):
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    act = ref.ACTS[(M + K) % 5]
    say("large_product", M, K, N, dtype, act)
    x, w = draw(1, M, K, dtype=dt), draw(2, K, N, std=K ** -0.5, dtype=dt)
    b, r = draw(3, N, std=0.3), draw(4, M, N, dtype=dt)
    X, W, R = x.double(), w.double(), r.double()
    z = X @ W + b.double()
    dz = ref.sum_bound(K, X.abs() @ W.abs() + b.double().abs())
    y = ref.act(act, z) + R
    got, gz = whtmix.linear(x.to(dev), w.to(dev), b.to(dev), act, r.to(dev), want_z=True)
    ref.check("y", got, y, ref.act_bound(act, z, dz) + ref.rounded(y, bf))
    ref.check("z", gz, z, dz + ref.rounded(z, bf))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(3600, 3500, 96), (2500, 2500, 1200), (40000, 136, 264),
                                   (30011, 70, 131)])
def test_large_backward(M, K, N, dtype):
    """dx over large tiles, dw over many parts of the rows."""
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    say("large_backward", M, K, N, dtype)
    x, w = draw(1, M, K, dtype=dt), draw(2, K, N, std=K ** -0.5, dtype=dt)
    dy, z = draw(3, M, N, dtype=dt), draw(4, M, N, dtype=dt)
    dx, dw, db = whtmix.linear_backward(x.to(dev), w.to(dev), dy.to(dev), z.to(dev), "silu")
    X, W, D = x.double(), w.double(), dy.double()
    d = D * ref.act_grad("silu", z.double())
    own = D.abs() * ref.grad_bound("silu", z.double())
    rnd = own + d.abs() * (2.0 ** -7.99 if bf else 4 * ref.U)
    rx, rw = d @ W.t(), X.t() @ d
    ref.check("dx", dx, rx, ref.sum_bound(N, d.abs() @ W.abs().t()) + rnd @ W.abs().t()
              + ref.rounded(rx, bf))
    ref.check("dw", dw, rw, ref.sum_bound(M, X.abs().t() @ d.abs()) + X.abs().t() @ rnd
              + ref.rounded(rw, bf))
    ref.check("db", db, d.sum(0), ref.sum_bound(M, d.abs().sum(0)) + own.sum(0) + 1e-30)


@pytest.mark.parametrize("out_mx", [False, True])
@pytest.mark.parametrize("M,K,N", [(3584, 256, 3584), (3600, 96, 3700), (3585, 544, 3531),
                                   (2000, 2080, 1000)])
def test_large_mx(M, K, N, out_mx):
    """8 bits on large tiles.  With K > 512 the scaled matrix instructions add the products of 64 k
    in a common alignment that keeps some 15 bits below the largest of them: each group of
    64 adds at most 2^-13 of its largest product to the error (two halves of the instruction,
    a bit each for the two roundings)."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    say("large_mx", M, K, N, out_mx)
    xq, xs = whtmix.quantize_mx(draw(1, M, K).to(dev))
    wq, ws = whtmix.quantize_mx(draw(2, N, K, std=K ** -0.5).to(dev))
    x = whtmix.dequantize_mx(xq, xs, K, torch.float32).cpu().double()
    w = whtmix.dequantize_mx(wq, ws, K, torch.float32).cpu().double()
    b = draw(3, N, std=0.3)
    z = x @ w.t() + b.double()
    dz = ref.sum_bound(K, x.abs() @ w.abs().t() + b.double().abs())
    if K > 512:
        gx = torch.nn.functional.pad(x.abs(), (0, -K % 64)).reshape(M, -1, 64).amax(-1)
        gw = torch.nn.functional.pad(w.abs(), (0, -K % 64)).reshape(N, -1, 64).amax(-1)
        dz = dz + 2.0 ** -13 * (gx @ gw.t())
    y = ref.act("gelu", z)
    by = ref.act_bound("gelu", z, dz) + (y.abs() + 1) * 2 * ref.U
    if not out_mx:
        got = whtmix.linear_mx(xq, xs, wq, ws, b.to(dev), "gelu")
        ref.check("y", got, y, by + ref.rounded(y, True))
        return
    q, s = whtmix.linear_mx(xq, xs, wq, ws, b.to(dev), "gelu", out_mx=True)
    unit = torch.exp2(s.cpu().double() - 127).repeat_interleave(32, -1)[:, :N]
    v = whtmix.dequantize_mx(q, s, N, torch.float32)
    step = torch.maximum(torch.exp2(torch.floor(torch.log2((y / unit).abs().clamp(min=1e-30)))
                                    - 3), torch.full_like(y, 2.0 ** -9)) * unit
    ref.check("q", v, y, step * 0.5 * (1 + 1e-6) + 2 * by)


def test_large_float32_operands_that_do_not_split():
    """Inf, NaN, and values beyond three bf16 terms where the operands are split first: the
    tiles they are in take float32 products, the others are what they were."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    M, K, N = 2500, 1200, 2500
    say("large, do not split")
    x, w = draw(1, M, K), draw(2, K, N, std=K ** -0.5)
    plain = whtmix.linear(x.to(dev), w.to(dev))
    x, w = x.clone(), w.clone()
    x[1, 3], x[700, 5], w[7, 1300] = math.inf, math.nan, -math.inf
    x[1900, :] *= 2.0 ** -110
    w[:, 2000] = w[:, 2000] * 2.0 ** -60
    x[2300, :] = x[2300, :].clamp(-1.9, 1.9) * 2.0 ** 127
    z = x.double() @ w.double()
    fin = torch.nan_to_num(x.double(), nan=0, posinf=0, neginf=0).abs() @ torch.nan_to_num(
        w.double(), nan=0, posinf=0, neginf=0).abs()
    # of the large row, the column whose sums stay in float32's range
    z[2300, :2000], z[2300, 2001:] = 0, 0
    got = whtmix.linear(x.to(dev), w.to(dev)).cpu()
    got[2300, :2000], got[2300, 2001:] = 0, 0
    ref.check("z", got, z, ref.sum_bound(K, fin) + 2.0 ** -140)
    rows = [r for r in range(M) if not (0 <= r < 256 or 512 <= r < 768 or r >= 1792)]
    cols = [c for c in range(N) if not (1280 <= c < 1536 or 1792 <= c < 2048)]
    assert torch.equal(got[rows][:, cols], plain.cpu()[rows][:, cols])


@pytest.mark.parametrize("M,K,N,act", [(32768, 128, 64, "gelu"), (33001, 100, 200, "silu"),
                                       (32800, 1, 72, "relu"), (40000, 128, 520, "gelu_tanh"),
                                       (36000, 127, 136, "gelu")])
def test_narrow_backward(M, K, N, act):
    """Many rows of narrow bf16 inputs: dz, its sums and dx in one pass."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    say("narrow_backward", M, K, N, act)
    dt = torch.bfloat16
    x, w = draw(1, M, K, dtype=dt), draw(2, K, N, std=K ** -0.5, dtype=dt)
    dy, z = draw(3, M, N, dtype=dt), draw(4, M, N, std=2.0, dtype=dt)
    args = x.to(dev), w.to(dev), dy.to(dev), z.to(dev), act
    dx, dw, db = whtmix.linear_backward(*args)
    X, W, D = x.double(), w.double(), dy.double()
    d = D * ref.act_grad(act, z.double())
    own = D.abs() * ref.grad_bound(act, z.double())
    rnd = own + d.abs() * 2.0 ** -7.99
    rx, rw = d @ W.t(), X.t() @ d
    ref.check("dx", dx, rx, ref.sum_bound(N, d.abs() @ W.abs().t()) + rnd @ W.abs().t()
              + ref.rounded(rx, True))
    ref.check("dw", dw, rw, ref.sum_bound(M, X.abs().t() @ d.abs()) + X.abs().t() @ rnd
              + ref.rounded(rw, True))
    ref.check("db", db, d.sum(0), ref.sum_bound(M, d.abs().sum(0)) + own.sum(0) + 1e-30)
    again = whtmix.linear_backward(*args)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db)))
    only, none, nodb = whtmix.linear_backward(*args, want_dw=False, want_dbias=False)
    assert torch.equal(only, dx) and none is None and nodb is None
