"""GPU tests of the feed-forward operators against the 64-bit reference."""
from __future__ import annotations

import math

import pytest
import torch

from tests import layer_ref as ref
from tests.gpu_util import device, say

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(seed, *shape, std=1.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype)


# widths: one element, odd, below and above a chunk, a block of 32, every lane
# count of the kernels' table, and past what registers hold
NORM_SHAPES = [(1, 1), (3, 2), (5, 7), (33, 8), (4, 31), (2, 32), (65, 33), (17, 64), (9, 100),
               (130, 128), (31, 255), (6, 256), (7, 513), (300, 1024), (3, 1111), (5, 2048),
               (1, 4096), (3, 4097), (2, 8200), (2, 16384), (2, 20000), (3, 33000), (2, 70001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", NORM_SHAPES)
@pytest.mark.parametrize("res", [False, True])
def test_norm(rows, C, dtype, res):
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("norm", rows, C, dtype, res)
    x, w = draw(1, rows, C, dtype=dt), 1 + draw(2, C, std=0.1)
    r = draw(3, rows, C, std=2.0, dtype=dt) if res else None
    y, h = whtmix.norm(x.to(dev), w.to(dev), r.to(dev) if res else None, eps=1e-5)
    t = x.double() + (r.double() if res else 0)
    rstd = 1 / (t.square().mean(-1, keepdim=True) + 1e-5).sqrt()
    n = t * rstd * w.double()
    bf = dtype == "bf16"
    rel = 8 * (4 + math.sqrt(C)) * ref.U
    # where x and the residual nearly cancel, t's own rounding counts
    dt_ = (x.double().abs() + (r.double().abs() if res else 0)) * ref.U * rstd * w.double().abs()
    ref.check("y", y, n, n.abs() * rel + dt_ + ref.rounded(n, bf))
    ref.check("h", h, t, ref.rounded(t, bf) + (x.double().abs() + t.abs()) * 2 * ref.U)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", NORM_SHAPES + [(1000, 128), (5000, 48), (2049, 520)])
@pytest.mark.parametrize("res", [False, True])
def test_norm_backward(rows, C, dtype, res):
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("norm_backward", rows, C, dtype, res)
    h, w = draw(1, rows, C, dtype=dt), 1 + draw(2, C, std=0.1)
    dy = draw(3, rows, C, dtype=dt)
    dh = draw(4, rows, C, dtype=dt) if res else None
    dx, dw = whtmix.norm_backward(h.to(dev), w.to(dev), dy.to(dev),
                                  dh.to(dev) if res else None, eps=1e-5)
    H, W, D = h.double(), w.double(), dy.double()
    rstd = 1 / (H.square().mean(-1, keepdim=True) + 1e-5).sqrt()
    n, g = H * rstd, D * W
    rx = rstd * (g - n * (g * n).mean(-1, keepdim=True))
    mag = rstd * (g.abs() + n.abs() * (g * n).abs().mean(-1, keepdim=True))
    if res:
        rx, mag = rx + dh.double(), mag + dh.double().abs()
    ref.check("dx", dx, rx, ref.sum_bound(C, mag) + ref.rounded(rx, dtype == "bf16"))
    ref.check("dw", dw, (D * n).sum(0),
              ref.sum_bound(rows, (D * n).abs().sum(0)) + ref.sum_bound(C, (D * n).abs().sum(0)))
    only, none = whtmix.norm_backward(h.to(dev), w.to(dev), dy.to(dev),
                                      dh.to(dev) if res else None, eps=1e-5, want_dweight=False)
    assert none is None and torch.equal(only, dx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", NORM_SHAPES)
def test_quantize_mx(rows, C, dtype):
    """Bit for bit the definition: values spread over e4m3's range, exact ties, block maxima at
    and beside 448 * 2^e, zero and subnormal blocks, Inf and NaN in a block."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("quantize_mx", rows, C, dtype)
    x = draw(1, rows, C) * torch.exp2(torch.randint(-12, 4, (rows, C),
                                                    generator=torch.Generator().manual_seed(2)))
    x[0, : min(C, 8)] = torch.tensor([448.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, -440.0,
                                      0.0, 432.0])[: min(C, 8)]
    if rows > 1:
        x[1, C // 2:] = 0.0
        x[1, C - 1] = 1e-38
    if rows > 2:
        x[2, C // 3] = math.inf
        x[2, C - 1] = math.nan
        x[2, 0] = 3e38
    x = x.to(dt)
    q, s = whtmix.quantize_mx(x.to(dev))
    values, scales = ref.mx_round(x.double())
    assert q.shape == (rows, whtmix.mx_width(C)) and torch.equal(s.cpu(), scales)
    back = q.cpu().float().double() * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)
    assert torch.equal(torch.nan_to_num(back[:, :C], nan=1e30),
                       torch.nan_to_num(values, nan=1e30))
    assert not back[:, C:].any()
    y = whtmix.dequantize_mx(q, s, C, dt)
    exact = values.to(dt)
    assert torch.equal(torch.nan_to_num(y.cpu().float(), nan=1e30),
                       torch.nan_to_num(exact.float(), nan=1e30))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", [(1, 1), (5, 33), (17, 64), (130, 128), (3, 1111), (2, 4096),
                                    (2, 8200), (2, 70001)])
def test_norm_mx(rows, C, dtype):
    """Each value is a nearest e4m3 value of the norm in 64 bits (half a step, with float32's
    error of the norm), and each block's scale the definition's or, where its maximum is within
    that error of a limit, a neighbour's."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("norm_mx", rows, C, dtype)
    x, w, r = draw(1, rows, C, dtype=dt), 1 + draw(2, C, std=0.1), draw(3, rows, C, dtype=dt)
    q, s, h = whtmix.norm_mx(x.to(dev), w.to(dev), r.to(dev), eps=1e-5)
    t = x.double() + r.double()
    n = t / (t.square().mean(-1, keepdim=True) + 1e-5).sqrt() * w.double()
    rel = 8 * (4 + math.sqrt(C)) * ref.U
    own = n.abs() * rel + (x.double().abs() + r.double().abs()) * 8 * ref.U
    scales = s.cpu().double() - 127
    lo = ref.mx_round(n * (1 - 2 * rel))[1].double() - 127
    hi = ref.mx_round(n * (1 + 2 * rel))[1].double() - 127
    assert ((scales >= lo) & (scales <= hi)).all()
    unit = torch.exp2(scales).repeat_interleave(32, -1)[:, :C]
    v = whtmix.dequantize_mx(q, s, C, torch.float32)
    step = torch.maximum(torch.exp2(torch.floor(torch.log2((n / unit).abs().clamp(min=1e-30)))
                                    - 3), torch.full_like(n, 2.0 ** -9)) * unit
    ref.check("q", v, n, step * 0.5 * (1 + 1e-6) + own)
    ref.check("h", h, t, ref.rounded(t, dtype == "bf16") + own)


# tokens, widths: single tokens, decode batches, tile edges, odd widths, long k, many rows
LINEAR_SHAPES = [(1, 1, 1), (1, 64, 64), (1, 4096, 512), (2, 33, 7), (7, 200, 130), (16, 1000, 96),
                 (17, 2048, 257), (31, 8, 300), (64, 64, 256), (65, 129, 127), (128, 128, 128),
                 (129, 96, 260), (200, 31, 33), (256, 512, 256), (257, 520, 520), (300, 1003, 517),
                 (511, 65, 1030), (1024, 256, 1024), (1500, 72, 200), (5000, 64, 256)]


def linear_case(M, K, N, dtype, act, res, seed=1):
    dt = DTYPES[dtype]
    x, w = draw(seed, M, K, dtype=dt), draw(seed + 1, K, N, std=K ** -0.5, dtype=dt)
    b = draw(seed + 2, N, std=0.3)
    r = draw(seed + 3, M, N, dtype=dt) if res else None
    z = x.double() @ w.double() + b.double()
    dz = ref.sum_bound(K, x.double().abs() @ w.double().abs() + b.double().abs())
    y = ref.act(act, z) + (r.double() if res else 0)
    by = ref.act_bound(act, z, dz) + ref.rounded(y, dtype == "bf16")
    return x, w, b, r, z, dz, y, by


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", LINEAR_SHAPES)
def test_linear(M, K, N, dtype):
    from paper_2607_25234_amd import whtmix
    dev = device()
    act, res = ref.ACTS[(M + K + N) % 5], (M + N) % 2 == 0
    say("linear", M, K, N, dtype, act, res)
    x, w, b, r, z, dz, y, by = linear_case(M, K, N, dtype, act, res)
    X, W, B = x.to(dev), w.to(dev), b.to(dev)
    R = r.to(dev) if res else None
    got, gz = whtmix.linear(X, W, B, act, R, want_z=True)
    ref.check("y", got, y, by)
    ref.check("z", gz, z, dz + ref.rounded(z, dtype == "bf16"))
    assert torch.equal(whtmix.linear(X, W, B, act, R), got)          # the same with no z
    if res:                                                          # onto the residual itself
        assert torch.equal(whtmix.linear(X, W, B, act, R, out=R), got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("M", [3, 140])
def test_linear_activations(M, dtype, act):
    """Every activation over its range: far tails, zero, both signs."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    K, N = 8, 272
    say("linear_activations", M, dtype, act)
    x = torch.zeros(M, K)
    x[:, 0] = torch.linspace(-3, 3, M)
    x[:, 1] = 1
    w = torch.zeros(K, N)
    w[0] = torch.linspace(-20, 20, N)
    w[1] = torch.linspace(-60, 60, N).roll(N // 2)
    x, w = x.to(dt), w.to(dt)
    z = x.double() @ w.double()
    y, gz = whtmix.linear(x.to(dev), w.to(dev), None, act, want_z=True)
    dz = ref.sum_bound(2, x.double().abs() @ w.double().abs())
    r = ref.act(act, z)
    ref.check("y", y, r, ref.act_bound(act, z, dz) + ref.rounded(r, dtype == "bf16") + 1e-30)
    dy = draw(9, M, N, dtype=dt)
    kept = gz.cpu().double()
    dx, dw, db = whtmix.linear_backward(x.to(dev), w.to(dev), dy.to(dev), gz, act)
    d = dy.double() * ref.act_grad(act, kept)
    own = dy.double().abs() * ref.grad_bound(act, kept)
    ref.check("db", db, d.sum(0), ref.sum_bound(M, d.abs().sum(0)) + own.sum(0) + 1e-30)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", LINEAR_SHAPES + [(20000, 64, 96), (9000, 40, 264)])
def test_linear_backward(M, K, N, dtype):
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    act = ref.ACTS[(M + K + N) % 5]
    say("linear_backward", M, K, N, dtype, act)
    x, w = draw(1, M, K, dtype=dt), draw(2, K, N, std=K ** -0.5, dtype=dt)
    dy, z = draw(3, M, N, dtype=dt), draw(4, M, N, std=2.0, dtype=dt)
    args = x.to(dev), w.to(dev), dy.to(dev), z.to(dev), act
    dx, dw, db = whtmix.linear_backward(*args)
    d = dy.double() * ref.act_grad(act, z.double())
    own = dy.double().abs() * ref.grad_bound(act, z.double())
    # dz is rounded to bf16 for the products: 2^-8 of each of its values
    rnd = own + (d.abs() * 2.0 ** -7.99 if bf and act != "none" else 4 * ref.U * d.abs())
    W, X = w.double(), x.double()
    rx, rw = d @ W.t(), X.t() @ d
    ref.check("dx", dx, rx, ref.sum_bound(N, d.abs() @ W.abs().t()) + rnd @ W.abs().t()
              + ref.rounded(rx, bf))
    ref.check("dw", dw, rw, ref.sum_bound(M, X.abs().t() @ d.abs()) + X.abs().t() @ rnd
              + ref.rounded(rw, bf))
    ref.check("db", db, d.sum(0), ref.sum_bound(M, d.abs().sum(0)) + own.sum(0) + 1e-30)
    for k in range(3):      # each alone is the same
        one = whtmix.linear_backward(*args, want_dx=k == 0, want_dw=k == 1, want_dbias=k == 2)
        assert torch.equal(one[k], (dx, dw, db)[k])
        assert all(v is None for i, v in enumerate(one) if i != k)


@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
def test_gradients_against_differences(act):
    """The kernels' gradients against central differences of the kernels' own forward pass
    (norm, then product) along a random direction: step e = 2^-6, off by e^2 of the third
    derivative and by the forward's float32 error over e, both below 1e-3 of the gradient's norm
    times the direction's."""
    from paper_2607_25234_amd import autograd, whtmix
    dev = device()
    M, K, N = 37, 72, 41
    say("differences", act)
    p = [draw(1, M, K), draw(2, M, K), 1 + draw(3, K, std=0.1), draw(4, K, N, std=K ** -0.5),
         draw(5, N, std=0.1)]
    dy, dh = draw(6, M, N).to(dev), draw(7, M, K).to(dev)

    def loss(x, r, g, w, b):
        y, h = autograd.whtmix_norm(x, g, r, 1e-5)
        o = autograd.whtmix_linear(y, w, b, act)
        return (o.double() * dy.double()).sum() + (h.double() * dh.double()).sum()

    leaf = [t.to(dev).requires_grad_() for t in p]
    loss(*leaf).backward()
    e = 2.0 ** -6
    for i, t in enumerate(p):
        v = draw(10 + i, *t.shape)
        v /= v.norm()
        with torch.no_grad():
            up, down = ([s.to(dev) + (k * e * v.to(dev) if j == i else 0)
                         for j, s in enumerate(p)] for k in (1, -1))
            num = float((loss(*up) - loss(*down)) / (2 * e))
        g = leaf[i].grad.double().cpu()
        assert abs(float((g * v.double()).sum()) - num) <= 1e-3 * float(g.norm()), i


MX_SHAPES = [(1, 32, 32), (1, 4096, 512), (2, 40, 7), (7, 200, 130), (17, 2048, 260), (33, 64, 96),
             (64, 1000, 100), (128, 128, 128), (130, 160, 300), (257, 520, 520), (300, 1003, 517),
             (1024, 256, 1024), (2000, 96, 40)]


@pytest.mark.parametrize("out", ["bf16", "f32", "mx"])
@pytest.mark.parametrize("M,K,N", MX_SHAPES)
def test_linear_mx(M, K, N, out):
    from paper_2607_25234_amd import whtmix
    dev = device()
    act, res = ref.ACTS[(M + K + N) % 5], (M + N) % 2 == 0
    say("linear_mx", M, K, N, out, act, res)
    dt = torch.float32 if out == "f32" else torch.bfloat16
    scale = torch.exp2(torch.arange(M) % 7 - 3.0)[:, None]
    xq, xs = whtmix.quantize_mx((draw(1, M, K) * scale).to(dev))
    wq, ws = whtmix.quantize_mx(draw(2, N, K, std=K ** -0.5).to(dev))
    x = whtmix.dequantize_mx(xq, xs, K, torch.float32).cpu().double()
    w = whtmix.dequantize_mx(wq, ws, K, torch.float32).cpu().double()
    b = draw(3, N, std=0.3)
    r = draw(4, M, N, dtype=dt) if res else None
    z = x @ w.t() + b.double()
    dz = ref.sum_bound(K, x.abs() @ w.abs().t() + b.double().abs())
    y = ref.act(act, z) + (r.double() if res else 0)
    by = ref.act_bound(act, z, dz) + (y.abs() + 1) * 2 * ref.U
    R = r.to(dev) if res else None
    if out != "mx":
        got = whtmix.linear_mx(xq, xs, wq, ws, b.to(dev), act, R, dtype=dt)
        assert got.dtype is dt
        ref.check("y", got, y, by + ref.rounded(y, out == "bf16"))
        return
    q, s = whtmix.linear_mx(xq, xs, wq, ws, b.to(dev), act, R, out_mx=True)
    assert q.shape == (M, whtmix.mx_width(N)) and not q.cpu().float()[:, N:].any()
    unit = torch.exp2(s.cpu().double() - 127).repeat_interleave(32, -1)[:, :N]
    v = whtmix.dequantize_mx(q, s, N, torch.float32)
    step = torch.maximum(torch.exp2(torch.floor(torch.log2((y / unit).abs().clamp(min=1e-30)))
                                    - 3), torch.full_like(y, 2.0 ** -9)) * unit
    ref.check("q", v, y, step * 0.5 * (1 + 1e-6) + 2 * by)
    # the scale of each block is the definition's for a maximum within the error
    top = torch.nn.functional.pad(y.abs(), (0, -N % 32)).reshape(M, -1, 32).amax(-1)
    slack = torch.nn.functional.pad(by, (0, -N % 32)).reshape(M, -1, 32).amax(-1)
    e = s.cpu().double() - 127
    assert (top - slack <= 448 * torch.exp2(e)).all()
    assert ((top + slack > 224 * torch.exp2(e)) | (e == -126)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_and_nan(dtype):
    """Inf and NaN in the operands come out where the formula puts them, and nowhere else."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    for M, K, N in [(5, 48, 40), (150, 264, 270)]:
        say("infinities", M, K, N, dtype)
        x, w, b, r, z, dz, y, by = linear_case(M, K, N, dtype, "none", False)
        x, w = x.clone(), w.clone()
        x[1, 3], x[2, 5], w[7, 11] = math.inf, math.nan, -math.inf
        x[3, :] = 3e38
        w[:, 13] = 2.0 ** -120
        z = x.double() @ w.double() + b.double()
        z = torch.where(z.abs() > 3.4e38, torch.sign(z) * math.inf, z)
        fin = torch.nan_to_num(x.double(), nan=0, posinf=0, neginf=0).abs() @ torch.nan_to_num(
            w.double(), nan=0, posinf=0, neginf=0).abs()
        keep = torch.ones(M, dtype=torch.bool)
        keep[3] = False            # its sums overflow or not by the order of the terms
        got = whtmix.linear(x.to(dev), w.to(dev), b.to(dev))
        bound = ref.sum_bound(K, fin + b.double().abs()) + ref.rounded(
            torch.nan_to_num(z, nan=0, posinf=0, neginf=0), dtype == "bf16")
        ref.check("y", got[keep.to(dev)], z[keep], bound[keep])
        # a column of the weights far below the splits' range, times the large row
        ref.check("tiny", got[3:4, 13:14], z[3:4, 13:14], bound[3:4, 13:14])
        x[3, :] = 1
        dy = draw(77, M, N, dtype=dt)
        dx, dw, db = whtmix.linear_backward(x.to(dev), w.to(dev), dy.to(dev))
        assert torch.isnan(dw[5]).all() and torch.isinf(dw[3]).all()
        rest = [k for k in range(K) if k not in (3, 5)]
        X, D = x.double()[:, rest], dy.double()
        ref.check("dw", dw[rest], X.t() @ D, ref.sum_bound(M, X.abs().t() @ D.abs())
                  + ref.rounded(X.t() @ D, dtype == "bf16"))
        assert torch.isfinite(db).all()
        assert torch.isinf(dx[:, 7]).all() and torch.isfinite(dx[:, rest[:3]]).all()


def test_float32_operands_that_do_not_split():
    """Rows of very small and very large float32 values keep float32's accuracy."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    M, K, N = 140, 96, 136
    say("do not split")
    for sx, sw in [(2.0 ** -110, 2.0 ** 60), (2.0 ** 127, 2.0 ** -60), (2.0 ** 50, 2.0 ** -115)]:
        x, w = draw(1, M, K).clamp(-1.9, 1.9) * sx, draw(2, K, N).clamp(-1.9, 1.9) * sw
        z = x.double() @ w.double()
        y = whtmix.linear(x.to(dev), w.to(dev))
        ref.check(f"{sx:g} {sw:g}", y, z, ref.sum_bound(K, x.double().abs() @ w.double().abs())
                  + 2.0 ** -140)


def test_rows_of_a_wider_tensor():
    """x as columns of a wider tensor, in three dimensions too."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    for dt in (torch.float32, torch.bfloat16):
        wide = draw(1, 4, 9, 200, dtype=dt).to(dev)
        w, b, g = draw(2, 72, 40, dtype=dt).to(dev), draw(3, 40).to(dev), draw(4, 72).to(dev)
        dy = draw(5, 4, 9, 40, dtype=dt).to(dev)
        for at in (0, 8, 101):
            x = wide[:, :, at:at + 72]
            c = x.contiguous()
            assert torch.equal(whtmix.linear(x, w, b), whtmix.linear(c, w, b))
            assert torch.equal(whtmix.norm(x, g)[0], whtmix.norm(c, g)[0])
            for u, v in zip(whtmix.quantize_mx(x), whtmix.quantize_mx(c)):
                assert torch.equal(u.view(torch.uint8), v.view(torch.uint8))
            for u, v in zip(whtmix.linear_backward(x, w, dy), whtmix.linear_backward(c, w, dy)):
                assert torch.equal(u, v)


def test_no_rows():
    from paper_2607_25234_amd import whtmix
    dev = device()
    for dt in (torch.float32, torch.bfloat16):
        x, w = torch.empty(0, 24, dtype=dt, device=dev), draw(1, 24, 40, dtype=dt).to(dev)
        g = draw(2, 24).to(dev)
        assert whtmix.norm(x, g, x)[0].shape == (0, 24)
        assert whtmix.linear(x, w).shape == (0, 40)
        dx, dw = whtmix.norm_backward(x, g, x)
        assert dx.shape == (0, 24) and not dw.any()
        dx, dw, db = whtmix.linear_backward(x, w, torch.empty(0, 40, dtype=dt, device=dev))
        assert dx.shape == (0, 24) and not dw.any() and not db.any()
        q, s = whtmix.quantize_mx(x)
        assert q.shape == (0, 32) and whtmix.dequantize_mx(q, s, 24).shape == (0, 24)


def test_large_offsets():
    """Offsets past 2^31 elements: the last rows of a bf16 tensor of 2.2 G elements."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    rows, C = 34_000, 65_536
    x = torch.zeros(rows, C, dtype=torch.bfloat16, device=dev)
    x[-3:] = draw(1, 3, C, dtype=torch.bfloat16).to(dev)
    g = (1 + draw(2, C, std=0.1)).to(dev)
    w = draw(3, C, 24, std=C ** -0.5, dtype=torch.bfloat16).to(dev)
    y, _ = whtmix.norm(x, g, out=x.clone())
    small, _ = whtmix.norm(x[-3:].contiguous(), g)
    assert torch.equal(y[-3:], small) and not y[:-3].any()
    del y
    o = whtmix.linear(x, w)
    assert not o[:-3].any()
    z = x[-3:].cpu().double() @ w.cpu().double()
    ref.check("linear", o[-3:], z,
              ref.sum_bound(C, x[-3:].cpu().double().abs() @ w.cpu().double().abs())
              + ref.rounded(z, True))


def test_streams_and_repeats():
    """Calls on another stream, and the same bits every time."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    x = draw(1, 3000, 136, dtype=torch.bfloat16).to(dev)
    w = draw(2, 136, 200, dtype=torch.bfloat16).to(dev)
    dy, g = draw(3, 3000, 200, dtype=torch.bfloat16).to(dev), draw(4, 136).to(dev)

    def calls():
        return (*whtmix.linear_backward(x, w, dy), whtmix.linear(x, w),
                *whtmix.norm_backward(x, g, x))

    torch.cuda.synchronize()
    first = calls()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = calls()
    side.synchronize()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, calls()):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_layer():
    """The layer's training step and its served form against the same steps in 64 bits."""
    from paper_2607_25234_amd.layer import MixerLayer, MixerLayerMx
    import numpy as np
    from oracle import oracle
    dev = device()
    torch.manual_seed(0)
    B, N, C, H = 2, 100, 64, 256
    layer = MixerLayer(N, C, H, dtype=torch.float32, device=dev)
    with torch.no_grad():
        for p in (layer.log_gain_tokens, layer.log_gain_channels, layer.b1, layer.b2):
            p.add_(torch.randn_like(p) * 0.1)
        layer.norm_weight.add_(torch.randn_like(layer.norm_weight) * 0.1)
    x = draw(1, B, N, C)
    y = layer(x.to(dev))
    p = {k: v.detach().cpu().double() for k, v in layer.named_parameters()}
    mixed = torch.from_numpy(np.asarray(oracle.default().whtmix_module_separable(
        x.numpy(), p["w_in"].float().numpy(), p["log_gain_tokens"].float().numpy(),
        p["log_gain_channels"].float().numpy(), p["w_out"].float().numpy()))).double()
    h = x.double() + mixed.reshape(B, N, C)
    n = h / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt() * p["norm_weight"]
    u = ref.act("gelu", n @ p["w1"] + p["b1"])
    r = h + u @ p["w2"] + p["b2"]
    assert float((y.detach().cpu().double() - r).norm() / r.norm()) <= 1e-5
    y.square().sum().backward()
    for name, q in layer.named_parameters():
        assert q.grad is not None and torch.isfinite(q.grad).all() and q.grad.abs().sum() > 0, name
    served = MixerLayerMx(layer)(x.to(dev)).cpu().double()
    # 8 bits: each operand's values are off by 2^-4 / sqrt(12) or so of themselves at most
    assert float((served - r).norm() / (r - h).norm()) <= 0.1
