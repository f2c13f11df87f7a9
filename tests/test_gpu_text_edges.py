"""GPU tests of layer norm, gated products and embedding where a small error would not show beside
the bounds of random rows: exact sums, calls that go round the grid, joined stretches."""
from __future__ import annotations

import pytest
import torch

from tests import layer_ref as ref
from tests import text_ref
from tests.gpu_util import device, say
from tests.test_gpu_layer import DTYPES, draw

pytestmark = pytest.mark.gpu


# ---- layer norm: the mean ----

def exact_rows(C, rows=6):
    """(large, small), both [rows, C] and their sum exact in bf16, with a known mean far below the
    last bit of the large values: up to 16 pairs v, -v of multiples of 1/2 in [64, 128), and 8
    multiples of 2^-13 that come to an odd one below 2^-6; zeros elsewhere, the columns from C / 2
    on among them.  Every partial sum is a multiple of 2^-13 below 2^11, which float32 holds: the
    row's sum is exact in any order."""
    g = torch.Generator().manual_seed(C)
    pairs = min(16, max(1, C // 64))
    large, small = torch.zeros(rows, C), torch.zeros(rows, C)
    for r in range(rows):
        at = torch.randperm(C // 2, generator=g)
        v = torch.randint(128, 256, (pairs,), generator=g) / 2
        large[r, at[:pairs]], large[r, at[pairs:2 * pairs]] = v, -v
        k = torch.randint(-60, 61, (8,), generator=g)
        k[7] = 2 * r + 71 - k[:7].sum()
        while k[7].abs() > 250:
            k[:7] = torch.randint(-20, 21, (7,), generator=g)
            k[7] = 2 * r + 71 - k[:7].sum()
        small[r, at[2 * pairs:2 * pairs + 8]] = k * 2.0 ** -13
    assert torch.equal(large + small, (large + small).bfloat16().float())
    return large, small


EXACT = [64, 1111, 2048, 4096, 8192, 40000]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", EXACT)
@pytest.mark.parametrize("res", [False, True])
def test_layer_norm_mean_of_exact_sums(C, dtype, res):
    """Where t is 0 the output is -mean * rstd * w, which nothing but the mean's own error can move: with
    an exact sum the mean is off by its division, 1 U of it, rstd by 4 U (the squares' sum, the
    division by C, the root) and the products by 2 U."""
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    say("exact_mean", C, dtype, res)
    large, small = exact_rows(C)
    t = large + small
    x, r = (large, small) if res else (t, None)
    w = 1 + draw(2, C, std=0.1)
    T = t.double()
    mu = T.mean(-1, keepdim=True)
    want = -mu * ((T - mu).square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w.double()
    zero = t == 0
    args = (x.to(dt).to(dev), w.to(dev), None, None if r is None else r.to(dt).to(dev))
    y, _ = whtmix.layer_norm(*args)
    off = (y.cpu().double() - want).abs()
    assert bool((off <= want.abs() * 8 * ref.U + ref.rounded(want, bf))[zero].all()), \
        float((off / want.abs())[zero].max())
    q, s, _ = whtmix.layer_norm_mx(*args)
    got = whtmix.dequantize_mx(q, s, C, torch.float32).cpu().double()
    first = (C // 2 + 31) // 32 * 32        # whole blocks of such values: e4m3's normal numbers
    off = ((got - want).abs() / want.abs())[:, first:]
    assert float(off.max()) <= 2.0 ** -4 + 8 * ref.U


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", EXACT)
def test_layer_norm_backward_mean_of_exact_sums(C, dtype):
    """The weight's gradient of the columns from C / 2 on is the sum over rows of -dy mean rstd: each
    term off by 8 U as above and the sum by 1 U of the terms' magnitudes a row."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("exact_mean_backward", C, dtype)
    large, small = exact_rows(C)
    h, dy, w = (large + small).to(dt), draw(3, *large.shape, dtype=dt), 1 + draw(2, C, std=0.1)
    _, dw, _ = whtmix.layer_norm_backward(h.to(dev), w.to(dev), dy.to(dev))
    T = h.double()
    mu = T.mean(-1, keepdim=True)
    terms = -dy.double() * mu * ((T - mu).square().mean(-1, keepdim=True) + 1e-6).rsqrt()
    off = (dw.cpu().double() - terms.sum(0)).abs()
    ok = off <= (8 + h.shape[0]) * ref.U * terms.abs().sum(0)
    assert bool(ok[C // 2:].all()), float((off / terms.abs().sum(0))[C // 2:].max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [64, 1111, 4096, 40000])
def test_layer_norm_of_the_largest_spread(C, dtype):
    """Distances all over a row at 0.97 of the bound 2^64 / sqrt(C), about 0 and about a mean
    of 64 times as much, whose own squares overflow."""
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    say("largest", C, dtype)
    sign = torch.where(torch.arange(C) % 2 == 0, 1.0, -1.0)
    sign = sign.repeat(4, 1)[:, torch.randperm(C, generator=torch.Generator().manual_seed(C))]
    a = 2.0 ** 64 / C ** 0.5 * 0.97
    if bf:      # whole steps of the mean's type too
        step = 2.0 ** (int(torch.tensor(a).log2().floor()) - 1)
        a = a // step * step
    mean = torch.tensor([0.0, 0.0, 64.0, -64.0])[:, None] * 2.0 ** int(torch.tensor(a).log2().floor())
    x = (mean + a * sign).to(dt)
    w, b = 1 + draw(2, C, std=0.1), draw(5, C, std=0.3)
    y, _ = whtmix.layer_norm(x.to(dev), w.to(dev), b.to(dev))
    want, bound, _ = text_ref.layer_norm(x, None, w, b, 1e-6)
    ref.check("y", y, want, bound + ref.rounded(want, bf))
    dy = draw(3, 4, C, dtype=dt)
    dx, dw, db = whtmix.layer_norm_backward(x.to(dev), w.to(dev), dy.to(dev))
    rx, bx, rw, bw, rb, bb = text_ref.layer_norm_backward(x, w, dy, None, 1e-6)
    ref.check("dx", dx, rx, bx + ref.rounded(rx, bf))
    ref.check("dweight", dw, rw, bw)
    ref.check("dbias", db, rb, bb)


# More rows than twice as many as the device holds at a time, the last round of them partial: each
# workgroup goes on from row to row with the next one on its way.
ROUNDS = [(2000, 4096, "bf16"), (2500, 1111, "f32"), (3200, 2048, "bf16"), (7000, 1024, "bf16"),
          (14001, 512, "bf16"), (27001, 250, "bf16"), (52003, 40, "f32"), (101003, 61, "bf16")]


@pytest.mark.parametrize("rows,C,dtype", ROUNDS)
@pytest.mark.parametrize("res", [False, True])
def test_layer_norm_round_the_grid(rows, C, dtype, res):
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    say("round_the_grid", rows, C, dtype, res)
    x, w, b = draw(1, rows, C, dtype=dt) + 0.5, 1 + draw(2, C, std=0.1), draw(5, C, std=0.3)
    r = draw(3, rows, C, std=2.0, dtype=dt) if res else None
    want, bound, t = text_ref.layer_norm(x, r, w, b, 1e-6)
    own = ref.rounded(t, bf) + (x.double().abs() + t.abs()) * 2 * ref.U

    def given():
        return x.to(dev), w.to(dev), b.to(dev), None if r is None else r.to(dev)

    y, h = whtmix.layer_norm(*given())
    ref.check("y", y, want, bound + ref.rounded(want, bf))
    ref.check("h", h, t, own)
    # y in x's place, and h in x's or the residual's, while later rows are on their way
    args = given()
    z, _ = whtmix.layer_norm(*args, out=args[0])
    assert z is args[0] and torch.equal(z, y)
    for at in (0, 3) if res else (0,):
        args = given()
        z = torch.empty_like(y)
        p = [0 if a is None else a.data_ptr() for a in args]
        assert whtmix.call_rows("whtmix_layer_norm_forward",
                                (p[0], p[3], p[1], p[2], z.data_ptr(), p[at]), (rows, C, C),
                                (whtmix.DTYPE_BF16 if bf else whtmix.DTYPE_F32,),
                                torch.cuda.current_stream().cuda_stream, 1e-6) == 0
        assert torch.equal(z, y) and torch.equal(args[at], h)
    # in 8 bits: the rounding's half step besides, of the block's scale below its normal numbers
    q, s, h8 = whtmix.layer_norm_mx(*given())
    assert torch.equal(h8, h)
    got = whtmix.dequantize_mx(q, s, C, torch.float32)
    last = s.cpu().double().sub(127).exp2().repeat_interleave(32, -1)[:, :C] * 2.0 ** -9
    ref.check("8 bits", got, want, bound + torch.maximum((want.abs() + bound) * 2.0 ** -4, last / 2))


# ---- gated products ----

@pytest.mark.parametrize("M,K,N,act", [(32768, 128, 64, "silu"), (49161, 97, 344, "gelu"),
                                       (49300, 128, 520, "relu")])
def test_gated_backward_of_frozen_weights(M, K, N, act):
    """Without the weights' gradients the pass of dzg, dzu and dx leaves those two out; dx and the
    biases' gradients are those of the whole call."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), torch.bfloat16
    say("gated_backward_frozen", M, K, N, act)
    x, wg, wu = (draw(s, *shape, dtype=dt).to(dev) for s, shape in
                 ((1, (M, K)), (2, (K, N)), (3, (K, N))))
    dy, zg, zu = (draw(s, M, N, dtype=dt).to(dev) for s in (11, 12, 13))
    whole = whtmix.gated_backward(x, wg, wu, dy, zg, zu, act)
    for bias in (True, False):
        got = whtmix.gated_backward(x, wg, wu, dy, zg, zu, act, want_dw=False, want_dbias=bias)
        assert got[1] is None and got[2] is None
        assert torch.equal(got[0], whole[0])
        if bias:
            assert torch.equal(got[3], whole[3]) and torch.equal(got[4], whole[4])


@pytest.mark.parametrize("M,K,N,act", [(32768, 128, 64, "silu"), (49161, 97, 344, "gelu"),
                                       (3000, 40, 77, "gelu_tanh")])
def test_linear_backward_of_frozen_weights(M, K, N, act):
    """The same of the single product."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), torch.bfloat16
    say("linear_backward_frozen", M, K, N, act)
    x, w, dy, z = (draw(s, *shape, dtype=dt).to(dev) for s, shape in
                   ((1, (M, K)), (2, (K, N)), (11, (M, N)), (12, (M, N))))
    whole = whtmix.linear_backward(x, w, dy, z, act)
    for dx in (True, False):
        for bias in (True, False):
            if dx or bias:
                got = whtmix.linear_backward(x, w, dy, z, act, want_dx=dx, want_dw=False,
                                             want_dbias=bias)
                assert got[1] is None
                if dx:
                    assert torch.equal(got[0], whole[0])
                if dx and bias:
                    assert torch.equal(got[2], whole[2])
                elif bias:      # the sums' order may be another
                    want = (dy.double() * ref.act_grad(act, z.double())).sum(0)
                    mag = (dy.double() * ref.act_grad(act, z.double())).abs().sum(0)
                    bound = ref.sum_bound(M, mag) + (dy.double().abs()
                                                     * ref.grad_bound(act, z.double())).sum(0)
                    ref.check("dbias", got[2], want.cpu(), bound.cpu())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("want", ["dx", "dw", "dbias"])
def test_products_backward_without_rows(dtype, want):
    """Each gradient alone of no rows: one of no rows, or zeros."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    x, dy = torch.empty(0, 24, dtype=dt, device=dev), torch.empty(0, 40, dtype=dt, device=dev)
    w = draw(1, 24, 40, dtype=dt).to(dev)
    wants = {"want_" + k: k == want for k in ("dx", "dw", "dbias")}
    got = (*whtmix.linear_backward(x, w, dy, **wants),
           *whtmix.gated_backward(x, w, w, dy, dy, dy, **wants))
    shapes = [{"dx": (0, 24), "dw": (24, 40), "dbias": (40,)}[k]
              for k in ("dx", "dw", "dbias", "dx", "dw", "dw", "dbias", "dbias")]
    kinds = ["dx", "dw", "dbias", "dx", "dw", "dw", "dbias", "dbias"]
    for g, shape, kind in zip(got, shapes, kinds):
        assert (g is None) is (kind != want)
        assert g is None or (g.shape == shape and not g.any())


# ---- embedding ----

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,C", [(20000, 600, 64), (70001, 5000, 8), (30000, 3, 1000),
                                      (9000, 256, 64), (50000, 200, 33)])
def test_embedding_gradient_of_long_runs(rows, V, C, dtype):
    """Runs over many stretches, workgroups and ranges: an id of half of the tokens, one of an eighth,
    and the rest.  Small whole numbers: float32 holds every partial sum, so the result is the
    sum in any order, rounded once."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("long_runs", rows, V, C, dtype)
    g = torch.Generator().manual_seed(rows)
    ids, u = torch.randint(-1, V, (rows,), generator=g), torch.rand(rows, generator=g)
    ids[u < 0.5] = V // 2
    ids[u > 0.875] = V - 1
    dy = torch.randint(-8, 9, (rows, C), generator=g)
    want = torch.zeros(V + 1, C, dtype=torch.int64).index_add_(0, ids % (V + 1), dy)[:V]
    assert int(dy.abs().sum(0).max()) < 1 << 24
    got = whtmix.embedding_backward(ids.to(dev), dy.to(dt).to(dev), V)
    assert torch.equal(got.cpu(), want.to(dt))
