"""GPU tests of layer norm, gated products and embedding against the 64-bit reference."""
from __future__ import annotations

import math

import pytest
import torch

from tests import layer_ref as ref
from tests import text_ref
from tests.gpu_util import device, say
from tests.test_gpu_layer import DTYPES, LINEAR_SHAPES, MX_SHAPES, NORM_SHAPES, draw

pytestmark = pytest.mark.gpu


# ---- layer norm ----

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", NORM_SHAPES)
@pytest.mark.parametrize("res", [False, True])
def test_layer_norm(rows, C, dtype, res):
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    say("layer_norm", rows, C, dtype, res)
    x, w = draw(1, rows, C, dtype=dt) + 0.5, 1 + draw(2, C, std=0.1)
    b = draw(5, C, std=0.3) if (rows + C) % 3 else None
    r = draw(3, rows, C, std=2.0, dtype=dt) if res else None
    y, h = whtmix.layer_norm(x.to(dev), w.to(dev), None if b is None else b.to(dev),
                             r.to(dev) if res else None, eps=1e-5)
    want, bound, t = text_ref.layer_norm(x, r, w, b, 1e-5)
    ref.check("y", y, want, bound + ref.rounded(want, bf))
    ref.check("h", h, t, ref.rounded(t, bf) + (x.double().abs() + t.abs()) * 2 * ref.U)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [5, 64, 300, 4096, 20000])
@pytest.mark.parametrize("mean", [300.0, -1e4, 1e6])
def test_layer_norm_of_a_large_mean(C, dtype, mean):
    """Rows whose spread is far below their mean, and rows without any."""
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    say("large_mean", C, dtype, mean)
    x = (mean + draw(1, 6, C, std=abs(mean) * 2.0 ** -6)).to(dt)
    x[2:4] = mean
    w, b = 1 + draw(2, C, std=0.1), draw(5, C, std=0.3)
    dy = draw(3, 6, C, dtype=dt)
    y, _ = whtmix.layer_norm(x.to(dev), w.to(dev), b.to(dev), eps=1e-3)
    want, bound, _ = text_ref.layer_norm(x, None, w, b, 1e-3)
    ref.check("y", y, want, bound + ref.rounded(want, bf))
    dx, dw, db = whtmix.layer_norm_backward(x.to(dev), w.to(dev), dy.to(dev), eps=1e-3)
    rx, bx, rw, bw, rb, bb = text_ref.layer_norm_backward(x, w, dy, None, 1e-3)
    ref.check("dx", dx, rx, bx + ref.rounded(rx, bf))
    ref.check("dw", dw, rw, bw)
    ref.check("db", db, rb, bb)


BACKWARD_SHAPES = NORM_SHAPES + [(1000, 128), (5000, 48), (2049, 520), (4000, 2048), (1300, 9000),
                                 (3001, 1023), (1000, 16384)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", BACKWARD_SHAPES)
@pytest.mark.parametrize("res", [False, True])
def test_layer_norm_backward(rows, C, dtype, res):
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    say("layer_norm_backward", rows, C, dtype, res)
    h, w = draw(1, rows, C, dtype=dt) - 0.5, 1 + draw(2, C, std=0.1)
    dy = draw(3, rows, C, dtype=dt)
    dh = draw(4, rows, C, dtype=dt) if res else None
    args = h.to(dev), w.to(dev), dy.to(dev), dh.to(dev) if res else None
    dx, dw, db = whtmix.layer_norm_backward(*args, eps=1e-5)
    rx, bx, rw, bw, rb, bb = text_ref.layer_norm_backward(h, w, dy, dh, 1e-5)
    ref.check("dx", dx, rx, bx + ref.rounded(rx, bf))
    ref.check("dw", dw, rw, bw)
    ref.check("db", db, rb, bb)
    for a, b in ((False, False), (True, False), (False, True)):
        one = whtmix.layer_norm_backward(*args, eps=1e-5, want_dweight=a, want_dbias=b)
        assert torch.equal(one[0], dx)
        assert torch.equal(one[1], dw) if a else one[1] is None
        assert torch.equal(one[2], db) if b else one[2] is None
    for onto in (2, 3) if res else (2,):        # dx in dy's or dh's place
        own = [t.clone() if t is not None else None for t in args]
        assert torch.equal(whtmix.layer_norm_backward(*own, eps=1e-5, dx=own[onto])[0], dx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", [(1, 1), (5, 33), (17, 64), (130, 128), (3, 1111), (2, 4096),
                                    (2, 8200), (3, 33000), (2, 70001)])
def test_layer_norm_mx(rows, C, dtype):
    """As test_norm_mx: each value a nearest e4m3 value of the norm in 64 bits, each block's
    scale the definition's or, where its maximum is at a limit within the error, a neighbour's."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("layer_norm_mx", rows, C, dtype)
    x, w, r = draw(1, rows, C, dtype=dt), 1 + draw(2, C, std=0.1), draw(3, rows, C, dtype=dt)
    b = draw(4, C, std=0.3)
    q, s, h = whtmix.layer_norm_mx(x.to(dev), w.to(dev), b.to(dev), r.to(dev), eps=1e-5)
    y, own, t = text_ref.layer_norm(x, r, w, b, 1e-5)
    assert q.shape == (rows, whtmix.mx_width(C)) and not q.cpu().float()[:, C:].any()
    pad = (0, -C % 32)
    top = torch.nn.functional.pad(y.abs(), pad).reshape(rows, -1, 32).amax(-1)
    slack = torch.nn.functional.pad(own, pad).reshape(rows, -1, 32).amax(-1)
    e = s.cpu().double() - 127
    assert (top - slack <= 448 * torch.exp2(e)).all()
    assert ((top + slack > 224 * torch.exp2(e)) | (e == -126)).all()
    unit = torch.exp2(e).repeat_interleave(32, -1)[:, :C]
    v = whtmix.dequantize_mx(q, s, C, torch.float32)
    step = torch.maximum(torch.exp2(torch.floor(torch.log2((y / unit).abs().clamp(min=1e-30)))
                                    - 3), torch.full_like(y, 2.0 ** -9)) * unit
    ref.check("q", v, y, step * 0.5 * (1 + 1e-6) + own)
    ref.check("h", h, t, ref.rounded(t, dtype == "bf16") + 2 * ref.U * t.abs())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_rows_apart(dtype):
    """Inf and NaN stay in their row (and in the columns' sums); y in x's place; columns of a
    wider tensor."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    for rows, C in ((5, 40), (6, 520), (5, 20000)):
        say("rows_apart", rows, C, dtype)
        x, r = draw(1, rows, C, dtype=dt).to(dev), draw(2, rows, C, dtype=dt).to(dev)
        w, b = draw(3, C).to(dev), draw(4, C).to(dev)
        want, kept = whtmix.layer_norm(x, w, b, r)
        bad = x.clone()
        bad[1, 3], bad[2, C - 1], bad[4, 0] = math.nan, math.inf, -math.inf
        y, _ = whtmix.layer_norm(bad, w, b, r)
        assert torch.isnan(y[[1, 2, 4]]).all() and torch.equal(y[[0, 3]], want[[0, 3]])
        dx = whtmix.layer_norm_backward(bad, w, r)[0]
        assert torch.isnan(dx[[1, 2, 4]]).all()
        assert torch.equal(dx[[0, 3]], whtmix.layer_norm_backward(x, w, r)[0][[0, 3]])
        for res in (None, r):
            y = x.clone()
            out, h = whtmix.layer_norm(y, w, b, res, out=y)
            assert out is y and torch.equal(y, whtmix.layer_norm(x, w, b, res)[0])
            assert h is None if res is None else torch.equal(h, kept)
        wide = torch.zeros(rows, C + 13, dtype=dt, device=dev)
        wide[:, 5:C + 5] = x
        assert torch.equal(whtmix.layer_norm(wide[:, 5:C + 5], w, b, r)[0], want)
        assert whtmix.layer_norm(x[:0], w, b)[0].shape == (0, C)
        dx, dw, db = whtmix.layer_norm_backward(x[:0], w, r[:0])
        assert dx.shape == (0, C) and not dw.any() and not db.any()


# ---- gated products ----

GATED_SHAPES = LINEAR_SHAPES + [(40, 100, 1000), (2000, 200, 72), (700, 136, 344)]


def gated_case(M, K, N, dtype, seed=1):
    dt = DTYPES[dtype]
    x = draw(seed, M, K, dtype=dt)
    wg, wu = (draw(seed + i, K, N, std=K ** -0.5, dtype=dt) for i in (1, 2))
    bg, bu = (draw(seed + i, N, std=0.3) if (M + i) % 4 else None for i in (3, 4))
    return x, wg, wu, bg, bu


def to(dev, *ts):
    return [None if t is None else t.to(dev) for t in ts]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", GATED_SHAPES)
def test_gated(M, K, N, dtype):
    from paper_2607_25234_amd import whtmix
    dev, bf = device(), dtype == "bf16"
    act = ref.ACTS[(M + K + N) % 5]
    say("gated", M, K, N, dtype, act)
    case = gated_case(M, K, N, dtype)
    args = to(dev, *case)
    y, zg, zu = whtmix.gated(*args, act, want_z=True)
    ry, by, rg, ru, bg, bu = text_ref.gated(*case, act)
    ref.check("y", y, ry, by + ref.rounded(ry, bf))
    ref.check("zg", zg, rg, bg + ref.rounded(rg, bf))
    ref.check("zu", zu, ru, bu + ref.rounded(ru, bf))
    out = torch.empty_like(y)
    assert whtmix.gated(*args, act, out=out) is out and torch.equal(out, y)     # the same with no z


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", GATED_SHAPES + [(20000, 64, 96), (9000, 40, 264)])
def test_gated_backward(M, K, N, dtype):
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    act = ref.ACTS[(M + K + N) % 5]
    say("gated_backward", M, K, N, dtype, act)
    x, wg, wu, _, _ = gated_case(M, K, N, dtype)
    dy, zg, zu = (draw(s, M, N, std=std, dtype=dt) for s, std in ((11, 1.0), (12, 2.0), (13, 2.0)))
    args = *to(dev, x, wg, wu, dy, zg, zu), act
    got = whtmix.gated_backward(*args)
    want = text_ref.gated_backward(x, wg, wu, dy, zg, zu, act, bf)
    for i, (name, g, (r, b)) in enumerate(zip(("dx", "dwg", "dwu", "dbg", "dbu"), got, want)):
        ref.check(name, g, r, b + (ref.rounded(r, bf) if i < 3 else 0))
    for which in range(3):      # each alone is the same
        one = whtmix.gated_backward(*args, want_dx=which == 0, want_dw=which == 1,
                                    want_dbias=which == 2)
        for i, (a, b) in enumerate(zip(one, got)):
            assert torch.equal(a, b) if (i + 1) // 2 == which else a is None


@pytest.mark.parametrize("M,K,N,act", [
    (49152, 128, 520, "silu"), (49151, 128, 520, "silu"), (49200, 60, 1024, "none"),
    (49153, 16, 1032, "gelu"), (49155, 7, 272, "relu"), (32769, 128, 256, "gelu_tanh"),
    (32767, 128, 256, "gelu"), (32768, 1, 64, "gelu"), (49300, 129, 344, "silu"),
    (49163, 90, 343, "relu")])
def test_gated_backward_of_many_rows(M, K, N, act):
    """dz, its sums and dx in one pass over the rows or apart: sizes at and beside the rule's, with
    rows and columns of dx that end inside a tile and N that ends inside a step."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), torch.bfloat16
    say("gated_backward_many", M, K, N, act)
    x, wg, wu, _, _ = gated_case(M, K, N, "bf16")
    dy, zg, zu = (draw(s, M, N, std=std, dtype=dt) for s, std in ((11, 1.0), (12, 2.0), (13, 2.0)))
    args = *to(dev, x, wg, wu, dy, zg, zu), act
    got = whtmix.gated_backward(*args)
    want = text_ref.gated_backward(x, wg, wu, dy, zg, zu, act, True)
    names = "dx", "dwg", "dwu", "dbg", "dbu"
    for i, (name, g, (r, b)) in enumerate(zip(names, got, want)):
        ref.check(name, g, r, b + (ref.rounded(r, True) if i < 3 else 0))
    again = whtmix.gated_backward(*args)
    assert all(torch.equal(a, b) for a, b in zip(again, got))
    for which in range(3):      # each alone: the sums' order may be another
        one = whtmix.gated_backward(*args, want_dx=which == 0, want_dw=which == 1,
                                    want_dbias=which == 2)
        for i, (name, g, (r, b)) in enumerate(zip(names, one, want)):
            if (i + 1) // 2 != which:
                assert g is None
            else:
                ref.check(name, g, r, b + (ref.rounded(r, True) if i < 3 else 0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(4096, 264, 1600), (2100, 520, 1601), (4100, 128, 344),
                                   (3001, 400, 2003)])
def test_gated_on_large_tiles(M, K, N, dtype):
    """Tiles of 256 x 256 forward and backward, and float32 operands split in a pass of their own;
    N at and beside the columns of a tile and of a step."""
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    say("gated_large", M, K, N, dtype)
    case = gated_case(M, K, N, dtype)
    x, wg, wu, _, _ = case
    y, zg, zu = whtmix.gated(*to(dev, *case), "silu", want_z=True)
    ry, by, rg, ru, bg, bu = text_ref.gated(*case, "silu")
    ref.check("y", y, ry, by + ref.rounded(ry, bf))
    ref.check("zg", zg, rg, bg + ref.rounded(rg, bf))
    ref.check("zu", zu, ru, bu + ref.rounded(ru, bf))
    dy = draw(11, M, N, dtype=dt)
    got = whtmix.gated_backward(*to(dev, x, wg, wu, dy), zg, zu, "silu")
    want = text_ref.gated_backward(x, wg, wu, dy, zg.cpu(), zu.cpu(), "silu", bf)
    for i, (name, g, (r, b)) in enumerate(zip(("dx", "dwg", "dwu", "dbg", "dbu"), got, want)):
        ref.check(name, g, r, b + (ref.rounded(r, bf) if i < 3 else 0))


@pytest.mark.parametrize("M,K,N", [(3001, 400, 4006), (2880, 130, 4090)])
def test_float32_products_in_tiles_of_192_rows(M, K, N):
    """Rows that 256 leave units idle with; the last tile goes past the operands' padding."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    say("192_rows", M, K, N)
    x, w = draw(1, M, K), draw(2, K, N, std=K ** -0.5)
    z = x.double() @ w.double()
    bound = ref.sum_bound(K, x.double().abs() @ w.double().abs())
    ref.check("z", whtmix.linear(x.to(dev), w.to(dev)), z, bound)
    x[M - 1], x[7] = x[M - 1] * 2.0 ** -110, x[7] * 2.0 ** -110      # rows that do not split
    w = w * 2.0 ** 40
    z = x.double() @ w.double()
    bound = ref.sum_bound(K, x.double().abs() @ w.double().abs())
    ref.check("tiny", whtmix.linear(x.to(dev), w.to(dev)), z, bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ref.ACTS)
def test_gated_activations(dtype, act):
    """Every activation over its range, against both signs of the other factor."""
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    say("gated_activations", dtype, act)
    M, K, N = 40, 8, 272
    x, wg, wu = torch.zeros(M, K), torch.zeros(K, N), torch.zeros(K, N)
    x[:, 0], x[:, 1] = torch.linspace(-3, 3, M), 1
    wg[0], wg[1] = torch.linspace(-20, 20, N), torch.linspace(-60, 60, N).roll(N // 2)
    wu[0], wu[1] = 1, torch.linspace(-2, 2, N)
    x, wg, wu = x.to(dt), wg.to(dt), wu.to(dt)
    y, zg, zu = whtmix.gated(*to(dev, x, wg, wu), activation=act, want_z=True)
    ry, by, *_ = text_ref.gated(x, wg, wu, None, None, act)
    ref.check("y", y, ry, by + ref.rounded(ry, bf) + 1e-30)
    dy = draw(9, M, N, dtype=dt)
    got = whtmix.gated_backward(*to(dev, x, wg, wu, dy), zg, zu, act)
    want = text_ref.gated_backward(x, wg, wu, dy, zg.cpu(), zu.cpu(), act, bf)
    for i, (g, (r, b)) in enumerate(zip(got, want)):
        ref.check(f"{i}", g, r, b + (ref.rounded(r, bf) if i < 3 else 0) + 1e-30)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(5, 48, 40), (150, 264, 270), (300, 300, 300)])
def test_gated_infinities_and_nan(M, K, N, dtype):
    """Inf and NaN of one weight reach its column (and row of the gradients) alone."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("gated_infinities", M, K, N, dtype)
    x, wg, wu, bg, bu = gated_case(M, K, N, dtype)
    clean = whtmix.gated(*to(dev, x, wg, wu, bg, bu), "silu")
    wg, wu = wg.clone(), wu.clone()
    wg[7, 11], wu[3, 5], wu[2, 9] = math.nan, math.inf, -math.inf
    y = whtmix.gated(*to(dev, x, wg, wu, bg, bu), "silu").cpu()
    rest = [n for n in range(N) if n not in (11, 5, 9)]
    assert torch.isnan(y[:, 11]).all() and not torch.isfinite(y[:, [5, 9]]).any()
    d = (y[:, rest].double() - clean.cpu()[:, rest].double()).abs()
    # other columns of a float32 tile may be formed by float32 products instead
    assert (d <= clean.cpu()[:, rest].double().abs() * 1e-3 + 1e-4).all()
    dy, zg, zu = (draw(s, M, N, dtype=dt) for s in (11, 12, 13))
    dx = whtmix.gated_backward(*to(dev, x, wg, wu, dy, zg, zu), "silu", want_dw=False,
                               want_dbias=False)[0].cpu()
    assert torch.isnan(dx[:, 7]).all() and not torch.isfinite(dx[:, [3, 2]]).any()
    assert torch.isfinite(dx[:, [k for k in range(K) if k not in (7, 3, 2)]]).all()
    x = x.clone()
    x[1, 4] = math.inf
    dwg, dwu = whtmix.gated_backward(*to(dev, x, wg, wu, dy, zg, zu), "silu", want_dx=False,
                                     want_dbias=False)[1:3]
    for dw in (dwg.cpu(), dwu.cpu()):
        assert not torch.isfinite(dw[4]).any()
        assert torch.isfinite(dw[[k for k in range(K) if k != 4]]).all()


def test_gated_float32_tiny_columns():
    """Columns of either weight far below what three bf16 terms hold, times large rows."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    for M, K, N in ((9, 72, 40), (50, 96, 136), (140, 96, 136), (1000, 640, 700)):
        say("gated_tiny", M, K, N)
        x, wg, wu, _, _ = gated_case(M, K, N, "f32")
        wg[:, 5] *= 2.0 ** -120
        wu[:, 6] *= 2.0 ** -120
        x = x * 2.0 ** 60
        y, zg, zu = whtmix.gated(*to(dev, x, wg, wu), activation="none", want_z=True)
        _, _, rg, ru, bg, bu = text_ref.gated(x, wg, wu, None, None, "none")
        ref.check("zg", zg, rg, bg + ref.rounded(rg, False))
        ref.check("zu", zu, ru, bu + ref.rounded(ru, False))


@pytest.mark.parametrize("out", ["bf16", "f32", "mx"])
@pytest.mark.parametrize("M,K,N", MX_SHAPES)
def test_gated_mx(M, K, N, out):
    from paper_2607_25234_amd import whtmix
    dev = device()
    act = ref.ACTS[(M + K + N) % 5]
    say("gated_mx", M, K, N, out, act)
    scale = torch.exp2(torch.arange(M) % 7 - 3.0)[:, None]
    xq, xs = whtmix.quantize_mx((draw(1, M, K) * scale).to(dev))
    g8, u8 = (whtmix.quantize_mx(draw(s, N, K, std=K ** -0.5).to(dev)) for s in (2, 3))
    x, wg, wu = (whtmix.dequantize_mx(*t, K, torch.float32).cpu() for t in ((xq, xs), g8, u8))
    b = draw(4, N, std=0.3), (draw(5, N, std=0.3) if M % 2 else None)
    y, by, *_ = text_ref.gated(x, wg.t(), wu.t(), *b, act)
    args = xq, xs, *g8, *u8, *to(dev, *b), act
    if out != "mx":
        got = whtmix.gated_mx(*args, dtype=DTYPES[out])
        assert got.dtype is DTYPES[out]
        ref.check("y", got, y, by + ref.rounded(y, out == "bf16"))
        again = torch.empty_like(got)
        assert whtmix.gated_mx(*args, out=again) is again and torch.equal(again, got)
        return
    q, s = whtmix.gated_mx(*args, out_mx=True)
    assert q.shape == (M, whtmix.mx_width(N)) and not q.cpu().float()[:, N:].any()
    e = s.cpu().double() - 127
    unit = torch.exp2(e).repeat_interleave(32, -1)[:, :N]
    v = whtmix.dequantize_mx(q, s, N, torch.float32)
    step = torch.maximum(torch.exp2(torch.floor(torch.log2((y / unit).abs().clamp(min=1e-30)))
                                    - 3), torch.full_like(y, 2.0 ** -9)) * unit
    ref.check("q", v, y, step * 0.5 * (1 + 1e-6) + 2 * by)
    top = torch.nn.functional.pad(y.abs(), (0, -N % 32)).reshape(M, -1, 32).amax(-1)
    slack = torch.nn.functional.pad(by, (0, -N % 32)).reshape(M, -1, 32).amax(-1)
    assert (top - slack <= 448 * torch.exp2(e)).all()
    assert ((top + slack > 224 * torch.exp2(e)) | (e == -126)).all()


def test_gated_rows_and_views():
    """No rows; columns of a wider tensor; odd addresses of every operand."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    for dt in (torch.float32, torch.bfloat16):
        say("gated_views", dt)
        wide = draw(1, 4, 9, 200, dtype=dt).to(dev)
        K, N = 72, 40
        wg, wu = (draw(s, K, N, dtype=dt).to(dev) for s in (2, 3))
        dy, zg, zu = (draw(s, 4, 9, N, dtype=dt).to(dev) for s in (4, 5, 6))
        for at in (0, 8, 101):
            x = wide[:, :, at:at + K]
            c = x.contiguous()
            assert torch.equal(whtmix.gated(x, wg, wu), whtmix.gated(c, wg, wu))
            for u, v in zip(whtmix.gated_backward(x, wg, wu, dy, zg, zu),
                            whtmix.gated_backward(c, wg, wu, dy, zg, zu)):
                assert torch.equal(u, v)
        x = wide[..., :K].contiguous()

        def moved(t):       # the same values, one element further on
            s = torch.empty(t.numel() + 1, dtype=t.dtype, device=dev)[1:].view(t.shape)
            return s.copy_(t)

        y, want = whtmix.gated(x, wg, wu), whtmix.gated_backward(x, wg, wu, dy, zg, zu)
        for i in range(6):
            p = [moved(t) if i == j else t for j, t in enumerate((x, wg, wu, dy, zg, zu))]
            assert torch.equal(whtmix.gated(*p[:3]), y)
            for u, v in zip(whtmix.gated_backward(*p), want):
                assert torch.equal(u, v)
        none = torch.empty(0, K, dtype=dt, device=dev), torch.empty(0, N, dtype=dt, device=dev)
        assert whtmix.gated(none[0], wg, wu).shape == (0, N)
        dx, *rest = whtmix.gated_backward(none[0], wg, wu, none[1], none[1], none[1])
        assert dx.shape == (0, K) and not any(t.any() for t in rest)


@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
def test_gradients_against_differences(act):
    """The kernels' gradients through embedding, layer norm and gated product against central
    differences of their own forward pass along a random direction (step 2^-6: its square
    times the third derivative, and the forward's float32 error over it, are below 1e-3 of the
    gradient's norm times the direction's)."""
    from paper_2607_25234_amd import autograd
    dev = device()
    M, V, K, N = 37, 19, 72, 41
    say("differences", act)
    ids = torch.randint(-1, V, (M,), generator=torch.Generator().manual_seed(0)).to(dev)
    p = [draw(0, V, K), draw(2, M, K), 1 + draw(3, K, std=0.1), draw(9, K, std=0.1),
         draw(4, K, N, std=K ** -0.5), draw(8, K, N, std=K ** -0.5), draw(5, N, std=0.1),
         draw(16, N, std=0.1)]
    dy, dh = draw(6, M, N).to(dev), draw(7, M, K).to(dev)

    def loss(table, r, g, b, wg, wu, bg, bu):
        x = autograd.whtmix_embedding(ids, table, 1.25)
        y, h = autograd.whtmix_layer_norm(x, g, b, r, 1e-5)
        o = autograd.whtmix_gated(y, wg, wu, bg, bu, act)
        return (o.double() * dy.double()).sum() + (h.double() * dh.double()).sum()

    leaf = [t.to(dev).requires_grad_() for t in p]
    loss(*leaf).backward()
    e = 2.0 ** -6
    for i, t in enumerate(p):
        v = draw(20 + i, *t.shape)
        v /= v.norm()
        with torch.no_grad():
            up, down = ([s.to(dev) + (k * e * v.to(dev) if j == i else 0)
                         for j, s in enumerate(p)] for k in (1, -1))
            num = float((loss(*up) - loss(*down)) / (2 * e))
        g = leaf[i].grad.double().cpu()
        assert abs(float((g * v.double()).sum()) - num) <= 1e-3 * float(g.norm()), i


# ---- embedding ----

def token_ids(kind, rows, V, seed=0):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(V, (rows,), generator=g)
    if kind == "padded":
        ids[torch.rand(rows, generator=g) < 0.3] = -1
    elif kind == "one":
        ids[:] = V // 2
    elif kind == "runs":        # long runs, in falling order
        ids = (V - 1 - torch.arange(rows) * max(1, min(V, 7)) // rows).clamp(min=0)
    elif kind == "none":
        ids[:] = -7
    elif kind == "skewed":      # half of them one token
        ids[torch.rand(rows, generator=g) < 0.5] = V - 1
    elif kind == "outside":
        ids[torch.rand(rows, generator=g) < 0.2] = V
        ids[:1] = 1 << 30
    return ids


KINDS = ["uniform", "padded", "one", "runs", "none", "skewed", "outside"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,C", [(1, 1, 1), (1, 300, 4096), (17, 131, 33), (64, 256, 64),
                                      (1000, 7, 100), (300, 70000, 8), (4097, 600, 520),
                                      (3, 5, 9001)])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_embedding(rows, V, C, dtype, index):
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    table = draw(1, V, C, dtype=dt)
    for kind in ("uniform", "padded", "outside"):
        say("embedding", rows, V, C, dtype, index, kind)
        ids = token_ids(kind, rows, V).to(index)
        for scale in (1.0, -3.7):
            y = whtmix.embedding(ids.to(dev), table.to(dev), scale)
            want = text_ref.embedding(ids, table, scale)
            # scale is rounded to float32, then the product, then the value
            ref.check(kind, y, want, ref.rounded(torch.nan_to_num(want), bf)
                      + 2 * ref.U * torch.nan_to_num(want).abs())
        if scale == 1.0:
            assert torch.equal(y, table.to(dev)[ids.to(dev)])
    ids = token_ids("uniform", rows, V).to(index).to(dev)
    out = torch.empty(rows, 1, C, dtype=dt, device=dev)
    assert whtmix.embedding(ids[:, None], table.to(dev), out=out) is out
    assert torch.equal(out[:, 0], table.to(dev)[ids.long()])


# rows: a token, ranges and tiles and one beside them, several tiles, more tiles than are
# added up without a pass of their own
EMBED_SHAPES = [(1, 1, 1), (1, 5000, 40), (7, 3, 5), (8, 256, 64), (9, 256, 64), (63, 40, 100),
                (1000, 2, 72), (4096, 256, 64), (4097, 255, 33), (12000, 511, 24), (12001, 512, 24),
                (20000, 70000, 16), (9000, 300000, 8), (5000, 50, 1032), (40, 9, 9001),
                (131072, 256, 64), (600000, 700, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,C", EMBED_SHAPES)
def test_embedding_backward(rows, V, C, dtype):
    from paper_2607_25234_amd import whtmix
    dev, dt, bf = device(), DTYPES[dtype], dtype == "bf16"
    dy = draw(3, rows, C, dtype=dt)
    for i, kind in enumerate(KINDS):
        index = torch.int32 if (rows + i) % 2 else torch.int64
        say("embedding_backward", rows, V, C, dtype, kind, index)
        ids = token_ids(kind, rows, V).to(index)
        scale = 0.3 if i % 2 else 1.0
        got = whtmix.embedding_backward(ids.to(dev), dy.to(dev), V, scale)
        want, bound = text_ref.embedding_backward(ids, dy, V, scale, bf)
        ref.check(kind, got, want, bound)
        assert torch.equal(got, whtmix.embedding_backward(ids.to(dev), dy.to(dev), V, scale))
        one = torch.bincount(ids[(ids >= 0) & (ids < V)].long(), minlength=V) == 1
        if scale == 1.0 and one.any():      # a token's only row, as it is
            at = torch.nonzero(one[ids.long().clamp(0, V - 1)] & (ids >= 0) & (ids < V))[:, 0]
            assert torch.equal(got.cpu()[ids[at].long()], dy[at])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,C", [(2048, 100, 16), (2049, 100, 16), (2048, 256, 64), (1025, 256, 32),
                                      (2500, 256, 128), (2500, 257, 128), (2500, 200, 129),
                                      (2500, 511, 64), (2500, 512, 64), (196608, 256, 128),
                                      (196609, 256, 128), (262144, 256, 128),
                                      (262145, 256, 128), (70000, 3, 1)])
def test_embedding_backward_of_few_ids(rows, V, C, dtype):
    """At and beside the sizes that choose between the tiles' sums and the whole sort."""
    from paper_2607_25234_amd import whtmix
    dev, bf = device(), dtype == "bf16"
    say("embedding_few", rows, V, C, dtype)
    gen = torch.Generator().manual_seed(rows + V + C)
    ids = torch.randint(-1, V + 1, (rows,), generator=gen)      # padding and one past the table
    ids[rows // 3: rows // 2] = V // 2                          # a long run
    dy = draw(3, rows, C, dtype=DTYPES[dtype])
    got = whtmix.embedding_backward(ids.to(dev), dy.to(dev), V, 0.5)
    want, bound = text_ref.embedding_backward(ids, dy, V, 0.5, bf)
    ref.check("dtable", got, want, bound)
    assert torch.equal(got, whtmix.embedding_backward(ids.to(dev), dy.to(dev), V, 0.5))


def test_embedding_order_of_sums():
    """Equal tokens are added in ascending order: 2^24 and then ones, which do not add to it, and
    as many rows of its negative, leave exactly the ones after it."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    say("order")
    dy = torch.ones(8, 4)
    dy[2], dy[5] = 2.0 ** 25, -2.0 ** 25
    ids = torch.tensor([3, 1, 3, 3, 1, 3, 3, 3], dtype=torch.int32)
    g = whtmix.embedding_backward(ids.to(dev), dy.to(dev), 4).cpu()
    assert torch.equal(g[3], torch.full((4,), 2.0)) and torch.equal(g[1], torch.full((4,), 2.0))
    assert not g[[0, 2]].any()


def test_embedding_nothing():
    from paper_2607_25234_amd import whtmix
    dev = device()
    for dt in (torch.float32, torch.bfloat16):
        ids = torch.empty(0, 5, dtype=torch.int64, device=dev)
        table = draw(1, 37, 19, dtype=dt).to(dev)
        assert whtmix.embedding(ids, table).shape == (0, 5, 19)
        g = whtmix.embedding_backward(ids, torch.empty(0, 5, 19, dtype=dt, device=dev), 37)
        assert g.shape == (37, 19) and not g.any()


def test_embedding_infinities():
    """Inf and NaN in a row of the gradient reach its token alone; padding's reach none."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    for dt in (torch.float32, torch.bfloat16):
        say("embedding_infinities", dt)
        ids = torch.randint(5, (500,), generator=torch.Generator().manual_seed(0))
        ids[10], ids[200], ids[300] = 3, -1, -1
        dy = draw(1, 500, 40, dtype=dt)
        clean = whtmix.embedding_backward(ids.to(dev), dy.to(dev), 5)
        dy[10], dy[200], dy[300] = math.nan, math.inf, math.nan
        g = whtmix.embedding_backward(ids.to(dev), dy.to(dev), 5)
        assert torch.isnan(g[3]).all()
        assert torch.equal(g[[0, 1, 2, 4]], clean[[0, 1, 2, 4]])


def test_embedding_large_offsets():
    """A table of 2.7 G elements, and tokens from its end; as many elements of y."""
    from paper_2607_25234_amd import whtmix
    dev, bf = device(), torch.bfloat16
    say("embedding_large")
    V, C = 42_000_000, 64
    table = torch.zeros(V, C, dtype=bf, device=dev)
    last = draw(1, 5, C, dtype=bf).to(dev)
    table[-5:] = last
    ids = torch.tensor([V - 1, 0, V - 5, V - 3, V - 1, V], device=dev)
    y = whtmix.embedding(ids, table)
    assert torch.equal(y[[0, 2, 3, 4]], last[[4, 0, 2, 4]]) and not y[1].any()
    assert torch.isnan(y[5]).all()
    del table
    dy = draw(2, 6, C, dtype=bf).to(dev)
    g = whtmix.embedding_backward(ids, dy, V)
    assert torch.equal(g[V - 5], dy[2]) and torch.equal(g[V - 3], dy[3])
    assert torch.equal(g[V - 1], (dy[0].float() + dy[4].float()).to(bf))
    g[[0, V - 5, V - 3, V - 1]] = 0
    assert int(torch.count_nonzero(g)) == 0
    del g
    many = torch.arange(V, device=dev, dtype=torch.int32) % 3
    y = whtmix.embedding(many, last[:3].contiguous())
    assert torch.equal(y[-3:], last[:3]) and torch.equal(y[1_000_002:1_000_005], last[:3])


# ---- as a program uses them ----

def all_calls(ids, table, dy, w, b, wg, wu, g8, u8):
    from paper_2607_25234_amd import whtmix
    e = whtmix.embedding(ids, table, 2.0)
    n, h = whtmix.layer_norm(e, w, b, dy)
    u, zg, zu = whtmix.gated(n, wg, wu, activation="silu", want_z=True)
    dn, dwg, dwu, dbg, dbu = whtmix.gated_backward(n, wg, wu, u, zg, zu, "silu")
    dh, dw, db = whtmix.layer_norm_backward(h, w, dn, dy)
    dt = whtmix.embedding_backward(ids, dh, table.shape[0], 2.0)
    q, s, k = whtmix.layer_norm_mx(e, w, b, dy)
    v = whtmix.gated_mx(q, s, *g8, *u8, activation="gelu")
    q, s = whtmix.gated_mx(q, s, *g8, *u8, activation="gelu", out_mx=True)
    return [e, n, h, u, zg, zu, dn, dwg, dwu, dbg, dbu, dh, dw, db, dt, k, v, q.view(torch.uint8), s]


def program(dev, dt, M, V, C, N, seed=0):
    from paper_2607_25234_amd import whtmix
    ids = token_ids("padded", M, V, seed).to(dev)
    w, b = 1 + draw(seed + 1, C, std=0.1).to(dev), draw(seed + 2, C, std=0.1).to(dev)
    wg, wu = (draw(seed + s, C, N, std=C ** -0.5, dtype=dt).to(dev) for s in (3, 4))
    g8, u8 = (whtmix.quantize_mx(t.t().contiguous()) for t in (wg, wu))
    return [ids, draw(seed + 5, V, C, dtype=dt).to(dev), draw(seed + 6, M, C, dtype=dt).to(dev),
            w, b, wg, wu, g8, u8]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ordinary_calls_and_the_others(dtype, monkeypatch):
    """Calls that the module on torch tensors takes give what the Python way does, and it takes
    them; those that are not ordinary go the Python way, which raises or takes them."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("ordinary", dtype)
    m = whtmix._ordinary()
    assert not isinstance(m, whtmix._NotBuilt)
    args = program(dev, dt, 300, 50, 264, 344)
    ids, table, dy, w, b, wg, wu, g8, u8 = args
    dy3 = dy.reshape(3, 100, 264)
    bg = torch.randn(344, device=dev)
    fast = all_calls(*args)
    more = [whtmix.layer_norm(dy3, w, None)[0], whtmix.layer_norm_mx(dy3, w)[0].view(torch.uint8),
            *whtmix.gated(dy3, wg, wu, bg, None, "gelu", want_z=True),
            whtmix.embedding(ids.reshape(3, 100).to(torch.int32), table),
            whtmix.embedding(ids[7], table)]
    kept = whtmix.layer_norm(torch.nn.Parameter(dy), w)
    assert whtmix.layer_norm(dy, w)[1] is dy and whtmix.layer_norm_mx(dy, w)[2] is dy
    taken = []
    monkeypatch.setattr(whtmix, "_ordinary_module", whtmix._NotBuilt())
    for x, y in zip(fast, all_calls(*args)):
        assert torch.equal(x, y) and x.dtype == y.dtype
    slow = [whtmix.layer_norm(dy3, w, None)[0], whtmix.layer_norm_mx(dy3, w)[0].view(torch.uint8),
            *whtmix.gated(dy3, wg, wu, bg, None, "gelu", want_z=True),
            whtmix.embedding(ids.reshape(3, 100).to(torch.int32), table),
            whtmix.embedding(ids[7], table)]
    for x, y in zip(more, slow):
        assert torch.equal(x, y) and x.shape == y.shape
    assert torch.equal(kept[0], whtmix.layer_norm(dy, w)[0])
    for name in ("layer_norm", "layer_norm_mx"):
        f = getattr(m, name)
        assert f(dy, w, b, dy, 1e-6) is not None
        for bad in ((dy[:, :8], w[:8], None, None, 1e-6), (dy, w[:8], b, None, 1e-6),
                    (dy, w.to(torch.bfloat16), b, None, 1e-6), (dy.double(), w, b, None, 1e-6),
                    (dy, w, b, dy3, 1e-6), (dy[0], w, b, None, 1e-6), (dy.cpu(), w, b, None, 1e-6),
                    (dy, w.cpu(), b, None, 1e-6), (dy[:0], w, b, dy[:0], 1e-6),
                    (dy, None, b, None, 1e-6), (None, w, b, None, 1e-6),
                    (dy.t(), w, b, None, 1e-6)):
            assert f(*bad) is None, (name, len(taken))
            taken.append(bad)
        assert f(dy, w, b, dy, -1.0) == 1 and f(dy, w, b, dy, math.nan) == 1     # a status
        with pytest.raises(TypeError):
            f(dy, w, b, dy)
        with pytest.raises(TypeError):
            f(dy, w, b, dy, "eps")
    assert m.gated(dy, wg, wu[:, :8], None, None, 4, False) is None
    assert m.gated(dy, wg[0], wu, None, None, 4, False) is None
    assert m.gated(dy, wg, wu, None, None, 9, False) == 1
    assert m.gated_backward(dy, wg, wu, dy, dy, dy, 4, True, True, True) is None
    assert m.gated_mx(dy, w, *g8, *u8, None, None, 4, False) is None
    assert m.embedding(ids.float(), table, 1.0) is None and m.embedding(ids, w, 1.0) is None
    assert m.embedding(ids, table, math.inf) == 1
    assert m.embedding_backward(ids, dy, 0, 1.0) is None
    assert m.embedding_backward(ids[:7], dy, 50, 1.0) is None
    monkeypatch.setattr(whtmix, "_ordinary_module", m)
    for f in (lambda: whtmix.layer_norm(dy, w, eps=-1.0), lambda: whtmix.embedding(ids, table, math.nan),
              lambda: whtmix.embedding_backward(ids, dy, 0)):
        with pytest.raises(whtmix.WhtmixError):
            f()
    with pytest.raises(ValueError):
        whtmix.gated(dy, wg, wu, activation="tanh")
    with pytest.raises(ValueError):
        whtmix.gated(dy, wg, wu[:, :8])
    with pytest.raises(ValueError):
        whtmix.embedding_backward(ids[:7], dy, 50)
    with pytest.raises(TypeError):
        whtmix.embedding(ids.float(), table)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,C,N", [(300, 50, 264, 344), (9000, 700, 64, 172), (49300, 200, 64, 344)])
def test_streams_repeats_and_graph_replays(M, V, C, N, dtype):
    """The same bits every time, on another stream, and from a graph captured on a stream whose
    workspace earlier calls sized, replayed on new inputs with eager work between."""
    dev, dt = device(), DTYPES[dtype]
    say("replays", M, V, C, N, dtype)
    args = program(dev, dt, M, V, C, N)
    first = all_calls(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = all_calls(*args)
    torch.cuda.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = all_calls(*args)
    for k in range(4):
        args[0].copy_(token_ids(KINDS[k % 4], M, V, k))
        args[1].copy_(draw(30 + k, V, C, dtype=dt))
        args[2].copy_(draw(40 + k, M, C, dtype=dt))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for i, (a, b) in enumerate(zip(got, all_calls(*args))):
            assert torch.equal(a, b), (k, i)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,C,N", [(300, 50, 264, 343), (9000, 700, 64, 172), (49300, 200, 64, 344),
                                     (3001, 130, 400, 1003)])
def test_after_a_call_full_of_nan(M, V, C, N, dtype):
    """What a call leaves in the workspace reaches no other call: the same bits after one whose
    intermediate values are all NaN."""
    dev, dt = device(), DTYPES[dtype]
    say("after_nan", M, V, C, N, dtype)
    args = program(dev, dt, M, V, C, N)
    first = all_calls(*args)
    bad = [args[0].clamp(min=0), *(torch.full_like(t, float("nan")) for t in args[1:7]), *args[7:]]
    assert all(t.isnan().all() for t in all_calls(*bad)[:14])
    for i, (a, b) in enumerate(zip(all_calls(*args), first)):
        assert torch.equal(a, b), i


def test_two_threads():
    """Two host threads, each on a stream of its own, get what one gets alone."""
    import threading
    dev = device()
    say("two_threads")
    cases = [program(dev, torch.bfloat16, 700, 40, 136, 200),
             program(dev, torch.float32, 5000, 3000, 72, 130, 50)]
    alone = [all_calls(*c) for c in cases]
    torch.cuda.synchronize()
    wrong = []

    def run(c, want):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(15):
                    got = all_calls(*c)
                    stream.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want)):
                        wrong.append("other bits")
        except Exception as e:      # told to the test's own thread
            wrong.append(repr(e))

    threads = [threading.Thread(target=run, args=a) for a in zip(cases, alone)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong


def hadamard(n):
    h = torch.ones(1, 1, dtype=torch.float64)
    while h.shape[0] < n:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h / math.sqrt(n)


# As for the layer alone: every tensor that a bf16 layer holds is rounded by up to 2^-8 of itself,
# ten of them forward and fourteen backward, here with both products' results of the gate (two
# more forward, four backward), two layers and the embedding.  float32: 1e-5 a layer.
@pytest.mark.parametrize("dtype,forward,backward", [("f32", 2e-5, 2e-5),
                                                    ("bf16", 25 * 2.0 ** -8, 37 * 2.0 ** -8)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_text_and_its_gradients(dtype, forward, backward, norm):
    """MixerText's output and every gradient, and each of its layers served in 8 bits, against
    the model written out in 64 bits."""
    from paper_2607_25234_amd.layer import MixerLayerMx, MixerText
    dev, dt = device(), DTYPES[dtype]
    torch.manual_seed(0)
    B, N, C, H, V = 2, 100, 64, 172, 50
    say("text", dtype, norm)
    model = MixerText(V, N, C, H, 2, dtype=dt, device=dev, norm=norm, gated=True,
                      activation="silu")
    with torch.no_grad():
        for name, p in model.named_parameters():
            if p.dtype == torch.float32 and p.dim() == 1:
                p.add_(torch.randn_like(p) * 0.1)
    ids = token_ids("padded", B * N, V).reshape(B, N)
    dy = draw(2, B, N, C, dtype=dt)
    y = model(ids.to(dev))
    y.backward(dy.to(dev))

    p = {k: v.detach().cpu().double().requires_grad_() for k, v in model.named_parameters()}
    ht, hc = hadamard(128), hadamard(C)
    x = p["table"][ids.clamp(min=0)] * (ids >= 0)[..., None] * C ** 0.5
    for i in range(2):
        q = {k[len(f"layers.{i}."):]: v for k, v in p.items() if k.startswith(f"layers.{i}.")}
        u = torch.nn.functional.pad(x @ q["w_in"], (0, 0, 0, 28))
        gain = torch.exp(q["log_gain_tokens"])[:, None] * torch.exp(q["log_gain_channels"])
        h = x + (ht @ (gain * (ht @ u @ hc)) @ hc)[:, :N] @ q["w_out"]
        d = h - h.mean(-1, keepdim=True) if norm == "layer" else h
        n = d / (d.square().mean(-1, keepdim=True) + 1e-6).sqrt() * q["norm_weight"]
        if norm == "layer":
            n = n + q["norm_bias"]
        f = ref.act("silu", n @ q["w1"] + q["b1"]) * (n @ q["w_up"] + q["b_up"])
        f = f @ q["w2"] + q["b2"]
        x_in, x = x, h + f
    x.backward(dy.double())

    def off(name, got, want, tol):
        err = float((got.detach().cpu().double() - want).norm() / want.norm())
        say(f"  {name}: {err:.2e} of {tol:.2e}")
        assert err <= tol, (name, err)

    off("y", y, x.detach(), forward)
    for name, q in model.named_parameters():
        assert q.grad.dtype == q.dtype
        off("d " + name, q.grad, p[name].grad, backward)
    # 8 bits: each operand's values are off by 2^-4 / sqrt(12) or so of themselves at most
    served = MixerLayerMx(model.layers[1])(x_in.detach().to(dt).to(dev))
    assert served.dtype is dt
    off("served", served, x.detach(),
        float(0.1 * f.detach().norm() / x.detach().norm()) + forward)
