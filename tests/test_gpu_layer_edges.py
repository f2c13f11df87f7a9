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


# gemm_kernel's tiles of 32, 64 and 128 rows: float32 operands split on their way
@pytest.mark.parametrize("M,K,N", [(9, 72, 40), (50, 96, 136), (140, 96, 136), (300, 200, 133)])
def test_float32_tiny_columns_among_others(M, K, N):
    """A column of w (and of x and dy, for dw; a row of w, for dx) far below what three bf16 terms
    hold, among normal ones: its sums, which a large other operand brings back to the normal
    range, keep float32's accuracy."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    say("tiny_columns", M, K, N)
    for e in (-112, -120, -124):
        x, w, dy = draw(1, M, K), draw(2, K, N), draw(3, M, N)
        tiny = w.clone()
        tiny[:, 5] *= 2.0 ** e
        tiny[7] *= 2.0 ** e
        big = x * 2.0 ** 60
        z = big.double() @ tiny.double()
        y = whtmix.linear(big.to(dev), tiny.to(dev))
        ref.check("z", y, z, ref.sum_bound(K, big.double().abs() @ tiny.double().abs()))
        dx = whtmix.linear_backward(x.to(dev), tiny.to(dev), (dy * 2.0 ** 60).to(dev),
                                    want_dw=False, want_dbias=False)[0]
        d = dy.double() * 2.0 ** 60
        ref.check("dx", dx, d @ tiny.double().t(),
                  ref.sum_bound(N, d.abs() @ tiny.double().abs().t()))
        for of_x in (True, False):
            a, b = (x.clone(), dy * 2.0 ** 60) if of_x else (big, dy.clone())
            (a if of_x else b)[:, 6] *= 2.0 ** e
            dw = whtmix.linear_backward(a.to(dev), w.to(dev), b.to(dev), want_dx=False,
                                        want_dbias=False)[1]
            a, b = a.double(), b.double()
            ref.check(f"dw {of_x}", dw, a.t() @ b, ref.sum_bound(M, a.abs().t() @ b.abs()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("M", [2, 32768])
def test_derivatives_at_large_values(M, dtype, act):
    """Every derivative at finite values up to the type's largest: 1 above zero and 0 below, from
    where float32 does not tell them apart.  (Many rows of narrow bf16 inputs take the pass
    that forms dz and dx together.)"""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("large_values", M, dtype, act)
    at = [200.0, 512.0, 1e3, 1e10, 1.9e19, 4.5e19, 1e20, 3e38]
    z = torch.tensor([s * v for v in at for s in (1, -1)] * 4).repeat(M, 1).to(dt)
    K, N = 4, z.shape[1]
    x, w, dy = (torch.ones(s, dtype=dt) for s in ((M, K), (K, N), (M, N)))
    w[:, 1::2] = 2
    dx, dw, db = whtmix.linear_backward(x.to(dev), w.to(dev), dy.to(dev),
                                        None if act == "none" else z.to(dev), act)
    d = (z > 0).double() if act != "none" else dy.double()
    assert torch.equal(db.cpu().double(), d.sum(0))
    assert torch.equal(dw.cpu().double(), (x.double().t() @ d).to(dt).double())
    assert torch.equal(dx.cpu().double(), d @ w.double().t())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_in_place(dtype):
    """y in x's place: with a residual h is a tensor of its own, without one x is gone."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    for rows, C in ((1, 7), (9, 520), (3, 20000)):
        say("norm_in_place", rows, C, dtype)
        x, r = draw(1, rows, C, dtype=dt).to(dev), draw(2, rows, C, dtype=dt).to(dev)
        w = draw(3, C).to(dev)
        for res in (None, r):
            want, kept = whtmix.norm(x, w, res)
            y = x.clone()
            out, h = whtmix.norm(y, w, res, out=y)
            assert out is y and torch.equal(y, want)
            assert h is None if res is None else torch.equal(h, kept)
        other = torch.empty_like(x)
        assert torch.equal(whtmix.norm(x, w, out=other)[1], x)


def test_no_rows_zeros_gradients_of_any_size():
    """M = 0: dw and dbias are zeros to the last element and nothing around them is written,
    from any alignment and past the 2^32 threads that one launch holds (8.6 GB of dw)."""
    from paper_2607_25234_amd import whtmix
    dev = device()
    for dt, code in ((torch.float32, 0), (torch.bfloat16, 1)):
        for K, N in ((1, 1), (3, 5), (1, 8), (7, 33), (65, 4099)):
            for at in (0, 1, 2, 5, 7):
                say("no_rows", dt, K, N, at)
                t = torch.ones(K * N + 32, dtype=dt, device=dev)
                b = torch.ones(N + 8, device=dev)
                status = whtmix.call_rows(
                    "whtmix_linear_backward",
                    (0, 0, 0, 0, 0, t[at:].data_ptr(), b[1:].data_ptr()), (0, K, N, K), (0, code),
                    torch.cuda.current_stream().cuda_stream)
                assert status == 0
                assert t[:at].all() and not t[at:at + K * N].any() and t[at + K * N:].all()
                assert b[0] == 1 and not b[1:N + 1].any() and b[N + 1:].all()
    K, N = (1 << 16) + 3, 1 << 15
    say("no_rows", K, N)
    t = torch.ones(K * N + 8, device=dev)
    assert whtmix.call_rows("whtmix_linear_backward", (0, 0, 0, 0, 0, t[1:].data_ptr(), 0),
                            (0, K, N, K), (0, 0), torch.cuda.current_stream().cuda_stream) == 0
    assert int(torch.count_nonzero(t)) == 8 and t[0] == 1 and t[-7:].all()


@pytest.mark.parametrize("M,K,N,act", [(49152, 128, 520, "gelu"), (49200, 60, 1024, "silu"),
                                       (49155, 7, 272, "gelu_tanh"), (32769, 128, 256, "relu"),
                                       (49151, 16, 264, "silu"), (50001, 9, 1032, "relu")])
def test_narrow_backward_on_both_sides_of_its_rule(M, K, N, act):
    """dz, its sums and dx of narrow bf16 inputs: rows and columns at which they are formed in
    one pass, and the next ones, at which they are not."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), torch.bfloat16
    say("narrow_rule", M, K, N, act)
    x, w = draw(1, M, K, dtype=dt), draw(2, K, N, std=K ** -0.5, dtype=dt)
    dy, z = draw(3, M, N, dtype=dt), draw(4, M, N, std=2.0, dtype=dt)
    dx, dw, db = whtmix.linear_backward(x.to(dev), w.to(dev), dy.to(dev), z.to(dev), act)
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


def test_graph_replays():
    """The sublayer forward and backward, and its 8-bit form, captured on a stream whose workspace
    earlier calls sized, then replayed on new inputs with eager work between: every replay
    gives the eager call's bits."""
    from paper_2607_25234_amd import whtmix
    dev, bf = device(), torch.bfloat16
    say("graph_replays")
    M, C, N = 300, 264, 520
    x, r, dy = (draw(i, M, C, dtype=bf).to(dev) for i in (1, 2, 3))
    w1, w2 = draw(4, C, N, std=C ** -0.5, dtype=bf).to(dev), draw(5, N, C, std=0.04, dtype=bf).to(dev)
    f1 = w1.float()
    g, b1, b2 = 1 + draw(6, C, std=0.1).to(dev), draw(7, N).to(dev), draw(8, C).to(dev)
    q1, q2 = whtmix.quantize_mx(w1.t().contiguous()), whtmix.quantize_mx(w2.t().contiguous())

    def step():
        y, h = whtmix.norm(x, g, r)
        u, z = whtmix.linear(y, w1, b1, "gelu", want_z=True)
        o = whtmix.linear(u, w2, b2, residual=h)
        du, dw2, db2 = whtmix.linear_backward(u, w2, dy)
        dn, dw1, db1 = whtmix.linear_backward(y, w1, du, z, "gelu")
        dx, dg = whtmix.norm_backward(h, g, dn, dy)
        wide = whtmix.linear(y.float(), f1, b1, "silu")
        q, s, k = whtmix.norm_mx(x, g, r)
        q, s = whtmix.linear_mx(q, s, *q1, b1, "gelu_tanh", out_mx=True)
        return [o, dx, dg, dw1, db1, dw2, db2, wide, whtmix.linear_mx(q, s, *q2, b2, residual=k)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = step()
    for k in range(4):
        for t, seed in ((x, 20), (r, 30), (dy, 40)):
            t.copy_(draw(seed + k, M, C, dtype=bf))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", [(4000, 2048), (1000, 16384), (1300, 9000), (3001, 1023)])
def test_norm_backward_round_the_grid(rows, C, dtype):
    """Rows on several waves that go round the grid three times and more."""
    from paper_2607_25234_amd import whtmix
    dev, dt = device(), DTYPES[dtype]
    say("norm_backward_round", rows, C, dtype)
    h, w = draw(1, rows, C, dtype=dt), 1 + draw(2, C, std=0.1)
    dy, dh = draw(3, rows, C, dtype=dt), draw(4, rows, C, dtype=dt)
    dx, dw = whtmix.norm_backward(h.to(dev), w.to(dev), dy.to(dev), dh.to(dev), eps=1e-5)
    H, W, D = h.double(), w.double(), dy.double()
    rstd = 1 / (H.square().mean(-1, keepdim=True) + 1e-5).sqrt()
    n, g = H * rstd, D * W
    rx = rstd * (g - n * (g * n).mean(-1, keepdim=True)) + dh.double()
    mag = rstd * (g.abs() + n.abs() * (g * n).abs().mean(-1, keepdim=True)) + dh.double().abs()
    ref.check("dx", dx, rx, ref.sum_bound(C, mag) + ref.rounded(rx, dtype == "bf16"))
    mag = (D * n).abs().sum(0)
    ref.check("dw", dw, (D * n).sum(0), ref.sum_bound(rows, mag) + ref.sum_bound(C, mag))


def test_two_threads():
    """Two host threads, each on a stream of its own, get what one gets alone."""
    import threading
    from paper_2607_25234_amd import whtmix
    dev = device()
    say("two_threads")
    cases = []
    for i, dt in enumerate((torch.bfloat16, torch.float32)):
        M, K, N = 700 + 100 * i, 200 + 40 * i, 136
        cases.append((draw(1 + i, M, K, dtype=dt).to(dev), draw(3 + i, K, N, dtype=dt).to(dev),
                      draw(5 + i, M, N, dtype=dt).to(dev), draw(7 + i, K).to(dev)))

    def calls(x, w, dy, g):
        return (*whtmix.linear_backward(x, w, dy, dy, "silu"), whtmix.linear(x, w),
                *whtmix.norm_backward(x, g, x))

    alone = [calls(*c) for c in cases]
    torch.cuda.synchronize()
    wrong = []

    def run(c, want):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(20):
                    got = calls(*c)
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


# Each tensor a bf16 layer holds is rounded by up to 2^-8 of itself: in the forward pass the block's
# result, h, the norm's, the hidden values and the output, each passed on with a slope of up to
# 1.3 (ten of them allowed); backward du, z, dz, the norm's gradient, h, dx, the block's three and
# the sum of x's two (fourteen).  float32: 1e-5, as the mixer's own tests have it.
@pytest.mark.parametrize("dtype,forward,backward", [("f32", 1e-5, 1e-5),
                                                    ("bf16", 10 * 2.0 ** -8, 14 * 2.0 ** -8)])
def test_layer_and_its_gradients(dtype, forward, backward):
    """MixerLayer's output and every gradient, and MixerLayerMx's output, against the layer
    written out in 64 bits (dense Hadamard products)."""
    from paper_2607_25234_amd.layer import MixerLayer, MixerLayerMx
    dev, dt = device(), DTYPES[dtype]
    torch.manual_seed(0)
    B, N, C, H = 2, 100, 64, 256
    say("layer", dtype)
    layer = MixerLayer(N, C, H, dtype=dt, device=dev)
    with torch.no_grad():
        for p in (layer.log_gain_tokens, layer.log_gain_channels, layer.b1, layer.b2,
                  layer.norm_weight):
            p.add_(torch.randn_like(p) * 0.1)
    x, dy = draw(1, B, N, C, dtype=dt), draw(2, B, N, C, dtype=dt)
    xd = x.to(dev).requires_grad_()
    y = layer(xd)
    y.backward(dy.to(dev))

    p = {k: v.detach().cpu().double().requires_grad_() for k, v in layer.named_parameters()}
    X = x.double().requires_grad_()
    ht, hc = hadamard(128), hadamard(C)
    u = torch.nn.functional.pad(X @ p["w_in"], (0, 0, 0, 28))
    gain = torch.exp(p["log_gain_tokens"])[:, None] * torch.exp(p["log_gain_channels"])
    m = (ht @ (gain * (ht @ u @ hc)) @ hc)[:, :N] @ p["w_out"]
    h = X + m
    n = h / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt() * p["norm_weight"]
    f = ref.act("gelu", n @ p["w1"] + p["b1"]) @ p["w2"] + p["b2"]
    r = h + f
    r.backward(dy.double())

    def off(name, got, want, tol):
        err = float((got.detach().cpu().double() - want).norm() / want.norm())
        say(f"  {name}: {err:.2e} of {tol:.2e}")
        assert err <= tol, (name, err)

    off("y", y, r.detach(), forward)
    off("dx", xd.grad, X.grad, backward)
    for name, q in layer.named_parameters():
        assert q.grad.dtype == q.dtype
        off("d " + name, q.grad, p[name].grad, backward)
    served = MixerLayerMx(layer)(x.to(dev))
    assert served.dtype is dt
    off("served", served, r.detach(),
        float(0.1 * f.detach().norm() / r.detach().norm()) + forward)
