"""The feed-forward sublayer's Python side without a GPU: autograd wrappers and the layer with
plain torch functions in the entry points' place."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from paper_2607_25234_amd import autograd, whtmix  # noqa: E402
from tests import layer_ref as ref  # noqa: E402


def plain_norm(x, weight, residual=None, eps=1e-6):
    h = x if residual is None else x + residual
    return h * torch.rsqrt(h.square().mean(-1, keepdim=True) + eps) * weight, h


def plain_linear(x, w, bias=None, activation="none", residual=None, want_z=False):
    z = x @ w if bias is None else x @ w + bias
    y = ref.act(activation, z)
    y = y if residual is None else y + residual
    return (y, z) if want_z else y


def plain_norm_backward(h, weight, dy, dh=None, eps=1e-6, want_dweight=True):
    r = torch.rsqrt(h.square().mean(-1, keepdim=True) + eps)
    n, g = h * r, dy * weight
    dx = r * (g - n * (g * n).mean(-1, keepdim=True))
    dw = (dy * n).reshape(-1, h.shape[-1]).sum(0)
    return dx if dh is None else dx + dh, dw if want_dweight else None


def plain_linear_backward(x, w, dy, z=None, activation="none", want_dx=True, want_dw=True,
                          want_dbias=True):
    dz = dy if z is None else dy * ref.act_grad(activation, z)
    K, N = w.shape
    return (dz @ w.t() if want_dx else None,
            x.reshape(-1, K).t() @ dz.reshape(-1, N) if want_dw else None,
            dz.reshape(-1, N).sum(0) if want_dbias else None)


@pytest.fixture
def plain(monkeypatch):
    for name in ("norm", "linear", "norm_backward", "linear_backward"):
        monkeypatch.setattr(whtmix, name, globals()["plain_" + name])


def test_second_derivatives_of_the_sublayer_are_refused(plain):
    """The kernels' gradients have no graph: a second backward pass through them raises, where
    it would return the share of what else it reaches (the residual's, here) alone."""
    x = torch.randn(6, 8, dtype=torch.float64, requires_grad=True)
    w = torch.randn(8, 8, dtype=torch.float64, requires_grad=True)
    b = torch.randn(8, dtype=torch.float64, requires_grad=True)
    for f, leaves in ((lambda: autograd.whtmix_linear(x, w, b, "silu", x), (x, w, b)),
                      (lambda: autograd.whtmix_linear(x, w, b), (x, w, b)),
                      (lambda: autograd.whtmix_norm(x, b, x)[0], (x, b)),
                      (lambda: autograd.whtmix_norm(x, b)[0], (x, b))):
        for leaf in leaves:
            loss = f().square().sum() + x.pow(3).sum()
            first, = torch.autograd.grad(loss, x, create_graph=True)
            with pytest.raises(RuntimeError, match="second derivative"):
                torch.autograd.grad(first.sum() + leaf.sum(), leaf)
            with pytest.raises(RuntimeError, match="second derivative"):
                first.sum().backward()


def test_first_derivatives_are_as_before(plain):
    """With and without a graph of the gradients, the plain functions' own."""
    x, r = (torch.randn(2, 3, 8, dtype=torch.float64, requires_grad=True) for _ in range(2))
    w = torch.randn(8, 5, dtype=torch.float64, requires_grad=True)
    b = torch.randn(5, dtype=torch.float64, requires_grad=True)
    g = torch.randn(8, dtype=torch.float64, requires_grad=True)
    leaves = (x, r, w, b, g)

    def loss(norm, linear):
        y, h = norm(x, g, r)
        return (linear(y, w, b, "gelu") * torch.arange(5)).sum() + h.pow(3).sum()

    want = torch.autograd.grad(loss(plain_norm, plain_linear), leaves)
    for graph in (False, True):
        got = torch.autograd.grad(loss(autograd.whtmix_norm, autograd.whtmix_linear), leaves,
                                  create_graph=graph)
        for a, b_ in zip(got, want):
            assert torch.allclose(a, b_, rtol=1e-10, atol=1e-12)
    res = autograd.whtmix_linear(x, w, b, "none", r @ w)         # the residual's own gradient
    a, = torch.autograd.grad((res * torch.arange(5)).sum(), r)
    assert torch.allclose(a, (torch.arange(5).double() @ w.t()).expand_as(r))


def test_second_derivatives_of_the_mixer_are_refused(monkeypatch):
    """The mixer's and the block's functions likewise (entry points of the right shapes)."""
    def grads(*ts):
        return tuple(torch.ones_like(t) for t in ts)

    for name, f in {
            "forward": lambda x, g: x * g,
            "backward": lambda x, dy, g, **k: grads(x, g),
            "forward_separable": lambda x, a, b: x * a[:, None] * b,
            "backward_separable": lambda x, dy, a, b, **k: grads(x, a, b),
            "module_forward": lambda x, i, g, o: x * g,
            "module_backward": lambda x, i, g, o, dy, **k: grads(x, i, o, g),
            "module_forward_separable": lambda x, i, a, b, o: x * a[:, None] * b,
            "module_backward_separable":
                lambda x, i, a, b, o, dy, **k: grads(x, i, o, a, b)}.items():
        monkeypatch.setattr(whtmix, name, f)
    x, g = (torch.randn(4, 8, requires_grad=True) for _ in range(2))
    a, b = (torch.randn(n, requires_grad=True) for n in (4, 8))
    i, o = (torch.randn(8, 8, requires_grad=True) for _ in range(2))
    for y, leaves in ((autograd.whtmix_mix(x, g), (x, g)),
                      (autograd.whtmix_mix_separable(x, a, b), (x, a, b)),
                      (autograd.whtmix_block(x, i, g, o), (x, i, g, o)),
                      (autograd.whtmix_block_separable(x, i, a, b, o), (x, i, a, b, o))):
        for leaf in leaves:
            first, = torch.autograd.grad(y.square().sum() + x.pow(3).sum(), x, create_graph=True)
            with pytest.raises(RuntimeError, match="second derivative"):
                torch.autograd.grad(first.sum() + leaf.sum(), leaf)
        first = torch.autograd.grad(y.sum(), leaves)
        assert all(torch.equal(f, torch.ones_like(t)) for f, t in zip(first, leaves))


def test_dtype_codes_before_torch_is_published(monkeypatch):
    """A thread that finds torch imported finds the element types' codes too."""
    seen = []

    class Codes(dict):
        def update(self, *a, **k):
            seen.append(whtmix._torch_module)
            super().update(*a, **k)

    monkeypatch.setattr(whtmix, "_torch_module", None)
    monkeypatch.setattr(whtmix, "_CODES", Codes())
    assert whtmix._torch() is torch and whtmix._torch_module is torch
    assert seen == [None] and whtmix._CODES[torch.bfloat16] == whtmix.DTYPE_BF16


def test_served_layer_keeps_the_weights_it_was_made_of(plain, monkeypatch):
    """MixerLayerMx is of one state of the layer, whatever becomes of the layer afterwards."""
    from paper_2607_25234_amd.layer import MixerLayer, MixerLayerMx
    monkeypatch.setattr(whtmix, "quantize_mx", lambda x: (x.clone(), None))
    monkeypatch.setattr(whtmix, "module_forward_separable",
                        lambda x, i, a, b, o: (x @ i) * (a[:, None] + 1) * (b + 1) @ o)
    monkeypatch.setattr(whtmix, "norm_mx", lambda x, w, r, eps: (
        (n := plain_norm(x, w, r, eps))[0], None, n[1]))
    monkeypatch.setattr(whtmix, "linear_mx", lambda q, s, w, ws, b, act="none", residual=None,
                        out_mx=False: (y := plain_linear(q, w.t(), b, act, residual),
                                       None) if out_mx else plain_linear(q, w.t(), b, act, residual))
    torch.manual_seed(0)
    layer = MixerLayer(4, 8, 16, dtype=torch.float32)
    x = torch.randn(2, 4, 8)
    served = MixerLayerMx(layer)
    want = served(x)
    for p in layer.parameters():
        with torch.no_grad():
            p.add_(torch.randn_like(p))
    assert torch.equal(served(x), want)
    assert not torch.equal(MixerLayerMx(layer)(x), want)


def test_rows_of_any_strides_are_copied(plain, monkeypatch):
    """x in strides that the entry points refuse (rows not contiguous, not a constant distance
    apart, or overlapping) is copied, as the mixer's functions do; other strides are passed on."""
    taken = []
    for name in ("norm", "linear", "linear_backward"):
        def entry(x, *a, f=getattr(whtmix, name), **k):
            taken.append(x)
            assert all(t.is_contiguous() for t in a if torch.is_tensor(t))
            return f(x, *a, **k)
        monkeypatch.setattr(whtmix, name, entry)
    w = torch.randn(8, 5, dtype=torch.float64, requires_grad=True)
    g = torch.randn(8, dtype=torch.float64)
    t = torch.randn(4, 6, 16, dtype=torch.float64, requires_grad=True)
    for view, copied in ((t[..., 3:11], False), (t[:, :3, :8], True),
                         (t.transpose(0, 1)[..., 4:12], True), (t[:, :, ::2], True),
                         (t[0, :1, :8].expand(5, 8), True), (t[0, :, 4:12], False)):
        taken.clear()
        bias = torch.randn(5, 2, dtype=torch.float64)[:, 0]
        loss = autograd.whtmix_linear(view, w, bias, "silu").sum()
        loss = loss + autograd.whtmix_norm(view, g, view.contiguous())[0].square().sum()
        got = torch.autograd.grad(loss, (t, w))
        for x in taken:
            rows, width, ld = whtmix._rows(x, "x")
            assert width == 8 and (rows <= 1 or ld >= 8)
            assert (x.data_ptr() == view.data_ptr()) is not copied
        loss = plain_linear(view, w, bias, "silu").sum()
        loss = loss + plain_norm(view, g, view)[0].square().sum()
        for a, b in zip(got, torch.autograd.grad(loss, (t, w))):
            assert torch.allclose(a, b, rtol=1e-9, atol=1e-11)


@pytest.mark.parametrize("dtype", [0, 1])
def test_workspace_of_the_norms_backward(monkeypatch, dtype):
    """What the header says: partial rows for dweight alone, and two floats a row for rows of more
    than 16384 elements alone."""
    import re
    if torch.cuda.device_count() > 0:
        pytest.skip("fake device addresses are for hosts without a GPU")
    monkeypatch.setenv("WHTMIX_TEST_FAIL_WORKSPACE", "1")

    def floats(rows, C, dweight):
        p = [(1 << 44) + (i << 40) for i in range(6)]
        p[5] *= dweight
        status = whtmix.call_rows("whtmix_norm_backward", tuple(p), (rows, C), (dtype,), 0, 1e-6)
        if status != 5:          # out of memory: the test hook's
            assert status         # (no GPU to launch on)
            return 0
        return int(re.search(r"of (\d+) bytes", whtmix.last_error()).group(1)) // 4

    for rows, C in ((1, 64), (10 ** 8, 8), (10 ** 6, 128), (5000, 4096), (3000, 16384)):
        assert C <= floats(rows, C, True) <= 1536 * C, (rows, C)
        assert floats(rows, C, False) == 0, (rows, C)
    for rows, C in ((1, 16392), (5000, 20000), (10 ** 6, 70001)):
        assert floats(rows, C, False) == 2 * rows, (rows, C)
        assert 2 * rows + C <= floats(rows, C, True) <= 2 * rows + 1536 * C, (rows, C)
