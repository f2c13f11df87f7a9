"""The Python side of layer norm, gated products and embedding without a GPU, beyond what the
tests of its results see: what a call without gradients is asked to keep."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from torch.utils._python_dispatch import TorchDispatchMode  # noqa: E402

from paper_2607_25234_amd import autograd, whtmix  # noqa: E402
from tests.test_layer_host import (plain_linear, plain_linear_backward, plain_norm,  # noqa: E402
                                   plain_norm_backward)
from tests.test_text_host import (plain_gated, plain_gated_backward, plain_layer_norm,  # noqa: E402
                                  plain_layer_norm_backward)


@pytest.fixture
def kept(monkeypatch):
    """What the products are asked to keep, call by call."""
    asked = []
    for name, f in (("gated", plain_gated), ("linear", plain_linear)):
        monkeypatch.setattr(whtmix, name, lambda *a, f=f, want_z=False: (
            asked.append(want_z), f(*a, want_z=want_z))[1])
    for f in (plain_norm, plain_layer_norm, plain_norm_backward, plain_layer_norm_backward,
              plain_gated_backward, plain_linear_backward):
        monkeypatch.setattr(whtmix, f.__name__[len("plain_"):], f)
    return asked


class Copies(TorchDispatchMode):
    """Counts the copies that contiguous() makes."""

    def __init__(self):
        super().__init__()
        self.count = 0

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.count += func is torch.ops.aten.clone.default
        return func(*args, **(kwargs or {}))


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_without_gradients_nothing_is_kept(kept, mode):
    """Parameters ask for gradients whatever the mode; a call that records none keeps no product
    before its activation, and copies no rows for a norm's backward pass."""
    p = torch.nn.Parameter
    x = torch.randn(6, 24)[:, 4:12]
    w, g, b = p(torch.randn(8, 8)), p(torch.ones(8)), p(torch.zeros(8))

    def run():
        kept.clear()
        with Copies() as copies:
            autograd.whtmix_gated(x, w, w, b, b)
            autograd.whtmix_linear(x, w, b, "silu")
            y, h = autograd.whtmix_layer_norm(x, g, b)
            z, s = autograd.whtmix_norm(x, g)
        assert h is x and s is x
        return copies.count

    assert run() == 2 and kept == [True, True]
    with mode():
        assert run() == 0 and kept == [False, False]
    w.requires_grad_(False), g.requires_grad_(False), b.requires_grad_(False)
    assert run() == 0 and kept == [False, False]


def test_gradients_of_calls_among_ones_without(kept):
    """A call that records gradients has them, whatever was called before it in another mode."""
    p = torch.nn.Parameter
    x, r = torch.randn(6, 8, dtype=torch.float64), torch.randn(6, 8, dtype=torch.float64)
    w, g, b = (p(torch.randn(s, dtype=torch.float64)) for s in ((8, 8), (8,), (8,)))

    def run(f):
        gated, linear, layer_norm, norm = f
        y, h = layer_norm(x, g, b, r)
        z, s = norm(gated(y, w, w, b, b), g)
        return (linear(z, w, b, "silu") + h + s).sum()

    own = (autograd.whtmix_gated, autograd.whtmix_linear, autograd.whtmix_layer_norm,
           autograd.whtmix_norm)
    with torch.no_grad():
        alone = run(own)
    got = torch.autograd.grad(run(own), (w, g, b))
    want = run((plain_gated, plain_linear, plain_layer_norm, plain_norm))
    assert torch.allclose(alone, want)
    for a, c in zip(got, torch.autograd.grad(want, (w, g, b))):
        assert torch.allclose(a, c, rtol=1e-10, atol=1e-12)


def test_the_functions_by_themselves(kept):
    """Applied without the mode they keep what they kept before."""
    p = torch.nn.Parameter
    x = torch.randn(6, 8, dtype=torch.float64)
    w, g, b = (p(torch.randn(s, dtype=torch.float64)) for s in ((8, 8), (8,), (8,)))
    y = autograd.WHTMixLayerNormFunction.apply(x, g, b, None, 1e-6)
    y = autograd.WHTMixGatedFunction.apply(y, w, w, b, b, "silu")
    y = autograd.WHTMixNormFunction.apply(y, g, None, 1e-6)
    y = autograd.WHTMixLinearFunction.apply(y, w, b, "silu", None)
    assert kept == [True, True]
    want = plain_linear(plain_norm(plain_gated(plain_layer_norm(x, g, b)[0], w, w, b, b), g)[0], w,
                        b, "silu")
    for a, c in zip(torch.autograd.grad(y.sum(), (w, g, b)),
                    torch.autograd.grad(want.sum(), (w, g, b))):
        assert torch.allclose(a, c, rtol=1e-10, atol=1e-12)
