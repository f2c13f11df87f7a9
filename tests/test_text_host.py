"""The Python side of layer norm, gated products and embedding without a GPU: autograd wrappers
and the layers, with plain torch functions in the entry points' place."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from paper_2607_25234_amd import autograd, whtmix  # noqa: E402
from tests import layer_ref as ref  # noqa: E402
from tests.test_layer_host import plain_linear, plain_norm  # noqa: E402


def plain_layer_norm(x, weight, bias=None, residual=None, eps=1e-6):
    h = x if residual is None else x + residual
    d = h - h.mean(-1, keepdim=True)
    y = d * torch.rsqrt(d.square().mean(-1, keepdim=True) + eps) * weight
    return y if bias is None else y + bias, h


def plain_layer_norm_backward(h, weight, dy, dh=None, eps=1e-6, want_dweight=True,
                              want_dbias=True):
    d = h - h.mean(-1, keepdim=True)
    r = torch.rsqrt(d.square().mean(-1, keepdim=True) + eps)
    n, g = d * r, dy * weight
    dx = r * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True))
    C = h.shape[-1]
    return (dx if dh is None else dx + dh, (dy * n).reshape(-1, C).sum(0) if want_dweight else None,
            dy.reshape(-1, C).sum(0) if want_dbias else None)


def plain_gated(x, w_gate, w_up, b_gate=None, b_up=None, activation="silu", want_z=False):
    zg = x @ w_gate if b_gate is None else x @ w_gate + b_gate
    zu = x @ w_up if b_up is None else x @ w_up + b_up
    y = ref.act(activation, zg) * zu
    return (y, zg, zu) if want_z else y


def plain_gated_backward(x, w_gate, w_up, dy, zg, zu, activation="silu", want_dx=True,
                         want_dw=True, want_dbias=True):
    dg, du = dy * zu * ref.act_grad(activation, zg), dy * ref.act(activation, zg)
    K, N = w_gate.shape
    X, G, V = x.reshape(-1, K), dg.reshape(-1, N), du.reshape(-1, N)
    return (dg @ w_gate.t() + du @ w_up.t() if want_dx else None,
            X.t() @ G if want_dw else None, X.t() @ V if want_dw else None,
            G.sum(0) if want_dbias else None, V.sum(0) if want_dbias else None)


def plain_embedding(ids, table, scale=1.0):
    return table[ids.clamp(min=0)] * scale * (ids >= 0).unsqueeze(-1)


def plain_embedding_backward(ids, dy, vocab, scale=1.0):
    g = dy.new_zeros(vocab + 1, dy.shape[-1])
    at = torch.where(ids < 0, vocab, ids).reshape(-1)
    return g.index_add_(0, at, dy.reshape(-1, dy.shape[-1]))[:-1] * scale


@pytest.fixture
def plain(monkeypatch):
    for name in ("layer_norm", "layer_norm_backward", "gated", "gated_backward", "embedding",
                 "embedding_backward"):
        monkeypatch.setattr(whtmix, name, globals()["plain_" + name])


def leaves():
    torch.manual_seed(0)
    p = {"table": (9, 8), "r": (2, 5, 8), "g": (8,), "b": (8,), "wg": (8, 7), "wu": (8, 7),
         "bg": (7,), "bu": (7,)}
    return {k: torch.randn(s, dtype=torch.float64, requires_grad=True) for k, s in p.items()}


IDS = torch.tensor([[0, 3, -1, 8, 3], [-4, 2, 2, 0, 1]])


def loss(p, embedding, layer_norm, gated, bias=True, residual=True):
    x = embedding(IDS, p["table"], 1.5)
    y, h = layer_norm(x, p["g"], p["b"] if bias else None, p["r"] if residual else None, 1e-6)
    u = gated(y, p["wg"], p["wu"], p["bg"] if bias else None, p["bu"] if bias else None, "silu")
    return (u * torch.arange(7)).sum() + h.pow(3).sum()


def own(p, **k):
    return loss(p, autograd.whtmix_embedding, autograd.whtmix_layer_norm, autograd.whtmix_gated, **k)


def test_first_derivatives(plain):
    """With and without biases, a residual and a graph of the gradients: the plain functions'."""
    p = leaves()
    for bias in (True, False):
        for residual in (True, False):
            used = [v for k, v in p.items()
                    if (bias or k not in ("b", "bg", "bu")) and (residual or k != "r")]
            k = dict(bias=bias, residual=residual)
            want = torch.autograd.grad(loss(p, plain_embedding, plain_layer_norm, plain_gated, **k),
                                       used)
            for graph in (False, True):
                got = torch.autograd.grad(own(p, **k), used, create_graph=graph)
                for a, b in zip(got, want):
                    assert torch.allclose(a, b, rtol=1e-10, atol=1e-12)


def test_only_what_is_asked_for(plain, monkeypatch):
    """Each leaf alone: its gradient, and the entry points are asked for no other; without any,
    nothing is kept."""
    p = leaves()
    want = dict(zip(p, torch.autograd.grad(
        loss(p, plain_embedding, plain_layer_norm, plain_gated), list(p.values()))))
    asked = []
    monkeypatch.setattr(whtmix, "gated_backward", lambda *a, **k: (
        asked.append(k), plain_gated_backward(*a, **k))[1])
    for name in p:
        q = {k: v.detach().requires_grad_(k == name) for k, v in p.items()}
        asked.clear()
        own(q).backward()
        assert torch.allclose(q[name].grad, want[name], rtol=1e-10, atol=1e-12), name
        if name in ("wg", "wu"):
            assert asked == [dict(want_dx=False, want_dw=True, want_dbias=False)]
        if name in ("bg", "bu"):
            assert asked == [dict(want_dx=False, want_dw=False, want_dbias=True)]
    kept = []
    monkeypatch.setattr(whtmix, "gated", lambda *a, want_z=False: (
        kept.append(want_z), plain_gated(*a, want_z=want_z))[1])
    own({k: v.detach() for k, v in p.items()})
    assert kept == [False]


def test_second_derivatives_are_refused(plain):
    p = leaves()
    for f, names in ((lambda: autograd.whtmix_layer_norm(p["r"], p["g"], p["b"])[0], "rgb"),
                     (lambda: autograd.whtmix_layer_norm(p["r"], p["g"], p["b"], p["r"])[0], "rgb"),
                     (lambda: autograd.whtmix_gated(p["r"], p["wg"], p["wu"], p["bg"], p["bu"]),
                      ("r", "wg", "wu", "bg", "bu"))):
        for name in names:
            total = f().square().sum() + p["r"].pow(3).sum()
            first, = torch.autograd.grad(total, p["r"], create_graph=True)
            with pytest.raises(RuntimeError, match="second derivative"):
                torch.autograd.grad(first.sum() + p[name].sum(), p[name])
    total = autograd.whtmix_embedding(IDS, p["table"]).square().sum() + p["table"].pow(3).sum()
    first, = torch.autograd.grad(total, p["table"], create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        first.sum().backward()


def test_rows_of_any_strides_are_copied(plain, monkeypatch):
    """x in strides that the entry points refuse is copied, other strides are passed on; every
    other tensor reaches them contiguous."""
    taken = []
    for name in ("layer_norm", "gated", "gated_backward", "embedding", "embedding_backward"):
        def entry(x, *a, f=getattr(whtmix, name), **k):
            taken.append(x)
            assert all(t.is_contiguous() for t in a if torch.is_tensor(t))
            return f(x, *a, **k)
        monkeypatch.setattr(whtmix, name, entry)
    p = leaves()
    t = torch.randn(4, 6, 16, dtype=torch.float64, requires_grad=True)
    wg = torch.randn(7, 8, dtype=torch.float64, requires_grad=True)
    for view, copied in ((t[..., 3:11], False), (t[:, :3, :8], True),
                         (t.transpose(0, 1)[..., 4:12], True), (t[:, :, ::2], True),
                         (t[0, :1, :8].expand(5, 8), True), (t[0, :, 4:12], False)):
        taken.clear()

        def run(norm, gated):
            u = gated(view, wg.t(), p["wu"], p["bg"], p["bu"], "gelu").sum()
            return u + norm(view, p["g"], p["b"], view)[0].square().sum()

        got = torch.autograd.grad(run(autograd.whtmix_layer_norm, autograd.whtmix_gated), (t, wg))
        for x in taken:
            rows, width, ld = whtmix._rows(x, "x")
            assert width == 8 and (rows <= 1 or ld >= 8)
            assert (x.data_ptr() == view.data_ptr()) is not copied
        for a, b in zip(got, torch.autograd.grad(run(plain_layer_norm, plain_gated), (t, wg))):
            assert torch.allclose(a, b, rtol=1e-9, atol=1e-11)
    ids = IDS.t()
    y = autograd.whtmix_embedding(ids, p["table"].t().contiguous().t(), 2.0)
    assert torch.equal(y, plain_embedding(ids, p["table"], 2.0))
    g, = torch.autograd.grad((y.transpose(0, 1) * torch.arange(8)).sum(), p["table"])
    want, = torch.autograd.grad((plain_embedding(IDS, p["table"], 2.0) * torch.arange(8)).sum(),
                                p["table"])
    assert torch.allclose(g, want)


@pytest.fixture
def plain_layers(plain, monkeypatch):
    monkeypatch.setattr(whtmix, "norm", plain_norm)
    monkeypatch.setattr(whtmix, "linear", plain_linear)
    block = lambda x, i, a, b, o: (x @ i) * (a[:x.shape[-2], None] + 1) * (b + 1) @ o  # noqa: E731
    monkeypatch.setattr(whtmix, "module_forward_separable", block)
    monkeypatch.setattr(autograd, "whtmix_block_separable", block)
    monkeypatch.setattr(whtmix, "quantize_mx", lambda x: (x.clone(), None))

    def mx(f):
        return lambda *a, **k: ((n := f(*a, **k))[0], None, n[1])

    monkeypatch.setattr(whtmix, "norm_mx", mx(plain_norm))
    monkeypatch.setattr(whtmix, "layer_norm_mx", mx(plain_layer_norm))
    monkeypatch.setattr(whtmix, "linear_mx", lambda q, s, w, ws, b, act="none", residual=None,
                        out_mx=False: (y := plain_linear(q, w.t(), b, act, residual),
                                       None) if out_mx else plain_linear(q, w.t(), b, act, residual))
    monkeypatch.setattr(whtmix, "gated_mx", lambda q, s, w, ws, u, us, b, c, act, out_mx=False:
                        (plain_gated(q, w.t(), u.t(), b, c, act), None))


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("gated", [False, True])
def test_layers_and_their_served_form(plain_layers, norm, gated):
    from paper_2607_25234_amd.layer import MixerLayer, MixerLayerMx, MixerText
    torch.manual_seed(0)
    text = MixerText(9, 5, 8, 16, 2, dtype=torch.float32, norm=norm, gated=gated)
    with torch.no_grad():
        for p in text.parameters():
            p.add_(torch.randn_like(p) * 0.1)
        x = plain_embedding(IDS, text.table, 8 ** 0.5)
        for layer in text.layers:
            h = x + whtmix.module_forward_separable(x, layer.w_in, layer.log_gain_tokens,
                                                    layer.log_gain_channels, layer.w_out)
            n = plain_layer_norm(h, layer.norm_weight, layer.norm_bias)[0] if norm == "layer" \
                else plain_norm(h, layer.norm_weight)[0]
            u = n @ layer.w1 + layer.b1
            u = ref.act("gelu", u) * (n @ layer.w_up + layer.b_up) if gated else ref.act("gelu", u)
            served = MixerLayerMx(layer)
            want = h + u @ layer.w2 + layer.b2
            assert torch.allclose(served(x), want, rtol=1e-5, atol=1e-5)
            x = want
        assert torch.allclose(text(IDS), x, rtol=1e-5, atol=1e-5)
        want = served(h)
        for p in layer.parameters():
            p.add_(torch.randn_like(p))
        assert torch.equal(served(h), want)     # of the state that it was made of
    with pytest.raises(ValueError):
        MixerLayer(5, 8, 16, norm="batch")


def test_layer_of_before_has_the_parameters_of_before():
    """Without the new options: the same names, drawn in the same order."""
    from paper_2607_25234_amd.layer import MixerLayer
    names = ["w_in", "w_out", "log_gain_tokens", "log_gain_channels", "norm_weight", "w1", "w2",
             "b1", "b2"]
    torch.manual_seed(3)
    layer = MixerLayer(5, 8, 16, dtype=torch.float32)
    assert [k for k, _ in layer.named_parameters()] == names
    torch.manual_seed(3)
    for name, (k, n) in (("w_in", (8, 8)), ("w_out", (8, 8)), ("w1", (8, 16)), ("w2", (16, 8))):
        assert torch.equal(getattr(layer, name), torch.randn(k, n) * k ** -0.5), name
