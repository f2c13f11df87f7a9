"""Layer norm, gated products and embedding in 64 bits on the CPU, with bounds of the kernels'
errors (not collected by pytest); layer_ref has the rules by which the bounds are formed."""
from __future__ import annotations

import math

import torch

from tests.layer_ref import U, act, act_bound, act_grad, grad_bound, rounded, sum_bound


def sums(n):
    """Of a float32 sum of n terms, per unit of its sum of magnitudes."""
    return 8 * (4 + math.sqrt(n)) * U


def layer_norm(x, r, w, b, eps):
    """(y, bound without its rounding, t) of rows x + r.  The mean of the float32 t is off by
    sums(C) of the mean magnitude; the distances from it carry that and lose it again with
    their own mean, whose error is sums(C) of their magnitudes, that error's share among them."""
    C = x.shape[-1]
    t = x.double() + (0 if r is None else r.double())
    own = U * (0 if r is None else 1) * t.abs()           # t's rounding
    d = t - t.mean(-1, keepdim=True)
    rstd = 1 / (d.square().mean(-1, keepdim=True) + eps).sqrt()
    n = d * rstd
    W = w.double()
    y = n * W + (0 if b is None else b.double())
    far = d.abs().mean(-1, keepdim=True) + sums(C) * t.abs().mean(-1, keepdim=True)
    at = own + own.mean(-1, keepdim=True) if r is not None else 0
    bound = ((n * W).abs() * (sums(C) + 4 * U) + W.abs() * rstd * (at + sums(C) * far)
             + 4 * U * y.abs())
    # the variance's error from the distances': 2 d (error of d), over the variance
    if r is not None:
        bound = bound + (n * W).abs() * 2 * (own * d.abs()).mean(-1, keepdim=True) * rstd ** 2
    return y, bound, t


def layer_norm_backward(h, w, dy, dh, eps):
    """(dx, its bound without the rounding, dw, bound, db, bound)."""
    rows, C = h.shape
    H, W, D = h.double(), w.double(), dy.double()
    d = H - H.mean(-1, keepdim=True)
    rstd = 1 / (d.square().mean(-1, keepdim=True) + eps).sqrt()
    n, g = d * rstd, D * W
    dx = rstd * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True))
    # n is off by sums(C) of itself and of the row's mean of magnitudes (which is at most 1),
    # and by what the mean's error leaves
    one = n.abs() + 1 + sums(C) * rstd * H.abs().mean(-1, keepdim=True)
    mag = rstd * (g.abs() + g.abs().mean(-1, keepdim=True)
                  + one * (g * n).abs().mean(-1, keepdim=True)
                  + n.abs() * (g.abs() * one).mean(-1, keepdim=True))
    if dh is not None:
        dx, mag = dx + dh.double(), mag + dh.double().abs()
    return (dx, sums(C) * mag, (D * n).sum(0),
            sum_bound(rows, (D * n).abs().sum(0)) + sums(C) * (D.abs() * one).sum(0),
            D.sum(0), sum_bound(rows, D.abs().sum(0)))


def gated(x, wg, wu, bg, bu, name):
    """(y, bound without its rounding, zg, zu, their bounds without theirs)."""
    X = x.double()
    K = x.shape[-1]
    z, bz = [], []
    for w, b in ((wg, bg), (wu, bu)):
        v = 0 if b is None else b.double()
        z.append(X @ w.double() + v)
        bz.append(sum_bound(K, X.abs() @ w.double().abs() + abs(v)))
    a = act(name, z[0])
    ba = act_bound(name, z[0], bz[0])
    y = a * z[1]
    return y, ba * (z[1].abs() + bz[1]) + a.abs() * bz[1] + 4 * U * y.abs(), *z, *bz


def gated_backward(x, wg, wu, dy, zg, zu, name, bf16):
    """[(dx, bound), (dwg, bound), (dwu, bound), (dbg, bound), (dbu, bound)], the roundings of the
    first three left to the caller.  dzg and dzu are rounded to bf16 for the products: 2^-8
    of each of their values."""
    X, D, G, V = x.double(), dy.double(), zg.double(), zu.double()
    M, N = dy.shape
    dg, du = D * V * act_grad(name, G), D * act(name, G)
    og = (D * V).abs() * grad_bound(name, G) + 4 * U * dg.abs()
    ou = D.abs() * act_bound(name, G, torch.zeros_like(G)) + 4 * U * du.abs()
    step = 2.0 ** -7.99 if bf16 else 2 * U
    out = []
    dx = bx = 0
    for d, o, w in ((dg, og, wg), (du, ou, wu)):
        W = w.double()
        dx = dx + d @ W.t()
        bx = bx + (sums(2 * N) * d.abs() + o + step * d.abs()) @ W.abs().t()
        out.append((X.t() @ d, sum_bound(M, X.abs().t() @ d.abs())
                    + X.abs().t() @ (o + step * d.abs())))
    for d, o in ((dg, og), (du, ou)):
        out.append((d.sum(0), sum_bound(M, d.abs().sum(0)) + o.sum(0) + 1e-30))
    return [(dx, bx), *out]


def embedding(ids, table, scale):
    """Rows, in 64 bits: zeros for padding, NaN past the table."""
    ids = ids.long()
    V = table.shape[0]
    y = table.double()[ids.clamp(0, V - 1)] * scale
    y[ids < 0] = 0
    y[ids >= V] = math.nan
    return y


def embedding_backward(ids, dy, vocab, scale, bf16):
    """(dtable, bound)."""
    ids, C = ids.reshape(-1).long(), dy.shape[-1]
    D = dy.double().reshape(-1, C)
    real = (ids >= 0) & (ids < vocab)
    ids, D = ids[real], D[real]
    zero = torch.zeros(vocab, C, dtype=torch.float64)
    g = zero.clone().index_add_(0, ids, D) * scale
    mag = zero.index_add_(0, ids, D.abs()) * abs(scale)
    n = torch.bincount(ids, minlength=vocab).double().sqrt()[:, None]
    return g, 8 * (4 + n) * U * mag + rounded(g, bf16)
