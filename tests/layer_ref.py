"""The feed-forward operators in 64 bits on the CPU, with bounds of the kernels' errors
(not collected by pytest).

Bounds hold element by element.  u = 2^-24 is float32's unit roundoff; sums of n
float32 terms are off by at most about sqrt(n) u of the sum of magnitudes (a
running sum's error is a random walk; 8 (4 + sqrt(n)) u leaves eight times that), and an
output rounded to bf16, of 8 significant bits, by 2^-8 of itself besides (2^-7.99 with what
comes before).
"""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def sum_bound(n, magnitudes):
    return 8 * (4 + math.sqrt(n)) * U * magnitudes


def rounded(r, bf16):
    """The rounding of an output r once to its type, bf16 or float32."""
    return r.abs() * (2.0 ** -7.99 if bf16 else 2 * U) + 2.0 ** -133


def act(name, z):
    if name == "none":
        return z
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    u = z if name == "silu" else math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)
    return z * torch.sigmoid(u)


def act_grad(name, z):
    if name == "relu":       # 0 at 0 (clamp's own gradient there is 1)
        return (z > 0).to(z.dtype)
    with torch.enable_grad():
        v = z.detach().clone().requires_grad_()
        return torch.autograd.grad(act(name, v).sum(), v)[0]


def act_bound(name, z, dz):
    """Error of act at a z off by dz: its slope is at most 1.13; erf is off by 1.5e-7 and the
    exponentials by a few u of their argument, both times |z|."""
    if name in ("none", "relu"):
        return dz
    return 1.2 * dz + z.abs() * (4e-7 + 8 * U * z.abs().clamp(max=100))


def grad_bound(name, z):
    if name in ("none", "relu"):
        return torch.zeros_like(z)
    return (1 + z.abs()) * (4e-7 + 16 * U * (1 + z.abs().clamp(max=100)))


def mx_round(v):
    """(values, scale bytes) of 64-bit rows in block-scaled 8 bits, from the definition: the
    least power of two in 2^-126 .. 2^120 that keeps the finite magnitudes within 448, then
    the nearest e4m3 value, ties to even; Inf and NaN become NaN."""
    R, C = v.shape
    b = torch.nn.functional.pad(v, (0, -C % 32)).reshape(R, -1, 32)
    fin = torch.isfinite(b)
    top = torch.where(fin, b, torch.zeros_like(b)).abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -126)
    for k in range(-125, 121):
        e = torch.where(top > 448 * 2.0 ** (k - 1), torch.full_like(e, k), e)
    unit = torch.exp2(e)
    t = (b / unit).abs()
    step = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6))) - 3)
    q = torch.sign(b) * torch.round(t / step) * step * unit
    q = torch.where(fin, q, torch.full_like(q, math.nan))
    return q.reshape(R, -1)[:, :C], (e[..., 0] + 127).to(torch.uint8)


def check(name, got, ref, bound):
    got = got.detach().double().cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fin), (name, "finite")
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), (name, "NaN")
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), (name, "Inf")
    bound = bound.expand_as(ref) if torch.is_tensor(bound) else torch.full_like(ref, bound)
    d, b = (got - ref).abs()[fin], bound[fin]
    worst = float((d / b).max()) if d.numel() else 0.0
    print(f"  {name}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, (name, worst)
