"""Timed cases of what a text model needs around the mixer: embedding, layer norm and the gated product.

A case is a dict of plain values:

    op     "layer_norm"        one call of the layer norm with the residual's addition
           "layer_norm_mx"     the same with its output in 8 bits with block scales, and read back
           "layer_norm_train"  the layer norm's forward and backward passes
           "gated"             act(x Wg + bg) * (x Wu + bu), the gated feed-forward product
           "gated_mx"          the same of 8-bit activations and weights with block scales
           "gated_train"       its forward pass, and the backward pass of a kept one
           "embed"             rows of a table by token ids, times a scale
           "embed_train"       the lookup, and the table's gradient
    dtype  "f32" or "bf16": the element type (the operands of gated_mx are in 8 bits)
    M      tokens (rows);  K  width of the stream;  N  hidden width (gated), vocabulary (embed), else 0
    act    activation of the gate: "none", "relu", "gelu", "gelu_tanh", "silu"
    residual  whether a residual is added before the norm;  bias  whether there are biases
    ids    how tokens are spread: "uniform", or "zipf" (the r-th token 1 / r as often as the first)
    pad    share of tokens that are padding (id -1): zeros, and no gradient
    long   64-bit ids (else 32-bit)

With `own` set the calls are the framework's; else the operators' plain forms in 32 bits.
8-bit values are float8 e4m3 in blocks of 32 along the row that share a power of two 2^(byte - 127), the
least one that keeps the block's largest magnitude within 448.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-6
BLOCK = 32
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _case(name, op, dtype, M, K, N=0, act="none", residual=False, bias=True, ids="uniform",
          pad=0.0, long=True):
    return {"name": name, "op": op, "dtype": dtype, "M": M, "K": K, "N": N, "act": act,
            "residual": residual, "bias": bias, "ids": ids, "pad": pad, "long": long}


def listed():
    return [
        # One new token of a 4096-wide stream: only latency counts.
        _case("layer_norm_token", "layer_norm", "bf16", 1, 4096, residual=True),
        # A prompt of 8192 tokens, output in 8 bits for the product that reads it.
        _case("layer_norm_mx_prompt", "layer_norm_mx", "bf16", 8192, 4096, residual=True),
        # A training step on four 1024x2048 stereo pairs: many short rows.
        _case("layer_norm_train_stereo64k", "layer_norm_train", "bf16", 4 * 65536, 128,
              residual=True),
        # A training step on a ragged batch of odd width, float32, no residual.
        _case("layer_norm_train_ragged", "layer_norm_train", "f32", 5003, 1111),
        # One new token through both projections of a 4096-wide model: the weights' bytes.
        _case("gated_token", "gated", "bf16", 1, 4096, 12288, "silu", bias=False),
        # 17 sequences decoded together through 8-bit weights.
        _case("gated_mx_decode", "gated_mx", "bf16", 17, 4096, 16384, "gelu_tanh"),
        # A training step on four 1024x2048 stereo pairs, hidden width 8/3 of the stream's.
        _case("gated_train_stereo64k", "gated_train", "bf16", 4 * 65536, 128, 344, "silu"),
        # A training step of odd widths and a ragged batch, float32.
        _case("gated_train_ragged", "gated_train", "f32", 3001, 1000, 2003, "gelu"),
        # A training step on 8192 tokens of a wide model: the largest products.
        _case("gated_train_prompt", "gated_train", "bf16", 8192, 4096, 12288, "silu", bias=False),
        # 17 sequences' next tokens out of a large vocabulary: the smallest call.
        _case("embed_decode", "embed", "bf16", 17, 4096, 131072, long=False),
        # A training step on 32 texts of 4096 bytes: few rows, each of very many tokens.
        _case("embed_train_text4k", "embed_train", "f32", 32 * 4096, 64, 256),
        # A training step on 65536 tokens of a padded batch: a wide table, tokens as text has them.
        _case("embed_train_vocab", "embed_train", "bf16", 65536, 1024, 50000, ids="zipf", pad=0.1),
    ]


# No drawn case costs more than the largest listed product, nor moves more than the largest
# training step of many short rows does.
MAX_FLOPS = 12 * 8192 * 4096 * 12288
MAX_BYTES = 1_280_000_000


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width in lo .. hi: a power of two, a multiple of 40, or any odd count."""
    kind = rng.random()
    if kind < 0.4:
        return 1 << rng.randint(math.ceil(math.log2(lo)), math.floor(math.log2(hi)))
    w = _log(rng, lo, hi)
    return max(40, w // 40 * 40) if kind < 0.7 else w | 1


def draw(rng):
    op = rng.choice(["layer_norm", "layer_norm_mx", "layer_norm_train", "gated", "gated_mx",
                     "gated_train", "embed", "embed_train", "embed_train"])
    while True:
        case = {"op": op, "dtype": "bf16" if op.endswith("mx") else rng.choice(["f32", "bf16"])}
        # Tokens: single ones and small batches as served, or prompts and training batches.
        small = not op.endswith("train") and rng.random() < 0.35
        case["M"] = rng.randint(1, 64) if small else _log(rng, 64, 262144)
        case["K"] = _width(rng, 64, 8192)
        case["N"] = (_width(rng, 64, 16384) if op.startswith("gated") else
                     _width(rng, 64, 131072) if op.startswith("embed") else 0)
        case["act"] = rng.choice(ACTS) if op.startswith("gated") else "none"
        case["residual"] = op.startswith("layer_norm") and rng.random() < 0.7
        case["bias"] = rng.random() < 0.7
        case["ids"] = rng.choice(["uniform", "zipf"])
        case["pad"] = rng.choice([0.0, 0.0, 0.05, 0.3])
        case["long"] = rng.random() < 0.7
        w = work(case)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return case


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


# ---- block-scaled 8 bits, plain form ----

def _quantize(v):
    """float32 [R, C] -> (float8 [R, Cp], uint8 [R, Cp/32]), Cp = C rounded up to 32."""
    R, C = v.shape
    Cp = -(-C // BLOCK) * BLOCK
    if Cp != C:
        v = torch.cat([v, v.new_zeros(R, Cp - C)], 1)
    b = v.reshape(R, Cp // BLOCK, BLOCK)
    m, e = torch.frexp(b.abs().amax(-1))
    e = (e - 9 + (m > 0.875)).clamp(-126, 120)
    q = torch.ldexp(b, -e.unsqueeze(-1)).to(torch.float8_e4m3fn)
    return q.reshape(R, Cp), (e + 127).to(torch.uint8)


def _values(q, scales, dtype=torch.float32):
    """The numbers that 8-bit values and their scales stand for."""
    R, Cp = q.shape
    b = q.to(dtype).reshape(R, Cp // BLOCK, BLOCK)
    one = torch.ones((), dtype=dtype, device=q.device)
    s = torch.ldexp(one, scales.to(torch.int32) - 127)
    return (b * s.unsqueeze(-1)).reshape(R, Cp)


def _scale(case):
    """Rows of the embedding are scaled to a size of about one, as models scale them."""
    return math.sqrt(case["K"])


def prepare(case, seed):
    op, M, K, N, dt = case["op"], case["M"], case["K"], case["N"], _dtype(case)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    s = {"case": dict(case)}
    if op.startswith("layer_norm"):
        s["x"] = (normal(M, K) + normal(K, std=0.5)).to(dt)
        s["w"] = 1 + normal(K, std=0.1)
        s["b"] = normal(K, std=0.1) if case["bias"] else None
        s["res"] = normal(M, K, std=2.0).to(dt) if case["residual"] else None
        if op == "layer_norm_train":
            s["dy"] = normal(M, K).to(dt)
            s["dh"] = normal(M, K).to(dt) if case["residual"] else None
    if op.startswith("gated"):
        s["bg"], s["bu"] = ((normal(N, std=0.1), normal(N, std=0.1)) if case["bias"]
                            else (None, None))
    if op == "gated_mx":
        s["xq"], s["xs"] = _quantize(normal(M, K))
        s["gq"], s["gs"] = _quantize(normal(N, K, std=K ** -0.5))
        s["uq"], s["us"] = _quantize(normal(N, K, std=K ** -0.5))
    elif op.startswith("gated"):
        s["x"] = normal(M, K).to(dt)
        s["wg"], s["wu"] = (normal(K, N, std=K ** -0.5).to(dt) for _ in range(2))
        if op == "gated_train":
            s["dy"] = normal(M, N).to(dt)
            # What an earlier forward pass on x kept for the backward pass, in the stream's type.
            for z, w, b in (("zg", "wg", "bg"), ("zu", "wu", "bu")):
                v = s["x"].float() @ s[w].float()
                s[z] = (v if s[b] is None else v + s[b]).to(dt)
    if op.startswith("embed"):
        s["table"] = normal(N, K, std=K ** -0.5).to(dt)
        if case["ids"] == "zipf":
            often = torch.cumsum(1 / torch.arange(1, N + 1, dtype=torch.float64, device="cuda"), 0)
            u = torch.rand(M, generator=g, device="cuda", dtype=torch.float64) * often[-1]
            ids = torch.searchsorted(often, u).clamp(max=N - 1)
        else:
            ids = torch.randint(N, (M,), generator=g, device="cuda")
        if case["pad"]:
            gone = torch.rand(M, generator=g, device="cuda") < case["pad"]
            ids = torch.where(gone, torch.full_like(ids, -1), ids)
        s["ids"] = ids if case["long"] else ids.to(torch.int32)
        if op == "embed_train":
            s["dy"] = normal(M, K).to(dt)
    return s


# ---- the plain forms ----

def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if name == "gelu_tanh":
        return z / (1 + torch.exp(-2 * (2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_grad(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return (0.5 * (1 + torch.erf(z * 0.5 ** 0.5))
                + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5)
    if name == "gelu_tanh":
        c = 2 * (2 / math.pi) ** 0.5
        s = 1 / (1 + torch.exp(-c * (z + 0.044715 * z * z * z)))
        return s + z * s * (1 - s) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s + z * s * (1 - s)
    return torch.ones_like(z)


def _centred(t):
    """(t - mean) / sqrt(variance + eps) and the factor, in 32 bits."""
    c = t - t.mean(-1, keepdim=True)
    rstd = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
    return c * rstd, rstd


def _product(x, w, b):
    z = x @ w
    return z if b is None else z + b


def _plain(s):
    case = s["case"]
    op, act, dt = case["op"], case["act"], _dtype(case)
    if op.startswith("layer_norm"):
        t = s["x"].float()
        if s["res"] is not None:
            t = t + s["res"].float()
        y = _centred(t)[0] * s["w"]
        if s["b"] is not None:
            y = y + s["b"]
        h = t.to(dt)
        if op == "layer_norm":
            return {"y": y.to(dt), "h": h}
        if op == "layer_norm_mx":
            return {"y": _values(*_quantize(y))[:, :case["K"]].to(dt), "h": h}
        n, rstd = _centred(h.float())
        dy = s["dy"].float()
        g = dy * s["w"]
        dx = rstd * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        out = {"y": y.to(dt), "h": h, "dx": dx.to(dt), "dw": (dy * n).sum(0)}
        return {**out, "db": dy.sum(0)} if s["b"] is not None else out
    if op == "gated_mx":
        x = _values(s["xq"], s["xs"])
        zg = _product(x, _values(s["gq"], s["gs"]).t(), s["bg"])
        zu = _product(x, _values(s["uq"], s["us"]).t(), s["bu"])
        return {"y": (_act(act, zg) * zu).to(dt)}
    if op.startswith("gated"):
        x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
        zg, zu = _product(x, wg, s["bg"]), _product(x, wu, s["bu"])
        y = (_act(act, zg) * zu).to(dt)
        if op == "gated":
            return {"y": y}
        out = {"y": y, "zg": zg.to(dt), "zu": zu.to(dt)}
        dy, zg, zu = s["dy"].float(), s["zg"].float(), s["zu"].float()
        dg, du = dy * zu * _act_grad(act, zg), dy * _act(act, zg)
        out.update(dx=(dg @ wg.t() + du @ wu.t()).to(dt), dwg=(x.t() @ dg).to(dt),
                   dwu=(x.t() @ du).to(dt))
        if s["bg"] is not None:
            out.update(dbg=dg.sum(0), dbu=du.sum(0))
        return out
    ids, scale = s["ids"].long(), _scale(case)                   # embed
    real = (ids >= 0).unsqueeze(-1)
    at = ids.clamp(min=0)
    y = s["table"][at].float() * scale
    out = {"y": torch.where(real, y, torch.zeros_like(y)).to(dt)}
    if op == "embed_train":
        dy = s["dy"].float()
        dtable = dy.new_zeros(case["N"], case["K"])
        dtable.index_add_(0, at, torch.where(real, dy, torch.zeros_like(dy)))
        out["dtable"] = (dtable * scale).to(dt)
    return out


# ---- the framework's operators ----

def _own(s):
    from paper_2607_25234_amd import whtmix

    case = s["case"]
    op, act = case["op"], case["act"]
    if op == "layer_norm_mx":
        q, scales, h = whtmix.layer_norm_mx(s["x"], s["w"], s["b"], s["res"], eps=EPS)
        return {"y": whtmix.dequantize_mx(q, scales, case["K"], _dtype(case)), "h": h}
    if op.startswith("layer_norm"):
        y, h = whtmix.layer_norm(s["x"], s["w"], s["b"], s["res"], eps=EPS)
        if op == "layer_norm":
            return {"y": y, "h": h}
        dx, dw, db = whtmix.layer_norm_backward(h, s["w"], s["dy"], s["dh"], eps=EPS,
                                                want_dbias=s["b"] is not None)
        out = {"y": y, "h": h, "dx": dx, "dw": dw}
        return {**out, "db": db} if s["b"] is not None else out
    if op == "gated_mx":
        return {"y": whtmix.gated_mx(s["xq"], s["xs"], s["gq"], s["gs"], s["uq"], s["us"],
                                     s["bg"], s["bu"], activation=act)}
    if op == "gated":
        return {"y": whtmix.gated(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], activation=act)}
    if op == "gated_train":
        y, zg, zu = whtmix.gated(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], activation=act,
                                 want_z=True)
        dx, dwg, dwu, dbg, dbu = whtmix.gated_backward(
            s["x"], s["wg"], s["wu"], s["dy"], s["zg"], s["zu"], activation=act,
            want_dbias=s["bg"] is not None)
        out = {"y": y, "zg": zg, "zu": zu, "dx": dx, "dwg": dwg, "dwu": dwu}
        return {**out, "dbg": dbg, "dbu": dbu} if s["bg"] is not None else out
    out = {"y": whtmix.embedding(s["ids"], s["table"], scale=_scale(case))}
    if op == "embed_train":
        out["dtable"] = whtmix.embedding_backward(s["ids"], s["dy"], case["N"],
                                                  scale=_scale(case))
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition in 64 bits ----

def _act64(name, z):
    """(act(z), act'(z)), the derivative by the product rule on z * S(z)."""
    one = torch.ones_like(z)
    if name == "none":
        return z, one
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "gelu":
        S = 0.5 * torch.erfc(-z / math.sqrt(2))
        dS = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:
        u, du = z, one
        if name == "gelu_tanh":
            c = math.sqrt(8 / math.pi)
            u, du = c * (z + 0.044715 * z ** 3), c * (1 + 0.134145 * z ** 2)
        S = torch.sigmoid(u)
        dS = S * torch.sigmoid(-u) * du
    return z * S, S + z * dS


def _round_mx64(v):
    """64-bit rows rounded to the nearest block-scaled 8-bit values (ties to even), in 64 bits."""
    R, C = v.shape
    b = torch.nn.functional.pad(v, (0, -C % BLOCK)).view(R, -1, BLOCK)
    top = b.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -118)
    unit = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(-126, 120))
    unit = torch.where(top > 448 * unit, 2 * unit, unit)          # log2's own rounding
    unit = torch.where(top <= 224 * unit, unit / 2, unit)
    t = (b / unit).abs()
    step = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6))) - 3)   # e4m3: 3 bits
    return (torch.sign(b) * torch.round(t / step) * step * unit).view(R, -1)[:, :C]


def _stats64(h, K):
    """Rows less their mean, and their standard deviation."""
    d = h - h.sum(-1, keepdim=True) / K
    return d, (d.pow(2).sum(-1, keepdim=True) / K + EPS).sqrt()


def exact(case, seed):
    s = prepare(case, seed)
    op, K, dt = case["op"], case["K"], _dtype(case)
    d = {k: v.double() for k, v in s.items()
         if torch.is_tensor(v) and v.dtype in (torch.float32, torch.bfloat16)}
    if op.startswith("layer_norm"):
        h = d["x"] + d["res"] if "res" in d else d["x"]
        c, sigma = _stats64(h, K)
        y = torch.addcmul(d["b"], c / sigma, d["w"]) if "b" in d else c / sigma * d["w"]
        if op == "layer_norm":
            return {"y": y, "h": h}
        if op == "layer_norm_mx":
            return {"y": _round_mx64(y), "h": h}
        c, sigma = _stats64(h.to(dt).double(), K)     # the backward pass reads the stream as stored
        n = c / sigma
        dn = d["dy"] * d["w"]
        along = (dn * n).sum(-1, keepdim=True) / K
        dx = (dn - dn.sum(-1, keepdim=True) / K - n * along) / sigma + d.get("dh", 0)
        out = {"y": y, "h": h, "dx": dx, "dw": (d["dy"] * n).sum(0)}
        return {**out, "db": d["dy"].sum(0)} if "b" in d else out
    if op.startswith("gated"):
        if op == "gated_mx":
            x = _values(s["xq"], s["xs"], torch.float64)
            wg, wu = (_values(s[q], s[b], torch.float64).t() for q, b in (("gq", "gs"), ("uq", "us")))
        else:
            x, wg, wu = d["x"], d["wg"], d["wu"]
        zg, zu = torch.mm(x, wg), torch.mm(x, wu)
        if "bg" in d:
            zg, zu = zg + d["bg"], zu + d["bu"]
        y = zu * _act64(case["act"], zg)[0]
        if op != "gated_train":
            return {"y": y}
        a, da = _act64(case["act"], d["zg"])          # the backward pass reads both as kept
        dg, du = d["dy"] * da * d["zu"], d["dy"] * a
        out = {"y": y, "zg": zg, "zu": zu,
               "dx": torch.addmm(torch.mm(dg, wg.t()), du, wu.t()),
               "dwg": torch.mm(x.t(), dg), "dwu": torch.mm(x.t(), du)}
        return {**out, "dbg": dg.sum(0), "dbu": du.sum(0)} if "bg" in d else out
    ids = s["ids"].long()
    rows = torch.cat([d["table"], d["table"].new_zeros(1, K)])   # a row of zeros for padding
    at = torch.where(ids < 0, torch.full_like(ids, case["N"]), ids)
    out = {"y": rows[at] * _scale(case)}
    if op == "embed_train":
        dtable = torch.zeros_like(rows).index_put_((at,), d["dy"], accumulate=True)
        out["dtable"] = dtable[:-1] * _scale(case)
    return out


def _distinct(case):
    """How many rows of the table a batch's tokens name, on average."""
    M, N = case["M"] * (1 - case["pad"]), case["N"]
    if case["ids"] == "uniform":
        return N * -math.expm1(M * math.log1p(-1 / N))
    p = 1 / np.arange(1, N + 1)
    p /= p.sum()
    return float(-np.expm1(M * np.log1p(-p)).sum())


def work(case):
    op, M, K, N = case["op"], case["M"], case["K"], case["N"]
    e = 4 if case["dtype"] == "f32" else 2
    res, vectors = bool(case["residual"]), 2 if case["bias"] else 1
    mx = 1 + 1 / BLOCK
    if op == "layer_norm":        # x, y (and the residual and the stream)
        return {"bytes": M * K * e * (4 if res else 3) + 4 * K * vectors, "flops": 8 * M * K}
    if op == "layer_norm_mx":     # written in 8 bits, read back and written as numbers
        return {"bytes": M * K * (e * (4 if res else 3) + 2 * mx) + 4 * K * vectors,
                "flops": 12 * M * K}
    if op == "layer_norm_train":  # forward: x, y (residual, stream); backward: stream, dy, (dh,) dx
        return {"bytes": M * K * e * (8 if res else 6) + 12 * K * vectors, "flops": 24 * M * K}
    bias = 8 * N if case["bias"] else 0
    if op == "gated":
        return {"bytes": e * (M * K + 2 * K * N + M * N) + bias, "flops": 4 * M * K * N}
    if op == "gated_mx":
        return {"bytes": mx * (M * K + 2 * K * N) + e * M * N + bias, "flops": 4 * M * K * N}
    if op == "gated_train":       # forward: x, weights, y, both z; backward: x, weights, both z, dy, dx, dw
        return {"bytes": e * (3 * M * K + 6 * K * N + 6 * M * N) + 2 * bias,
                "flops": 12 * M * K * N}
    read = (8 if case["long"] else 4) * M + e * int(_distinct(case)) * K
    if op == "embed":             # ids, the rows that they name, y
        return {"bytes": read + e * M * K, "flops": M * K}
    return {"bytes": read + e * (2 * M * K + N * K), "flops": 3 * M * K}
