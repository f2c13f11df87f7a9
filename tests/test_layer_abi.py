"""The feed-forward entry points' argument checks, on the host: every refusal comes before any
HIP call, through the call module and through ctypes alike."""
from __future__ import annotations

import ctypes

import pytest

from paper_2607_25234_amd import whtmix

INVALID, DTYPE, MISALIGNED, MEMORY, LARGE = 1, 3, 4, 5, 7
FAR = [(1 << 40) + (i << 34) for i in range(9)]      # addresses 16 GiB apart

# name: pointers (of which may be null), sizes, codes, eps
GOOD = {
    "whtmix_norm_forward": (5, (4, 64, 64), (0,), (1e-6,)),
    "whtmix_norm_mx_forward": (6, (64, 64, 64), (0,), (1e-6,)),
    "whtmix_norm_backward": (6, (4, 64), (0,), (1e-6,)),
    "whtmix_quantize_mx": (3, (64, 64, 64), (0,), ()),
    "whtmix_dequantize_mx": (3, (64, 64), (0,), ()),
    "whtmix_linear_forward": (6, (4, 64, 96, 64), (1, 0), ()),
    "whtmix_linear_backward": (7, (4, 64, 96, 64), (1, 0), ()),
    "whtmix_linear_mx_forward": (9, (64, 64, 96), (1, 0), ()),
}
# which pointers a call cannot do without, and where the outputs are
NEEDED = {
    "whtmix_norm_forward": (0, 2, 3), "whtmix_norm_mx_forward": (0, 2, 3, 4),
    "whtmix_norm_backward": (0, 1, 2, 4), "whtmix_quantize_mx": (0, 1, 2),
    "whtmix_dequantize_mx": (0, 1, 2), "whtmix_linear_forward": (0, 1, 4),
    "whtmix_linear_backward": (0, 1, 2, 3), "whtmix_linear_mx_forward": (0, 1, 2, 3),
}
OUTPUTS = {
    "whtmix_norm_forward": (3, 4), "whtmix_norm_mx_forward": (3, 4, 5),
    "whtmix_norm_backward": (4, 5), "whtmix_quantize_mx": (1, 2), "whtmix_dequantize_mx": (2,),
    "whtmix_linear_forward": (4, 5), "whtmix_linear_backward": (4, 5, 6),
    "whtmix_linear_mx_forward": (6,),
}
IN_PLACE = {("whtmix_norm_forward", 3, 0), ("whtmix_norm_forward", 4, 0),
            ("whtmix_norm_forward", 4, 1), ("whtmix_norm_mx_forward", 5, 0),
            ("whtmix_norm_mx_forward", 5, 1), ("whtmix_norm_backward", 4, 2),
            ("whtmix_norm_backward", 4, 3), ("whtmix_linear_forward", 4, 3),
            ("whtmix_linear_mx_forward", 6, 5)}


def pointers(name):
    p = FAR[:GOOD[name][0]]
    if name == "whtmix_linear_mx_forward":
        p[7] = p[8] = 0          # y, not 8 bits
    return p


def status(name, p, sizes, codes, eps):
    st = whtmix.call_rows(name, tuple(p), tuple(sizes), tuple(codes), 0, *eps)
    f = getattr(whtmix.lib(), name)
    assert st == f(*p, *sizes, *eps, *codes, 0)
    assert st, (name, p, sizes, codes, eps)       # a call that went through would launch
    return st


@pytest.mark.parametrize("name", GOOD)
def test_sizes_codes_and_eps(name):
    n, sizes, codes, eps = GOOD[name]
    p = pointers(name)
    for code in (2, -1, 99):
        assert status(name, p, sizes, (*codes[:-1], code), eps) == DTYPE
    widths = {"whtmix_linear_forward": (1, 2), "whtmix_linear_backward": (1, 2),
              "whtmix_linear_mx_forward": (1, 2)}.get(name, (1,))
    bad = list(sizes)
    bad[0] = -1
    assert status(name, p, bad, codes, eps) == INVALID
    for i in widths:
        for v, want in ((0, INVALID), (-5, INVALID), (1 << 22 | 1, LARGE)):
            bad = list(sizes)
            bad[i] = v
            if len(sizes) > 2 and "mx_forward" not in name or name == "whtmix_norm_mx_forward":
                bad[-1] = max(bad[-1], v)         # ldx follows the width
            assert status(name, p, bad, codes, eps) == want, (i, v)
    bad = list(sizes)
    bad[0] = (1 << 30) + 1
    assert status(name, p, bad, codes, eps) == LARGE
    if name in ("whtmix_norm_forward", "whtmix_norm_mx_forward", "whtmix_quantize_mx",
                "whtmix_linear_forward", "whtmix_linear_backward"):
        assert status(name, p, (*sizes[:-1], 63), codes, eps) == INVALID      # ldx below the width
        assert status(name, p, (*sizes[:-1], (1 << 31) + 1), codes, eps) == LARGE
    if eps:
        for e in (-1e-6, float("nan"), float("inf"), 1e39):
            assert status(name, p, sizes, codes, (e,)) == INVALID
    if len(codes) == 2:
        for act in (-1, 5, 1 << 20):
            assert status(name, p, sizes, (act, 0), eps) == INVALID


@pytest.mark.parametrize("name", GOOD)
def test_pointers(name):
    n, sizes, codes, eps = GOOD[name]
    for i in NEEDED[name]:
        p = pointers(name)
        p[i] = 0
        assert status(name, p, sizes, codes, eps) == INVALID, i
    p = pointers(name)
    for i in [i for i, v in enumerate(p) if v]:
        q = list(p)
        q[i] += 1
        eight_bits = {"whtmix_norm_mx_forward": (4,), "whtmix_quantize_mx": (2,),
                      "whtmix_dequantize_mx": (1,), "whtmix_linear_mx_forward": (1, 3)}
        if i not in eight_bits.get(name, ()):       # scales are bytes: any address
            assert status(name, q, sizes, codes, eps) == MISALIGNED, i
    for o in OUTPUTS[name]:
        for i in range(n):
            if i == o or not p[i]:
                continue
            q = list(p)
            q[o] = q[i]
            if (name, o, i) not in IN_PLACE:
                assert status(name, q, sizes, codes, eps) == INVALID, (o, i)
            q[o] = q[i] + 16                        # a partial overlap is never allowed
            assert status(name, q, sizes, codes, eps) == INVALID, (o, i)


def test_outputs_and_their_combinations():
    assert status("whtmix_linear_backward", [*FAR[:4], 0, 0, 0], (4, 64, 96, 64), (1, 0), ()) \
        == INVALID
    for y, q, s in ((1, 1, 1), (0, 1, 0), (0, 0, 1), (0, 0, 0), (1, 0, 1), (1, 1, 0)):
        p = FAR[:9]
        for i, keep in zip((6, 7, 8), (y, q, s)):
            p[i] *= keep
        assert status("whtmix_linear_mx_forward", p, (4, 64, 96), (0, 0), ()) == INVALID
    # x in a wider array is not overwritten in place
    assert status("whtmix_norm_forward", [FAR[0], 0, FAR[2], FAR[0], 0], (4, 64, 80), (0,),
                  (1e-6,)) == INVALID


def test_no_rows_is_a_no_op():
    for name in ("whtmix_norm_forward", "whtmix_norm_mx_forward", "whtmix_quantize_mx",
                 "whtmix_dequantize_mx", "whtmix_linear_forward", "whtmix_linear_mx_forward"):
        n, sizes, codes, eps = GOOD[name]
        assert whtmix.call_rows(name, (0,) * n, (0, *sizes[1:]), codes, 0, *eps) == 0


def test_workspace_failure(monkeypatch):
    torch = pytest.importorskip("torch")
    if torch.cuda.device_count() > 0:
        pytest.skip("fake device addresses are for hosts without a GPU")
    monkeypatch.setenv("WHTMIX_TEST_FAIL_WORKSPACE", "1")
    for name in ("whtmix_norm_backward", "whtmix_linear_backward"):
        n, sizes, codes, eps = GOOD[name]
        assert status(name, pointers(name), sizes, codes, eps) == MEMORY
    assert "WHTMIX_TEST_FAIL_WORKSPACE" in whtmix.last_error()
    assert status("whtmix_linear_forward", pointers("whtmix_linear_forward"), (1, 4096, 64, 4096),
                  (0, 1), ()) == MEMORY


def test_call_module_refuses_what_no_entry_point_takes():
    m = whtmix._call()
    addr = ctypes.cast(whtmix.lib().whtmix_norm_forward, ctypes.c_void_p).value
    for args in ((addr, (0,) * 4, (0,) * 3, (0,), 0, 1e-6), (addr, (0,) * 5, (0,) * 3, (0,), 0),
                 (addr, (0,) * 10, (0,) * 3, (0,), 0), (addr, (0,) * 5, (0,) * 3, (0,)),
                 (addr, [0] * 5, (0,) * 3, (0,), 0, 1e-6), (addr,)):
        with pytest.raises(TypeError):
            m.call_rows(*args)
    with pytest.raises(TypeError):
        m.call_rows(addr, (0.5,) * 5, (1,) * 3, (0,), 0, 1e-6)
    with pytest.raises(OverflowError):
        m.call_rows(addr, (0,) * 5, (1 << 70,) * 3, (0,), 0, 1e-6)
    with pytest.raises(ValueError):
        m.call_rows(0, (0,) * 5, (1,) * 3, (0,), 0, 1e-6)


def test_python_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    x, w, g = torch.zeros(4, 64), torch.zeros(64, 32), torch.ones(64)
    for f in (lambda: whtmix.norm(x, g), lambda: whtmix.norm_mx(x, g),
              lambda: whtmix.norm_backward(x, g, x), lambda: whtmix.quantize_mx(x),
              lambda: whtmix.linear(x, w), lambda: whtmix.linear_backward(x, w, x),
              lambda: whtmix.dequantize_mx(x.to(torch.float8_e4m3fn), g.to(torch.uint8)),
              lambda: whtmix.linear_mx(x, g, w, g)):
        with pytest.raises(ValueError):
            f()


def test_rows_of_python_tensors():
    """(rows, width, ld) of what linear() and norm() take as x, and what they refuse."""
    torch = pytest.importorskip("torch")
    t = torch.zeros(3, 5, 40)
    assert whtmix._rows(t, "x") == (15, 40, 40)
    assert whtmix._rows(t[..., 8:24], "x") == (15, 16, 40)
    assert whtmix._rows(t[1], "x") == (5, 40, 40)
    assert whtmix._rows(t[:, 0], "x") == (3, 40, 200)
    assert whtmix._rows(t[:, 1:2, 3:9], "x") == (3, 6, 200)
    assert whtmix._rows(t[0:0], "x")[0] == 0
    assert whtmix._rows(t[:1, :1, 5:9], "x")[:2] == (1, 4)
    with pytest.raises(ValueError):
        whtmix._rows(t[:, :4], "x")             # rows not a constant distance apart
    with pytest.raises(ValueError):
        whtmix._rows(t.transpose(1, 2), "x")    # rows not contiguous
    with pytest.raises(ValueError):
        whtmix._rows(t[0, 0], "x")
    with pytest.raises(ValueError):
        whtmix._rows(t[:, :, ::2], "x")
    with pytest.raises(ValueError):
        whtmix._rows(t[:1].expand(4, 5, 40), "x")     # one row for many: overlapping
    with pytest.raises(ValueError):
        whtmix._activation("tanh")
    assert [whtmix.mx_width(c) for c in (1, 32, 33, 4096)] == [32, 32, 64, 4096]
