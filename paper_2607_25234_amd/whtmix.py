"""Python binding of the WHTMix C ABI (include/whtmix.h).

Argument marshalling only: every step of the mixer runs in the HIP kernels of
``libwhtmix.so``.  PyTorch supplies device memory and the current stream.
There is no fallback: if the library is missing, importing the functions
that need it raises.

    y = forward(x, gain)          # x [B, N, C] (or [N, C]) f32/bf16, gain [N, C] f32
    n, h = norm(y, weight, x)     # the residual's addition and a norm
    u = linear(n, w1, b1, activation="gelu")      # the feed-forward products
    o = linear(u, w2, b2, residual=h)
    e = embedding(ids, table, scale=8.0)          # rows of a table by token ids
    n, h = layer_norm(e, weight, bias)
    u = gated(n, w_gate, w_up, activation="silu")         # act(n w_gate) * (n w_up)
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libwhtmix.so")

SUCCESS = 0
DTYPE_F32, DTYPE_BF16 = 0, 1
PLANS = {"auto": 0, "small": 1, "fused": 2, "three_pass": 3, "one_launch": 4,
         "wave_tiles": 5, "two_pass": 6}
PLAN_NAMES = {v: k for k, v in PLANS.items()}

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
MX_BLOCK = 32
INDEX_I32, INDEX_I64 = 0, 1

# Every symbol include/whtmix.h declares.
EXPORTS = (
    "whtmix_backward",
    "whtmix_backward_separable",
    "whtmix_dequantize_mx",
    "whtmix_embedding_backward",
    "whtmix_embedding_forward",
    "whtmix_forward",
    "whtmix_forward_ex",
    "whtmix_forward_noalloc",
    "whtmix_forward_separable",
    "whtmix_gated_backward",
    "whtmix_gated_forward",
    "whtmix_gated_mx_forward",
    "whtmix_layer_norm_backward",
    "whtmix_layer_norm_forward",
    "whtmix_layer_norm_mx_forward",
    "whtmix_linear_backward",
    "whtmix_linear_forward",
    "whtmix_linear_mx_forward",
    "whtmix_module_backward",
    "whtmix_module_backward_separable",
    "whtmix_module_forward",
    "whtmix_module_forward_separable",
    "whtmix_norm_backward",
    "whtmix_norm_forward",
    "whtmix_norm_mx_forward",
    "whtmix_plan_describe",
    "whtmix_quantize_mx",
    "whtmix_status_string",
    "whtmix_last_error",
    "whtmix_release_workspaces",
    "whtmix_stream_status",
    "whtmix_version",
)
ERROR_DEVICE_TIMEOUT = 8


class WhtmixError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})"
                         + (f" [{last_error()}]" if last_error() else ""))


class Options(ctypes.Structure):
    _fields_ = [("plan", ctypes.c_int), ("events", ctypes.c_void_p * 4),
                ("spin_limit", ctypes.c_uint32)]


MODULE_PATHS = {0: "small", 1: "mfma", 2: "unfused"}


class PlanInfo(ctypes.Structure):
    _fields_ = [("plan", ctypes.c_int), ("kernels", ctypes.c_int),
                ("log2_slice", ctypes.c_int), ("outer_bits", ctypes.c_int),
                ("run_bits", ctypes.c_int), ("workspace_bytes", ctypes.c_int64),
                ("padded_tokens", ctypes.c_int64), ("module_path", ctypes.c_int),
                ("module_outer_bits", ctypes.c_int), ("module_backward_fused", ctypes.c_int)]


# The row operators' entry points: counts of pointers, sizes and int codes, and whether
# eps (the embedding's scale) stands before the codes.
_ROW_CALLS = {
    "whtmix_norm_forward": (5, 3, 1, True),
    "whtmix_norm_mx_forward": (6, 3, 1, True),
    "whtmix_norm_backward": (6, 2, 1, True),
    "whtmix_quantize_mx": (3, 3, 1, False),
    "whtmix_dequantize_mx": (3, 2, 1, False),
    "whtmix_linear_forward": (6, 4, 2, False),
    "whtmix_linear_backward": (7, 4, 2, False),
    "whtmix_linear_mx_forward": (9, 3, 2, False),
    "whtmix_layer_norm_forward": (6, 3, 1, True),
    "whtmix_layer_norm_mx_forward": (7, 3, 1, True),
    "whtmix_layer_norm_backward": (7, 2, 1, True),
    "whtmix_gated_forward": (8, 4, 2, False),
    "whtmix_gated_backward": (11, 4, 2, False),
    "whtmix_gated_mx_forward": (11, 3, 2, False),
    "whtmix_embedding_forward": (3, 3, 2, True),
    "whtmix_embedding_backward": (3, 3, 2, True),
}

_lib = None


def lib():
    """The loaded libwhtmix.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with "
                "`python -m paper_2607_25234_amd.build` (there is no fallback)")
        try:
            # Load torch's HIP runtime first so that the library binds to the
            # same runtime instance (same soname) as the tensors and streams.
            import torch  # noqa: F401
        except ImportError:
            pass
        L = ctypes.CDLL(LIB_PATH)
        i64, vp = ctypes.c_int64, ctypes.c_void_p
        L.whtmix_forward.argtypes = [vp, vp, vp, i64, i64, i64, ctypes.c_int, vp]
        L.whtmix_forward.restype = ctypes.c_int
        L.whtmix_forward_ex.argtypes = [vp, vp, vp, i64, i64, i64, ctypes.c_int, vp,
                                        ctypes.POINTER(Options)]
        L.whtmix_forward_ex.restype = ctypes.c_int
        L.whtmix_forward_noalloc.argtypes = [vp, vp, vp, i64, i64, i64, ctypes.c_int, vp]
        L.whtmix_forward_noalloc.restype = ctypes.c_int
        L.whtmix_forward_separable.argtypes = [vp, vp, vp, vp, i64, i64, i64, ctypes.c_int, vp,
                                               ctypes.POINTER(Options)]
        L.whtmix_forward_separable.restype = ctypes.c_int
        L.whtmix_module_forward.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ctypes.c_int,
                                            vp, ctypes.POINTER(Options)]
        L.whtmix_module_forward.restype = ctypes.c_int
        L.whtmix_module_forward_separable.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64,
                                                      ctypes.c_int, vp, ctypes.POINTER(Options)]
        L.whtmix_module_forward_separable.restype = ctypes.c_int
        L.whtmix_module_backward.argtypes = [vp] * 9 + [i64, i64, i64, ctypes.c_int, vp,
                                                         ctypes.POINTER(Options)]
        L.whtmix_module_backward.restype = ctypes.c_int
        L.whtmix_module_backward_separable.argtypes = [vp] * 11 + [i64, i64, i64, ctypes.c_int,
                                                                   vp, ctypes.POINTER(Options)]
        L.whtmix_module_backward_separable.restype = ctypes.c_int
        L.whtmix_backward.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ctypes.c_int, vp,
                                      ctypes.POINTER(Options)]
        L.whtmix_backward.restype = ctypes.c_int
        L.whtmix_backward_separable.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64,
                                                ctypes.c_int, vp, ctypes.POINTER(Options)]
        L.whtmix_backward_separable.restype = ctypes.c_int
        for name, (np, nz, nc, eps) in _ROW_CALLS.items():
            f = getattr(L, name)
            f.argtypes = ([vp] * np + [i64] * nz + ([ctypes.c_double] if eps else [])
                          + [ctypes.c_int] * nc + [vp])
            f.restype = ctypes.c_int
        L.whtmix_plan_describe.argtypes = [i64, i64, i64, ctypes.c_int,
                                           ctypes.POINTER(Options), ctypes.POINTER(PlanInfo)]
        L.whtmix_plan_describe.restype = ctypes.c_int
        L.whtmix_status_string.argtypes = [ctypes.c_int]
        L.whtmix_status_string.restype = ctypes.c_char_p
        L.whtmix_last_error.argtypes = []
        L.whtmix_last_error.restype = ctypes.c_char_p
        L.whtmix_release_workspaces.argtypes = []
        L.whtmix_release_workspaces.restype = ctypes.c_int
        L.whtmix_version.argtypes = []
        L.whtmix_version.restype = ctypes.c_int
        L.whtmix_stream_status.argtypes = [vp]
        L.whtmix_stream_status.restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().whtmix_status_string(status).decode()


def last_error() -> str:
    return lib().whtmix_last_error().decode()


def _options(plan: str | int = "auto", events=None, spin_limit: int = 0) -> Options:
    o = Options()
    o.plan = PLANS[plan] if isinstance(plan, str) else int(plan)
    for i, ev in enumerate(events or ()):
        o.events[i] = ev
    o.spin_limit = int(spin_limit)
    return o


def stream_status(stream: int | None = None) -> int:
    """whtmix_stream_status: synchronise the stream and return (and clear)
    the error word of its single-launch calls (SUCCESS or
    ERROR_DEVICE_TIMEOUT).  stream: a hipStream_t as int (default: torch's
    current stream)."""
    if stream is None:
        import torch
        stream = torch.cuda.current_stream().cuda_stream
    return int(lib().whtmix_stream_status(stream))


def plan_describe(B: int, N: int, C: int, dtype: str = "f32", plan: str | int = "auto") -> dict:
    """How a shape would run; raises WhtmixError on an invalid shape."""
    info = PlanInfo()
    opt = _options(plan)
    st = lib().whtmix_plan_describe(B, N, C, DTYPE_BF16 if dtype == "bf16" else DTYPE_F32,
                                    ctypes.byref(opt), ctypes.byref(info))
    if st != SUCCESS:
        raise WhtmixError(st, "whtmix_plan_describe")
    return {"plan": PLAN_NAMES[info.plan], "kernels": info.kernels,
            "log2_slice": info.log2_slice, "outer_bits": info.outer_bits,
            "run_bits": info.run_bits, "workspace_bytes": info.workspace_bytes,
            "padded_tokens": info.padded_tokens,
            "module_path": MODULE_PATHS.get(info.module_path),
            "module_outer_bits": info.module_outer_bits,
            "module_backward_fused": bool(info.module_backward_fused)}


_call_mod = None


def _call():
    """The CPython call module of the entry points
    (csrc/whtmix_pycall.c), bound to the functions of the loaded library.
    It is built with the library; there is no fallback."""
    global _call_mod
    if _call_mod is None:
        L = lib()
        try:
            from paper_2607_25234_amd import _whtmix_call as m
        except ImportError as e:
            raise ImportError("the binding's call module (_whtmix_call) is missing: build it "
                              "with `python -m paper_2607_25234_amd.build`") from e
        m.bind(ctypes.cast(L.whtmix_forward_ex, ctypes.c_void_p).value,
               ctypes.cast(L.whtmix_forward_separable, ctypes.c_void_p).value)
        _call_mod = m
    return _call_mod


_entry = {}


def _call_entry(name, *args, plan="auto", events=None) -> int:
    """The entry point `name` through the call module, by the address of the
    function in the loaded library."""
    addr = _entry.get(name)
    if addr is None:
        addr = _entry[name] = ctypes.cast(getattr(lib(), name), ctypes.c_void_p).value
    o, opt = _opt_address(plan, events, 0)
    try:
        st = _call().call(addr, *args, opt)
    except TypeError:   # a pointer given as a ctypes object: converted as ctypes does
        st = getattr(lib(), name)(*args, None if o is None else ctypes.byref(o))
    del o
    return st


def _opt_address(plan, events, spin_limit):
    """(structure, address) of the options argument; (None, 0) for NULL, when
    every option is its default (the library then takes AUTO, no events, the
    default spin limit).  The caller keeps the structure alive across the call."""
    if events is None and not spin_limit and (plan == "auto" or plan == 0):
        return None, 0
    o = _options(plan, events, spin_limit)
    return o, ctypes.addressof(o)


def forward_raw(x_ptr: int, gain_ptr: int, y_ptr: int, B: int, N: int, C: int,
                dtype: int, stream: int, plan: str | int = "auto", events=None,
                spin_limit: int = 0) -> int:
    """Direct call of whtmix_forward_ex with integer pointers; returns the status."""
    o, addr = _opt_address(plan, events, spin_limit)
    st = _call().forward_ex(x_ptr, gain_ptr, y_ptr, B, N, C, dtype, stream, addr)
    del o
    return st


def forward_noalloc_raw(x_ptr: int, gain_ptr: int, y_ptr: int, B: int, N: int, C: int,
                        dtype: int, stream: int) -> int:
    """Direct call of whtmix_forward_noalloc (the fixed-scratch variant that
    allocates nothing); returns the status."""
    return lib().whtmix_forward_noalloc(x_ptr, gain_ptr, y_ptr, B, N, C, dtype, stream)


def padded_tokens(N: int) -> int:
    """N_pad: rows N .. N_pad-1 are taken as zeros so that H_N acts on a
    power-of-two length (section III-B)."""
    return 1 << max(0, (int(N) - 1).bit_length())


def forward_separable_raw(x_ptr: int, gt_ptr: int, gc_ptr: int, y_ptr: int, B: int, N: int,
                          C: int, dtype: int, stream: int, plan: str | int = "auto",
                          events=None) -> int:
    """Direct call of whtmix_forward_separable; returns the status."""
    o, addr = _opt_address(plan, events, 0)
    st = _call().forward_separable(x_ptr, gt_ptr, gc_ptr, y_ptr, B, N, C, dtype, stream, addr)
    del o
    return st


def _check(x, out):
    import torch

    if not x.is_cuda:
        raise ValueError("x must be on a GPU device")
    if x.dtype is torch.float32:
        dt = DTYPE_F32
    elif x.dtype is torch.bfloat16:
        dt = DTYPE_BF16
    else:
        raise TypeError(f"x must be float32 or bfloat16, got {x.dtype}")
    xx = x.unsqueeze(0) if x.dim() == 2 else x
    if xx.dim() != 3:
        raise ValueError("x must be [B, N, C] or [N, C]")
    if not xx.is_contiguous():
        raise ValueError("x must be contiguous")
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype != x.dtype or not out.is_contiguous() \
            or out.device != x.device:
        raise ValueError("out must be a contiguous tensor like x")
    return xx, dt, out


def _gain(t, shape, x, what):
    import torch

    # get_device() is -1 on the CPU
    if t.get_device() != x.get_device() or t.dtype is not torch.float32 or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float32 tensor on x's device")
    if t.shape != shape:
        raise ValueError(f"{what} shape {tuple(t.shape)} != {tuple(shape)}")


_current = None


def _torch_current():
    """torch's functions that read the current device's index and the handle of a
    device's current stream: those that build no object (private to torch), or
    the public ones in a torch that has not got them."""
    global _current
    if _current is None:
        import torch

        device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        stream = (getattr(torch._C, "_cuda_getCurrentRawStream", None)
                  or (lambda i: torch.cuda.current_stream(i).cuda_stream))
        _current = device, stream
    return _current


def _on_device(x, stream, raw, ptrs, sizes, *options) -> int:
    """raw(*ptrs, *sizes, stream, *options) with x's device current, on `stream`
    or the device's current stream.  The device is switched only when it is
    not current already, and the stream's handle is read without building a
    Stream object: entering torch.cuda.device and torch.cuda.current_stream
    took 1.4 and 2.0 us of a 16 us call."""
    i = x.get_device()
    device, current_stream = _current or _torch_current()
    st = current_stream(i) if stream is None else stream.cuda_stream
    if device() == i:
        return raw(*ptrs, *sizes, st, *options)
    import torch

    with torch.cuda.device(i):
        return raw(*ptrs, *sizes, st, *options)


def forward(x, gain, out=None, plan: str | int = "auto", stream=None, events=None,
            spin_limit: int = 0):
    """y[b] = H_N (G o (H_N x[b] H_C)) H_C on the GPU (section III-B, eqs. (2)-(3)).

    x: torch tensor [B, N, C] or [N, C], float32 or bfloat16, on a ROCm device.
    gain: float32 [N_pad, C] (N_pad = N rounded up to a power of two; rows past
    N count as zeros) on the same device.  out: optional tensor like x (may
    be x itself for in-place).  stream: a torch.cuda.Stream (default: the
    current stream)."""
    xx, dt, out = _check(x, out)
    B, N, C = xx.shape
    _gain(gain, (padded_tokens(N), C), x, "gain")
    status = _on_device(x, stream, forward_raw,
                        (xx.data_ptr(), gain.data_ptr(), out.data_ptr()), (B, N, C, dt), plan,
                        events, spin_limit)
    if status != SUCCESS:
        raise WhtmixError(status, "whtmix_forward")
    return out


def forward_separable(x, log_gain_tokens, log_gain_channels, out=None,
                      plan: str | int = "auto", stream=None, events=None):
    """The paper's parametrisation (eq. (2) then eq. (3)) with log-domain gains:
    log_gain_tokens float32 [N_pad], log_gain_channels float32 [C]."""
    xx, dt, out = _check(x, out)
    B, N, C = xx.shape
    _gain(log_gain_tokens, (padded_tokens(N),), x, "log_gain_tokens")
    _gain(log_gain_channels, (C,), x, "log_gain_channels")
    status = _on_device(x, stream, forward_separable_raw,
                        (xx.data_ptr(), log_gain_tokens.data_ptr(),
                         log_gain_channels.data_ptr(), out.data_ptr()), (B, N, C, dt), plan,
                        events)
    if status != SUCCESS:
        raise WhtmixError(status, "whtmix_forward_separable")
    return out


def module_forward_raw(x_ptr: int, w_in_ptr: int, gain_ptr: int, w_out_ptr: int, y_ptr: int,
                       B: int, N: int, C: int, dtype: int, stream: int,
                       plan: str | int = "auto", events=None) -> int:
    """Direct call of whtmix_module_forward; returns the status."""
    return _call_entry("whtmix_module_forward", x_ptr, w_in_ptr, gain_ptr, w_out_ptr, y_ptr,
                       B, N, C, dtype, stream, plan=plan, events=events)


def module_forward_separable_raw(x_ptr: int, w_in_ptr: int, gt_ptr: int, gc_ptr: int,
                                 w_out_ptr: int, y_ptr: int, B: int, N: int, C: int,
                                 dtype: int, stream: int, plan: str | int = "auto",
                                 events=None) -> int:
    """Direct call of whtmix_module_forward_separable; returns the status."""
    return _call_entry("whtmix_module_forward_separable", x_ptr, w_in_ptr, gt_ptr, gc_ptr,
                       w_out_ptr, y_ptr, B, N, C, dtype, stream, plan=plan, events=events)


def _weight(w, C, x, what):
    if w.get_device() != x.get_device() or w.dtype is not x.dtype or not w.is_contiguous():
        raise ValueError(f"{what} must be a contiguous tensor of x's dtype on x's device")
    if w.shape != (C, C):
        raise ValueError(f"{what} shape {tuple(w.shape)} != {(C, C)}")


def module_forward(x, w_in, gain, w_out, out=None, plan: str | int = "auto", stream=None,
                   events=None):
    """The whole block of section III-B, eqs. (1)-(4): Y = mixer(X W_in) W_out with
    the joint gain.  w_in, w_out: [C, C] tensors of x's dtype (Z[n][j] = sum_i
    X[n][i] W_in[i][j]); gain: float32 [N_pad, C]."""
    xx, dt, out = _check(x, out)
    B, N, C = xx.shape
    _weight(w_in, C, x, "w_in")
    _weight(w_out, C, x, "w_out")
    _gain(gain, (padded_tokens(N), C), x, "gain")
    status = _on_device(x, stream, module_forward_raw,
                        (xx.data_ptr(), w_in.data_ptr(), gain.data_ptr(), w_out.data_ptr(),
                         out.data_ptr()), (B, N, C, dt), plan, events)
    if status != SUCCESS:
        raise WhtmixError(status, "whtmix_module_forward")
    return out


def module_forward_separable(x, w_in, log_gain_tokens, log_gain_channels, w_out, out=None,
                             plan: str | int = "auto", stream=None, events=None):
    """The whole block with the paper's log-domain gains (eqs. (1)-(4))."""
    xx, dt, out = _check(x, out)
    B, N, C = xx.shape
    _weight(w_in, C, x, "w_in")
    _weight(w_out, C, x, "w_out")
    _gain(log_gain_tokens, (padded_tokens(N),), x, "log_gain_tokens")
    _gain(log_gain_channels, (C,), x, "log_gain_channels")
    status = _on_device(x, stream, module_forward_separable_raw,
                        (xx.data_ptr(), w_in.data_ptr(), log_gain_tokens.data_ptr(),
                         log_gain_channels.data_ptr(), w_out.data_ptr(), out.data_ptr()),
                        (B, N, C, dt), plan, events)
    if status != SUCCESS:
        raise WhtmixError(status, "whtmix_module_forward_separable")
    return out


def backward_raw(x_ptr, dy_ptr, gain_ptr, dx_ptr, dgain_ptr, B, N, C, dtype, stream,
                 plan: str | int = "auto", events=None) -> int:
    """Direct call of whtmix_backward (0 for a skipped output); returns the status."""
    return _call_entry("whtmix_backward", x_ptr, dy_ptr, gain_ptr, dx_ptr, dgain_ptr, B, N, C,
                       dtype, stream, plan=plan, events=events)


def backward_separable_raw(x_ptr, dy_ptr, gt_ptr, gc_ptr, dx_ptr, dgt_ptr, dgc_ptr, B, N, C,
                           dtype, stream, plan: str | int = "auto", events=None) -> int:
    """Direct call of whtmix_backward_separable; returns the status."""
    return _call_entry("whtmix_backward_separable", x_ptr, dy_ptr, gt_ptr, gc_ptr, dx_ptr,
                       dgt_ptr, dgc_ptr, B, N, C, dtype, stream, plan=plan, events=events)


def _same(a, x, what):
    if a.shape != x.shape or a.dtype != x.dtype or a.device != x.device or not a.is_contiguous():
        raise ValueError(f"{what} must be a contiguous tensor like x")


def backward(x, dy, gain, want_dx: bool = True, want_dgain: bool = True, dx=None,
             plan: str | int = "auto", stream=None):
    """Gradients through forward(x, gain) for the upstream gradient dy:
    returns (dx, dgain); dx = the mixer applied to dy, dgain [N_pad, C]
    float32 = sum_b T(x_b) o T(dy_b).  An output not wanted is None."""
    import torch

    xx, dt, _ = _check(x, x)
    _same(dy, x, "dy")
    B, N, C = xx.shape
    _gain(gain, (padded_tokens(N), C), x, "gain")
    if want_dx and dx is None:
        dx = torch.empty_like(dy)
    if dx is not None:
        _same(dx, x, "dx")
    dgain = torch.empty_like(gain) if want_dgain else None
    if dx is None and dgain is None:
        raise ValueError("nothing to compute")
    status = _on_device(x, stream, backward_raw,
                        (xx.data_ptr(), dy.data_ptr(), gain.data_ptr(),
                         dx.data_ptr() if dx is not None else 0,
                         dgain.data_ptr() if dgain is not None else 0), (B, N, C, dt), plan)
    if status != SUCCESS:
        raise WhtmixError(status, "whtmix_backward")
    return dx, dgain


def backward_separable(x, dy, log_gain_tokens, log_gain_channels, want_dx: bool = True,
                       want_dgains: bool = True, dx=None, plan: str | int = "auto",
                       stream=None):
    """Gradients through forward_separable: returns (dx, d_log_gain_tokens,
    d_log_gain_channels); outputs not wanted are None."""
    import torch

    xx, dt, _ = _check(x, x)
    _same(dy, x, "dy")
    B, N, C = xx.shape
    _gain(log_gain_tokens, (padded_tokens(N),), x, "log_gain_tokens")
    _gain(log_gain_channels, (C,), x, "log_gain_channels")
    if want_dx and dx is None:
        dx = torch.empty_like(dy)
    if dx is not None:
        _same(dx, x, "dx")
    dgt = torch.empty_like(log_gain_tokens) if want_dgains else None
    dgc = torch.empty_like(log_gain_channels) if want_dgains else None
    if dx is None and dgt is None:
        raise ValueError("nothing to compute")
    status = _on_device(x, stream, backward_separable_raw,
                        (xx.data_ptr(), dy.data_ptr(), log_gain_tokens.data_ptr(),
                         log_gain_channels.data_ptr(), dx.data_ptr() if dx is not None else 0,
                         dgt.data_ptr() if dgt is not None else 0,
                         dgc.data_ptr() if dgc is not None else 0), (B, N, C, dt), plan)
    if status != SUCCESS:
        raise WhtmixError(status, "whtmix_backward_separable")
    return dx, dgt, dgc


def module_backward_raw(x_ptr, w_in_ptr, gain_ptr, w_out_ptr, dy_ptr, dx_ptr, dw_in_ptr,
                        dw_out_ptr, dgain_ptr, B, N, C, dtype, stream,
                        plan: str | int = "auto", events=None) -> int:
    """Direct call of whtmix_module_backward; returns the status."""
    return _call_entry("whtmix_module_backward", x_ptr, w_in_ptr, gain_ptr, w_out_ptr, dy_ptr,
                       dx_ptr, dw_in_ptr, dw_out_ptr, dgain_ptr, B, N, C, dtype, stream,
                       plan=plan, events=events)


def module_backward_separable_raw(x_ptr, w_in_ptr, gt_ptr, gc_ptr, w_out_ptr, dy_ptr, dx_ptr,
                                  dw_in_ptr, dw_out_ptr, dgt_ptr, dgc_ptr, B, N, C, dtype,
                                  stream, plan: str | int = "auto", events=None) -> int:
    """Direct call of whtmix_module_backward_separable; returns the status."""
    return _call_entry("whtmix_module_backward_separable", x_ptr, w_in_ptr, gt_ptr, gc_ptr,
                       w_out_ptr, dy_ptr, dx_ptr, dw_in_ptr, dw_out_ptr, dgt_ptr, dgc_ptr,
                       B, N, C, dtype, stream, plan=plan, events=events)


def module_backward(x, w_in, gain, w_out, dy, want_dgain: bool = True, dx=None,
                    plan: str | int = "auto", stream=None):
    """Gradients through module_forward for the upstream gradient dy: returns
    (dx, dw_in, dw_out, dgain), the weight and gain gradients in float32
    (dgain None when not wanted)."""
    import torch

    xx, dt, _ = _check(x, x)
    _same(dy, x, "dy")
    B, N, C = xx.shape
    _weight(w_in, C, x, "w_in")
    _weight(w_out, C, x, "w_out")
    _gain(gain, (padded_tokens(N), C), x, "gain")
    if dx is None:
        dx = torch.empty_like(dy)
    _same(dx, x, "dx")
    f32 = dict(dtype=torch.float32, device=x.device)
    dw_in, dw_out = torch.empty((C, C), **f32), torch.empty((C, C), **f32)
    dgain = torch.empty_like(gain) if want_dgain else None
    status = _on_device(x, stream, module_backward_raw,
                        (xx.data_ptr(), w_in.data_ptr(), gain.data_ptr(), w_out.data_ptr(),
                         dy.data_ptr(), dx.data_ptr(), dw_in.data_ptr(), dw_out.data_ptr(),
                         dgain.data_ptr() if dgain is not None else 0), (B, N, C, dt), plan)
    if status != SUCCESS:
        raise WhtmixError(status, "whtmix_module_backward")
    return dx, dw_in, dw_out, dgain


def module_backward_separable(x, w_in, log_gain_tokens, log_gain_channels, w_out, dy,
                              want_dgains: bool = True, dx=None, plan: str | int = "auto",
                              stream=None):
    """Gradients through module_forward_separable: returns (dx, dw_in, dw_out,
    d_log_gain_tokens, d_log_gain_channels)."""
    import torch

    xx, dt, _ = _check(x, x)
    _same(dy, x, "dy")
    B, N, C = xx.shape
    _weight(w_in, C, x, "w_in")
    _weight(w_out, C, x, "w_out")
    _gain(log_gain_tokens, (padded_tokens(N),), x, "log_gain_tokens")
    _gain(log_gain_channels, (C,), x, "log_gain_channels")
    if dx is None:
        dx = torch.empty_like(dy)
    _same(dx, x, "dx")
    f32 = dict(dtype=torch.float32, device=x.device)
    dw_in, dw_out = torch.empty((C, C), **f32), torch.empty((C, C), **f32)
    dgt = torch.empty_like(log_gain_tokens) if want_dgains else None
    dgc = torch.empty_like(log_gain_channels) if want_dgains else None
    status = _on_device(x, stream, module_backward_separable_raw,
                        (xx.data_ptr(), w_in.data_ptr(), log_gain_tokens.data_ptr(),
                         log_gain_channels.data_ptr(), w_out.data_ptr(), dy.data_ptr(),
                         dx.data_ptr(), dw_in.data_ptr(), dw_out.data_ptr(),
                         dgt.data_ptr() if dgt is not None else 0,
                         dgc.data_ptr() if dgc is not None else 0), (B, N, C, dt), plan)
    if status != SUCCESS:
        raise WhtmixError(status, "whtmix_module_backward_separable")
    return dx, dw_in, dw_out, dgt, dgc


# ---- the feed-forward sublayer ----

def call_rows(name, pointers, sizes, codes, stream, *eps) -> int:
    """Direct call of a feed-forward entry point with integer pointers (0 for
    none), its sizes and its int codes in the header's order; returns the status."""
    addr = _entry.get(name)
    if addr is None:
        addr = _entry[name] = ctypes.cast(getattr(lib(), name), ctypes.c_void_p).value
    return _call().call_rows(addr, pointers, sizes, codes, stream, *eps)


def _run_rows(name, dev, stream, pointers, sizes, codes, *eps):
    """The entry point on device number dev, on `stream` or its current stream; raises
    WhtmixError on a refusal."""
    device, current_stream = _current or _torch_current()
    st = current_stream(dev) if stream is None else stream.cuda_stream
    if device() == dev:
        status = call_rows(name, pointers, sizes, codes, st, *eps)
    else:
        with _torch().cuda.device(dev):
            status = call_rows(name, pointers, sizes, codes, st, *eps)
    if status != SUCCESS:
        raise WhtmixError(status, name)


_torch_module = None


def _torch():
    """torch, imported on first use (an import statement in a call takes 0.3 us)."""
    global _torch_module
    if _torch_module is None:
        import torch
        # the codes first: another thread takes the module for the sign that they are there
        _CODES.update({torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16})
        _INDEX.update({torch.int32: INDEX_I32, torch.int64: INDEX_I64})
        _torch_module = torch
    return _torch_module


_CODES = {}
_INDEX = {}


def _operand(t, what):
    """(dtype code, rows, width, ld, device number) of x: a float32 or bfloat16 tensor
    [..., C] on a GPU whose rows are contiguous and a constant distance apart (columns of
    a wider tensor, or contiguous)."""
    _torch_module or _torch()
    if not t.is_cuda:
        raise ValueError(f"{what} must be on a GPU device")
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be float32 or bfloat16, got {t.dtype}")
    return (code, *_rows(t, what), t.get_device())


def _rows(t, what):
    """(rows, width, ld) of a tensor [..., C] whose rows are a constant distance apart."""
    if t.dim() < 2:
        raise ValueError(f"{what} must be [..., rows, columns]")
    C = t.shape[-1]
    if t.is_contiguous():
        return (t.numel() // C if C else 0), C, C
    if t.stride(-1) != 1 and C != 1:
        raise ValueError(f"{what}'s rows must be contiguous")
    ld, rows = t.stride(-2), t.shape[-2]
    if rows == 1 and t.dim() == 2:
        ld = max(ld, C)
    for size, stride in zip(reversed(t.shape[:-2]), reversed(t.stride()[:-2])):
        if rows == 1:
            ld = stride
        elif size != 1 and stride != rows * ld:
            raise ValueError(f"{what}'s rows must be a constant distance apart")
        rows *= size
    return rows, C, max(ld, C) if rows <= 1 else ld


def _tensor(t, shape, dtype, dev, what):
    """The address of a contiguous tensor of this shape and dtype on device dev."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    if t.shape != shape:
        raise ValueError(f"{what} shape {tuple(t.shape)} != {tuple(shape)}")
    raise ValueError(f"{what} must be a contiguous {dtype} tensor on x's device")


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _activation(name):
    code = ACTIVATIONS.get(name)
    if code is None:
        raise ValueError(f"activation {name!r}: one of {', '.join(ACTIVATIONS)}")
    return code


def mx_width(C: int) -> int:
    """Values stored for a row of C in block-scaled 8 bits."""
    return -(-C // MX_BLOCK) * MX_BLOCK


def _new_mx(x, lead, C):
    T, w = _torch(), mx_width(C)
    return (x.new_empty((*lead, w), dtype=T.float8_e4m3fn),
            x.new_empty((*lead, w // MX_BLOCK), dtype=T.uint8))


def _mx(q, scales, what):
    """(rows, stored width, the two addresses, device number) of block-scaled rows."""
    T = _torch_module or _torch()
    if not q.is_cuda:
        raise ValueError(f"{what} must be on a GPU device")
    if q.dtype is not T.float8_e4m3fn or q.dim() < 2 or not q.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float8_e4m3fn tensor [..., rows, columns]")
    w, dev = q.shape[-1], q.get_device()
    if w % MX_BLOCK or w == 0:
        raise ValueError(f"{what}'s width {w} is not a multiple of {MX_BLOCK}")
    return (q.numel() // w, w, q.data_ptr(),
            _tensor(scales, (*q.shape[:-1], w // MX_BLOCK), T.uint8, dev, f"{what}'s scales"), dev)


def norm(x, weight, residual=None, eps: float = 1e-6, out=None, stream=None):
    """Root-mean-square norm with the residual's addition: (y, h) with
    h = x + residual (x itself without one) and
    y = h / sqrt(mean(h^2) + eps) * weight, formed before h is rounded.

    x: [..., C] float32 or bfloat16 (rows may be columns of a wider tensor);
    weight: float32 [C]; residual: a contiguous tensor of x's shape and type;
    out: optional contiguous tensor for y (may be x itself; without a residual
    h is None then, since x holds y)."""
    T = _torch_module or _torch()
    dt, rows, C, ld, dev = _operand(x, "x")
    shape, dtype = x.shape, x.dtype
    pw = _tensor(weight, (C,), T.float32, dev, "weight")
    h, pr, ph = x, 0, 0
    if residual is not None:
        pr = _tensor(residual, shape, dtype, dev, "residual")
        h = T.empty_like(residual)
        ph = h.data_ptr()
    if out is None:
        out = T.empty_like(x, memory_format=T.contiguous_format)
        py = out.data_ptr()
    else:
        py = _tensor(out, shape, dtype, dev, "out")
        if residual is None and py == x.data_ptr():
            h = None
    _run_rows("whtmix_norm_forward", dev, stream, (x.data_ptr(), pr, pw, py, ph), (rows, C, ld),
              (dt,), eps)
    return out, h


def norm_mx(x, weight, residual=None, eps: float = 1e-6, stream=None):
    """norm() with y in block-scaled 8 bits: (q, scales, h), q float8_e4m3fn
    [..., mx_width(C)] and scales uint8 [..., mx_width(C) / 32]; a value is
    q * 2^(scale - 127)."""
    T = _torch_module or _torch()
    dt, rows, C, ld, dev = _operand(x, "x")
    shape = x.shape
    pw = _tensor(weight, (C,), T.float32, dev, "weight")
    h, pr, ph = x, 0, 0
    if residual is not None:
        pr = _tensor(residual, shape, x.dtype, dev, "residual")
        h = T.empty_like(residual)
        ph = h.data_ptr()
    q, scales = _new_mx(x, shape[:-1], C)
    _run_rows("whtmix_norm_mx_forward", dev, stream,
              (x.data_ptr(), pr, pw, q.data_ptr(), scales.data_ptr(), ph), (rows, C, ld), (dt,),
              eps)
    return q, scales, h


def norm_backward(h, weight, dy, dh=None, eps: float = 1e-6, want_dweight: bool = True, dx=None,
                  stream=None):
    """Gradients through norm() from its kept h: (dx, dweight), dx the gradient
    of x and of the residual (dh, the gradient of h, is added), dweight float32
    (None when not wanted).  dx may be dy or dh."""
    T = _torch_module or _torch()
    dt, rows, C, _, dev = _operand(h, "h")
    shape, dtype = h.shape, h.dtype
    ptr = (_tensor(h, shape, dtype, dev, "h"), _tensor(weight, (C,), T.float32, dev, "weight"),
           _tensor(dy, shape, dtype, dev, "dy"),
           0 if dh is None else _tensor(dh, shape, dtype, dev, "dh"))
    if dx is None:
        dx = T.empty_like(h)
    dweight = T.empty_like(weight) if want_dweight else None
    _run_rows("whtmix_norm_backward", dev, stream,
              (*ptr, _tensor(dx, shape, dtype, dev, "dx"), _ptr(dweight)), (rows, C), (dt,), eps)
    return dx, dweight


def quantize_mx(x, stream=None):
    """x [..., C] in block-scaled 8 bits along its rows: (q, scales) as norm_mx.
    Weights [K, N] are laid out once by their columns: quantize_mx(w.t())
    after .contiguous()."""
    dt, rows, C, ld, dev = _operand(x, "x")
    q, scales = _new_mx(x, x.shape[:-1], C)
    _run_rows("whtmix_quantize_mx", dev, stream, (x.data_ptr(), q.data_ptr(), scales.data_ptr()),
              (rows, C, ld), (dt,))
    return q, scales


def dequantize_mx(q, scales, C: int | None = None, dtype=None, stream=None):
    """The values q and scales stand for, [..., C] (default: the stored width)
    in dtype (bfloat16, the default, or float32)."""
    T = _torch_module or _torch()
    dtype = dtype or T.bfloat16
    code = _CODES.get(dtype)
    if stream is None and C is not None and code is not None:
        r = (_ordinary_module or _ordinary()).dequantize_mx(q, scales, C, code)
        if r is not None:
            return _taken(r, "dequantize_mx")[0]
    rows, w, pq, ps, dev = _mx(q, scales, "q")
    C = w if C is None else C
    if mx_width(C) != w:
        raise ValueError(f"{C} columns are not stored in {w}")
    if code is None:
        raise TypeError(f"the output must be float32 or bfloat16, not {dtype}")
    y = q.new_empty((*q.shape[:-1], C), dtype=dtype)
    _run_rows("whtmix_dequantize_mx", dev, stream, (pq, ps, y.data_ptr()), (rows, C), (code,))
    return y


def linear(x, w, bias=None, activation: str = "none", residual=None, want_z: bool = False,
           out=None, stream=None):
    """activation(x w + bias) + residual; with want_z also z = x w + bias, which
    linear_backward reads: (y, z).

    x: [..., K] float32 or bfloat16 (rows may be columns of a wider tensor);
    w: [K, N] of x's type; bias: float32 [N]; residual: a contiguous [..., N]
    of x's type; activation: "none", "relu", "gelu", "gelu_tanh" or "silu"; out:
    optional contiguous tensor for y (may be the residual)."""
    T = _torch_module or _torch()
    dt, M, K, ld, dev = _operand(x, "x")
    act, dtype = _activation(activation), x.dtype
    if w.dim() != 2:
        raise ValueError("w must be [K, N]")
    N = w.shape[1]
    pw = _tensor(w, (K, N), dtype, dev, "w")
    shape = (*x.shape[:-1], N)
    pb = 0 if bias is None else _tensor(bias, (N,), T.float32, dev, "bias")
    pr = 0 if residual is None else _tensor(residual, shape, dtype, dev, "residual")
    if out is None:
        out = x.new_empty(shape)
        py = out.data_ptr()
    else:
        py = _tensor(out, shape, dtype, dev, "out")
    z = T.empty_like(out) if want_z else None
    _run_rows("whtmix_linear_forward", dev, stream, (x.data_ptr(), pw, pb, pr, py, _ptr(z)),
              (M, K, N, ld), (act, dt))
    return (out, z) if want_z else out


def linear_backward(x, w, dy, z=None, activation: str = "none", want_dx: bool = True,
                    want_dw: bool = True, want_dbias: bool = True, stream=None):
    """Gradients through linear() for the upstream gradient dy: (dx, dw, dbias),
    dx and dw in x's type, dbias float32; what is not wanted is None.  z: what
    linear kept (not needed for activation "none").  The residual's gradient is dy."""
    T = _torch_module or _torch()
    dt, M, K, ld, dev = _operand(x, "x")
    act, dtype = _activation(activation), x.dtype
    if w.dim() != 2:
        raise ValueError("w must be [K, N]")
    N = w.shape[1]
    pw = _tensor(w, (K, N), dtype, dev, "w")
    shape = (*x.shape[:-1], N)
    pdy = _tensor(dy, shape, dtype, dev, "dy")
    pz = 0
    if act:
        if z is None:
            raise ValueError(f"activation {activation!r} needs z")
        pz = _tensor(z, shape, dtype, dev, "z")
    if not (want_dx or want_dw or want_dbias):
        raise ValueError("nothing to compute")
    dx = T.empty_like(x, memory_format=T.contiguous_format) if want_dx else None
    dw = T.empty_like(w) if want_dw else None
    db = x.new_empty(N, dtype=T.float32) if want_dbias else None
    _run_rows("whtmix_linear_backward", dev, stream,
              (x.data_ptr(), pw, pdy, pz, _ptr(dx), _ptr(dw), _ptr(db)), (M, K, N, ld), (act, dt))
    return dx, dw, db


def linear_mx(xq, xs, wq, ws, bias=None, activation: str = "none", residual=None,
              out_mx: bool = False, dtype=None, out=None, stream=None):
    """linear() on block-scaled 8 bits: xq, xs as norm_mx or quantize_mx give
    them, [..., K]; wq, ws the weights' columns as rows, [N, K].  Returns y
    [..., N] in dtype (the residual's or out's, else bfloat16), or with out_mx
    (q, scales) of the result.  Sums of more than 512 k are float32 throughout
    only for a float32 y (the others: up to 1e-5 of the sum of magnitudes off)."""
    T = _torch_module or _torch()
    M, K, pxq, pxs, dev = _mx(xq, xs, "xq")
    act = _activation(activation)
    if wq.dim() != 2:
        raise ValueError("wq must be [N, K]")
    N, Kw, pwq, pws, wdev = _mx(wq, ws, "wq")
    if Kw != K or wdev != dev:
        raise ValueError(f"wq must hold rows of {K} on xq's device")
    lead = xq.shape[:-1]
    pb = 0 if bias is None else _tensor(bias, (N,), T.float32, dev, "bias")
    if dtype is None:
        like = residual if residual is not None else out
        dtype = like.dtype if like is not None else T.bfloat16
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"the output must be float32 or bfloat16, not {dtype}")
    pr = 0 if residual is None else _tensor(residual, (*lead, N), dtype, dev, "residual")
    q = s = None
    if out_mx:
        if out is not None:
            raise ValueError("out is for outputs that are not in 8 bits")
        q, s = _new_mx(xq, lead, N)
    elif out is None:
        out = xq.new_empty((*lead, N), dtype=dtype)
    else:
        _tensor(out, (*lead, N), dtype, dev, "out")
    _run_rows("whtmix_linear_mx_forward", dev, stream,
              (pxq, pxs, pwq, pws, pb, pr, _ptr(out), _ptr(q), _ptr(s)), (M, K, N), (act, code))
    return (q, s) if out_mx else out


# ---- layer norm, gated products, embedding ----

_ORDINARY = ("layer_norm_forward", "layer_norm_mx_forward", "layer_norm_backward", "gated_forward",
             "gated_backward", "gated_mx_forward", "embedding_forward", "embedding_backward",
             "dequantize_mx")
_ordinary_module = None


class _NotBuilt:
    """In the place of the module below where it is not built: no call is taken."""

    def __getattr__(self, name):
        return lambda *args: None


def _ordinary():
    """The module (csrc/whtmix_torch.cc) that makes ordinary calls of these functions in C++:
    checks, allocations and the entry point, 2 to 4 us a call less than here.  Its functions
    return None for calls that they leave to the code here, and a status that is not
    success as an int."""
    global _ordinary_module
    if _ordinary_module is None:
        T, L = _torch(), lib()
        try:
            from paper_2607_25234_amd import _whtmix_torch as m
        except ImportError:
            m = _NotBuilt()
        else:
            m.bind(tuple(ctypes.cast(getattr(L, "whtmix_" + name), ctypes.c_void_p).value
                         for name in _ORDINARY), T.nn.Parameter)
        _ordinary_module = m
    return _ordinary_module


def _taken(result, name):
    """An ordinary call's tensors."""
    if type(result) is int:
        raise WhtmixError(result, "whtmix_" + name)
    return result


def layer_norm(x, weight, bias=None, residual=None, eps: float = 1e-6, out=None, stream=None):
    """Layer norm with the residual's addition: (y, h) with h = x + residual (x itself
    without one) and y = (h - mean(h)) / sqrt(mean((h - mean(h))^2) + eps) * weight + bias,
    formed before h is rounded.

    x: [..., C] float32 or bfloat16 (rows may be columns of a wider tensor);
    weight, bias: float32 [C]; residual: a contiguous tensor of x's shape and type;
    out: optional contiguous tensor for y (may be x itself; without a residual
    h is None then, since x holds y)."""
    if out is None and stream is None:
        r = (_ordinary_module or _ordinary()).layer_norm(x, weight, bias, residual, eps)
        if r is not None:
            return _taken(r, "layer_norm_forward")
    T = _torch_module or _torch()
    dt, rows, C, ld, dev = _operand(x, "x")
    shape, dtype = x.shape, x.dtype
    pw = _tensor(weight, (C,), T.float32, dev, "weight")
    pb = 0 if bias is None else _tensor(bias, (C,), T.float32, dev, "bias")
    h, pr, ph = x, 0, 0
    if residual is not None:
        pr = _tensor(residual, shape, dtype, dev, "residual")
        h = T.empty_like(residual)
        ph = h.data_ptr()
    if out is None:
        out = T.empty_like(x, memory_format=T.contiguous_format)
        py = out.data_ptr()
    else:
        py = _tensor(out, shape, dtype, dev, "out")
        if residual is None and py == x.data_ptr():
            h = None
    _run_rows("whtmix_layer_norm_forward", dev, stream, (x.data_ptr(), pr, pw, pb, py, ph),
              (rows, C, ld), (dt,), eps)
    return out, h


def layer_norm_mx(x, weight, bias=None, residual=None, eps: float = 1e-6, stream=None):
    """layer_norm() with y in block-scaled 8 bits: (q, scales, h), q and scales as norm_mx."""
    if stream is None:
        r = (_ordinary_module or _ordinary()).layer_norm_mx(x, weight, bias, residual, eps)
        if r is not None:
            return _taken(r, "layer_norm_mx_forward")
    T = _torch_module or _torch()
    dt, rows, C, ld, dev = _operand(x, "x")
    shape = x.shape
    pw = _tensor(weight, (C,), T.float32, dev, "weight")
    pb = 0 if bias is None else _tensor(bias, (C,), T.float32, dev, "bias")
    h, pr, ph = x, 0, 0
    if residual is not None:
        pr = _tensor(residual, shape, x.dtype, dev, "residual")
        h = T.empty_like(residual)
        ph = h.data_ptr()
    q, scales = _new_mx(x, shape[:-1], C)
    _run_rows("whtmix_layer_norm_mx_forward", dev, stream,
              (x.data_ptr(), pr, pw, pb, q.data_ptr(), scales.data_ptr(), ph), (rows, C, ld),
              (dt,), eps)
    return q, scales, h


def layer_norm_backward(h, weight, dy, dh=None, eps: float = 1e-6, want_dweight: bool = True,
                        want_dbias: bool = True, dx=None, stream=None):
    """Gradients through layer_norm() from its kept h: (dx, dweight, dbias), dx the gradient
    of x and of the residual (dh, the gradient of h, is added), the others float32 (None
    when not wanted).  dx may be dy or dh."""
    if dx is None and stream is None:
        r = (_ordinary_module or _ordinary()).layer_norm_backward(h, weight, dy, dh, eps,
                                                                 want_dweight, want_dbias)
        if r is not None:
            return _taken(r, "layer_norm_backward")
    T = _torch_module or _torch()
    dt, rows, C, _, dev = _operand(h, "h")
    shape, dtype = h.shape, h.dtype
    ptr = (_tensor(h, shape, dtype, dev, "h"), _tensor(weight, (C,), T.float32, dev, "weight"),
           _tensor(dy, shape, dtype, dev, "dy"),
           0 if dh is None else _tensor(dh, shape, dtype, dev, "dh"))
    if dx is None:
        dx = T.empty_like(h)
    dweight = T.empty_like(weight) if want_dweight else None
    dbias = T.empty_like(weight) if want_dbias else None
    _run_rows("whtmix_layer_norm_backward", dev, stream,
              (*ptr, _tensor(dx, shape, dtype, dev, "dx"), _ptr(dweight), _ptr(dbias)), (rows, C),
              (dt,), eps)
    return dx, dweight, dbias


def _gates(x, w_gate, w_up, K, dev):
    """(N, the weights' addresses) of a gated product's weights."""
    if w_gate.dim() != 2:
        raise ValueError("w_gate must be [K, N]")
    N = w_gate.shape[1]
    return (N, _tensor(w_gate, (K, N), x.dtype, dev, "w_gate"),
            _tensor(w_up, (K, N), x.dtype, dev, "w_up"))


def gated(x, w_gate, w_up, b_gate=None, b_up=None, activation: str = "silu",
          want_z: bool = False, out=None, stream=None):
    """activation(x w_gate + b_gate) * (x w_up + b_up), both products in one kernel; with
    want_z also both products with their biases, which gated_backward reads: (y, z_gate, z_up).

    x: [..., K] float32 or bfloat16 (rows may be columns of a wider tensor); w_gate, w_up:
    [K, N] of x's type; b_gate, b_up: float32 [N]; activation as linear's; out: optional
    contiguous [..., N] tensor for y."""
    if out is None and stream is None:
        r = (_ordinary_module or _ordinary()).gated(x, w_gate, w_up, b_gate, b_up,
                                                   _activation(activation), want_z)
        if r is not None:
            return _taken(r, "gated_forward") if want_z else _taken(r, "gated_forward")[0]
    T = _torch_module or _torch()
    dt, M, K, ld, dev = _operand(x, "x")
    act, dtype = _activation(activation), x.dtype
    N, pg, pu = _gates(x, w_gate, w_up, K, dev)
    shape = (*x.shape[:-1], N)
    pbg = 0 if b_gate is None else _tensor(b_gate, (N,), T.float32, dev, "b_gate")
    pbu = 0 if b_up is None else _tensor(b_up, (N,), T.float32, dev, "b_up")
    if out is None:
        out = x.new_empty(shape)
        py = out.data_ptr()
    else:
        py = _tensor(out, shape, dtype, dev, "out")
    zg = T.empty_like(out) if want_z else None
    zu = T.empty_like(out) if want_z else None
    _run_rows("whtmix_gated_forward", dev, stream,
              (x.data_ptr(), pg, pu, pbg, pbu, py, _ptr(zg), _ptr(zu)), (M, K, N, ld), (act, dt))
    return (out, zg, zu) if want_z else out


def gated_backward(x, w_gate, w_up, dy, z_gate, z_up, activation: str = "silu",
                   want_dx: bool = True, want_dw: bool = True, want_dbias: bool = True,
                   stream=None):
    """Gradients through gated() for the upstream gradient dy: (dx, dw_gate, dw_up, db_gate,
    db_up), the biases' float32 and the others in x's type; what is not wanted is None.
    z_gate, z_up: what gated kept."""
    if stream is None:
        r = (_ordinary_module or _ordinary()).gated_backward(
            x, w_gate, w_up, dy, z_gate, z_up, _activation(activation), want_dx, want_dw, want_dbias)
        if r is not None:
            return _taken(r, "gated_backward")
    T = _torch_module or _torch()
    dt, M, K, ld, dev = _operand(x, "x")
    act, dtype = _activation(activation), x.dtype
    N, pg, pu = _gates(x, w_gate, w_up, K, dev)
    shape = (*x.shape[:-1], N)
    pdy = _tensor(dy, shape, dtype, dev, "dy")
    pzg = _tensor(z_gate, shape, dtype, dev, "z_gate")
    pzu = _tensor(z_up, shape, dtype, dev, "z_up")
    if not (want_dx or want_dw or want_dbias):
        raise ValueError("nothing to compute")
    dx = T.empty_like(x, memory_format=T.contiguous_format) if want_dx else None
    dwg, dwu = (T.empty_like(w_gate), T.empty_like(w_up)) if want_dw else (None, None)
    dbg = x.new_empty(N, dtype=T.float32) if want_dbias else None
    dbu = x.new_empty(N, dtype=T.float32) if want_dbias else None
    _run_rows("whtmix_gated_backward", dev, stream,
              (x.data_ptr(), pg, pu, pdy, pzg, pzu, _ptr(dx), _ptr(dwg), _ptr(dwu), _ptr(dbg),
               _ptr(dbu)), (M, K, N, ld), (act, dt))
    return dx, dwg, dwu, dbg, dbu


def gated_mx(xq, xs, wgq, wgs, wuq, wus, b_gate=None, b_up=None, activation: str = "silu",
             out_mx: bool = False, dtype=None, out=None, stream=None):
    """gated() on block-scaled 8 bits: xq, xs as norm_mx or quantize_mx give them, [..., K];
    wgq, wgs and wuq, wus the weights' columns as rows, [N, K].  Returns y [..., N] in dtype
    (out's, else bfloat16), or with out_mx (q, scales) of the result.  Sums as linear_mx's."""
    if dtype is None and out is None and stream is None:
        r = (_ordinary_module or _ordinary()).gated_mx(
            xq, xs, wgq, wgs, wuq, wus, b_gate, b_up, _activation(activation), out_mx)
        if r is not None:
            return _taken(r, "gated_mx_forward") if out_mx else _taken(r, "gated_mx_forward")[0]
    T = _torch_module or _torch()
    M, K, pxq, pxs, dev = _mx(xq, xs, "xq")
    act = _activation(activation)
    if wgq.dim() != 2:
        raise ValueError("wgq must be [N, K]")
    N, Kw, pgq, pgs, wdev = _mx(wgq, wgs, "wgq")
    if Kw != K or wdev != dev:
        raise ValueError(f"wgq must hold rows of {K} on xq's device")
    if wuq.shape != wgq.shape:
        raise ValueError("wuq must have wgq's shape")
    _, _, puq, pus, udev = _mx(wuq, wus, "wuq")
    if udev != dev:
        raise ValueError("wuq must be on xq's device")
    lead = xq.shape[:-1]
    pbg = 0 if b_gate is None else _tensor(b_gate, (N,), T.float32, dev, "b_gate")
    pbu = 0 if b_up is None else _tensor(b_up, (N,), T.float32, dev, "b_up")
    if dtype is None:
        dtype = out.dtype if out is not None else T.bfloat16
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"the output must be float32 or bfloat16, not {dtype}")
    q = s = None
    if out_mx:
        if out is not None:
            raise ValueError("out is for outputs that are not in 8 bits")
        q, s = _new_mx(xq, lead, N)
    elif out is None:
        out = xq.new_empty((*lead, N), dtype=dtype)
    else:
        _tensor(out, (*lead, N), dtype, dev, "out")
    _run_rows("whtmix_gated_mx_forward", dev, stream,
              (pxq, pxs, pgq, pgs, puq, pus, pbg, pbu, _ptr(out), _ptr(q), _ptr(s)), (M, K, N),
              (act, code))
    return (q, s) if out_mx else out


def _ids(ids, like, what):
    """(index code, address) of a contiguous int32 or int64 tensor on the device of `like`."""
    code = _INDEX.get(ids.dtype)
    if code is None:
        raise TypeError(f"ids must be int32 or int64, got {ids.dtype}")
    if not ids.is_contiguous() or ids.get_device() != like.get_device():
        raise ValueError(f"ids must be contiguous and on {what}'s device")
    return code, ids.data_ptr()


def embedding(ids, table, scale: float = 1.0, out=None, stream=None):
    """scale * table[ids], [*ids.shape, C] of the table's type: the rows of table [vocab, C]
    (float32 or bfloat16, contiguous) that ids (int32 or int64, any shape) name.  A negative id
    is padding, whose row is zeros; an id of vocab or more gives NaN.  out: optional contiguous
    tensor for the rows."""
    if out is None and stream is None:
        r = (_ordinary_module or _ordinary()).embedding(ids, table, scale)
        if r is not None:
            return _taken(r, "embedding_forward")[0]
    _torch_module or _torch()
    if table.dim() != 2:
        raise ValueError("table must be [vocab, C]")
    dt, V, C, _, dev = _operand(table, "table")
    pt = _tensor(table, (V, C), table.dtype, dev, "table")
    index, pi = _ids(ids, table, "table")
    shape = (*ids.shape, C)
    if out is None:
        out = table.new_empty(shape)
        py = out.data_ptr()
    else:
        py = _tensor(out, shape, table.dtype, dev, "out")
    _run_rows("whtmix_embedding_forward", dev, stream, (pi, pt, py), (ids.numel(), V, C),
              (index, dt), scale)
    return out


def embedding_backward(ids, dy, vocab: int, scale: float = 1.0, stream=None):
    """The gradient of embedding()'s table [vocab, C] for the upstream gradient dy
    [*ids.shape, C], in dy's type: every row is written, in an order of sums that does not
    change from run to run.  Padding and ids of vocab or more have none."""
    if stream is None:
        r = (_ordinary_module or _ordinary()).embedding_backward(ids, dy, vocab, scale)
        if r is not None:
            return _taken(r, "embedding_backward")[0]
    _torch_module or _torch()
    if not dy.is_cuda:
        raise ValueError("dy must be on a GPU device")
    dt = _CODES.get(dy.dtype)
    if dt is None:
        raise TypeError(f"dy must be float32 or bfloat16, got {dy.dtype}")
    if dy.dim() < 1:
        raise ValueError("dy must be [*ids.shape, C]")
    C, dev = dy.shape[-1], dy.get_device()
    pdy = _tensor(dy, (*ids.shape, C), dy.dtype, dev, "dy")
    index, pi = _ids(ids, dy, "dy")
    dtable = dy.new_empty((vocab, C))
    _run_rows("whtmix_embedding_backward", dev, stream, (pi, pdy, dtable.data_ptr()),
              (ids.numel(), vocab, C), (index, dt), scale)
    return dtable


def release_workspaces() -> None:
    st = lib().whtmix_release_workspaces()
    if st != SUCCESS:
        raise WhtmixError(st, "whtmix_release_workspaces")
