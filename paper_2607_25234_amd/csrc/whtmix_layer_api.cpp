// C entry points of the feed-forward sublayer's operators: argument checks,
// then workspace and launches.  Declared in include/whtmix.h.
#include <cmath>
#include <cstdint>
#include <exception>
#include <initializer_list>

#include "whtmix.h"
#include "whtmix_layer.h"

namespace {

using whtmix::mx_width;

constexpr int64_t kMaxRows = int64_t(1) << 30;
constexpr int64_t kMaxWidth = int64_t(1) << 22;

struct Range {
    const void *p;
    uint64_t bytes;
    uintptr_t at() const { return reinterpret_cast<uintptr_t>(p); }
};

bool overlap(const Range &a, const Range &b)
{
    return a.p && b.p && a.at() < b.at() + b.bytes && b.at() < a.at() + a.bytes;
}

// An output apart from all the inputs and the other outputs given.
bool apart(const Range &out, std::initializer_list<Range> others)
{
    for (const Range &r : others)
        if (overlap(out, r)) return false;
    return true;
}

bool aligned(std::initializer_list<const void *> ps, uintptr_t to)
{
    for (const void *p : ps)
        if (reinterpret_cast<uintptr_t>(p) % to) return false;
    return true;
}

int check_dtype(int dtype)
{
    return dtype == WHTMIX_DTYPE_F32 || dtype == WHTMIX_DTYPE_BF16 ? WHTMIX_SUCCESS
                                                                   : WHTMIX_ERROR_UNSUPPORTED_DTYPE;
}

uint64_t elt(int dtype) { return dtype == WHTMIX_DTYPE_BF16 ? 2 : 4; }

// Sizes: rows >= 0 and widths >= 1 within the limits, ld >= width.  Every byte
// count then fits 64 bits.
int check_sizes(int64_t rows, std::initializer_list<int64_t> widths, int64_t ld, int64_t ld_width)
{
    if (rows < 0 || ld < ld_width) return WHTMIX_ERROR_INVALID_VALUE;
    for (int64_t w : widths)
        if (w < 1) return WHTMIX_ERROR_INVALID_VALUE;
    if (rows > kMaxRows || ld > (int64_t(1) << 31)) return WHTMIX_ERROR_TOO_LARGE;
    for (int64_t w : widths)
        if (w > kMaxWidth) return WHTMIX_ERROR_TOO_LARGE;
    return WHTMIX_SUCCESS;
}

// Bytes from the first row to the end of the last.
uint64_t span(int64_t rows, int64_t width, int64_t ld, uint64_t e)
{
    return rows > 0 ? ((uint64_t)(rows - 1) * ld + width) * e : 0;
}

int done(hipError_t e, const char *what)
{
    return e == hipSuccess ? WHTMIX_SUCCESS : whtmix::report_hip(e, what);
}

// No exception leaves a C entry point.
template <typename F> int guarded(F f) noexcept
{
    try {
        return f();
    } catch (const std::exception &) {
        return WHTMIX_ERROR_OUT_OF_MEMORY;
    }
}

// launch(workspace) with `bytes` of the stream's workspace (none: null).
template <typename F> int with_workspace(void *stream, uint64_t bytes, const char *what, F launch)
{
    if (bytes == 0) return done(launch(nullptr), what);
    whtmix::WorkspaceLock lock;
    float *ws = nullptr;
    const int st = whtmix::stream_workspace(stream, (int64_t)bytes, &ws);
    return st != WHTMIX_SUCCESS ? st : done(launch(ws), what);
}

bool bad_eps(double eps) { return !(eps >= 0.0) || !std::isfinite((float)eps); }

int norm_impl(const void *x, const void *residual, const float *weight, bool mx, void *y, void *q,
              uint8_t *scales, void *h, int64_t rows, int64_t C, int64_t ldx, double eps,
              int dtype, void *stream, bool quantize_only)
{
    int st = check_dtype(dtype);
    if (st == WHTMIX_SUCCESS) st = check_sizes(rows, {C}, ldx, C);
    if (st != WHTMIX_SUCCESS) return st;
    if (!quantize_only && bad_eps(eps)) return WHTMIX_ERROR_INVALID_VALUE;
    if (rows == 0) return WHTMIX_SUCCESS;
    if (!x || (!quantize_only && !weight) || (mx ? !q || !scales : !y))
        return WHTMIX_ERROR_INVALID_VALUE;
    const uint64_t e = elt(dtype);
    if (!aligned({x, residual, y, h}, e) || !aligned({weight}, 4) || !aligned({q}, 16))
        return WHTMIX_ERROR_MISALIGNED;
    const Range rx{x, span(rows, C, ldx, e)}, rr{residual, span(rows, C, C, e)},
        rw{weight, (uint64_t)C * 4}, ry{y, span(rows, C, C, e)}, rh{h, span(rows, C, C, e)},
        rq{q, (uint64_t)rows * mx_width(C)},
        rs{scales, (uint64_t)rows * (mx_width(C) / whtmix::kMxBlock)};
    const bool same_y = y == x && ldx == C, h_x = h == x && ldx == C, h_r = h == residual;
    if (!apart(ry, {rr, rw, rh}) || (!same_y && overlap(ry, rx)) || !apart(rh, {rw, rq, rs}) ||
        (!h_x && overlap(rh, rx)) || (!h_r && overlap(rh, rr)) || !apart(rq, {rx, rr, rw, rs}) ||
        !apart(rs, {rx, rr, rw}))
        return WHTMIX_ERROR_INVALID_VALUE;
    const whtmix::NormArgs a{x, residual, weight, y, h, q, scales, rows, C, ldx, (float)eps,
                             dtype, static_cast<hipStream_t>(stream)};
    return done(whtmix::launch_norm(a), mx ? "norm in 8 bits" : "norm");
}

int check_act(int act)
{
    return act >= WHTMIX_ACT_NONE && act <= WHTMIX_ACT_SILU ? WHTMIX_SUCCESS
                                                            : WHTMIX_ERROR_INVALID_VALUE;
}

}  // namespace

extern "C" {

int whtmix_norm_forward(const void *x, const void *residual, const float *weight, void *y, void *h,
                        int64_t rows, int64_t C, int64_t ldx, double eps, int dtype, void *stream)
{
    return guarded([&] {
        return norm_impl(x, residual, weight, false, y, nullptr, nullptr, h, rows, C, ldx, eps,
                         dtype, stream, false);
    });
}

int whtmix_norm_mx_forward(const void *x, const void *residual, const float *weight, void *q,
                           uint8_t *scales, void *h, int64_t rows, int64_t C, int64_t ldx,
                           double eps, int dtype, void *stream)
{
    return guarded([&] {
        return norm_impl(x, residual, weight, true, nullptr, q, scales, h, rows, C, ldx, eps,
                         dtype, stream, false);
    });
}

int whtmix_quantize_mx(const void *x, void *q, uint8_t *scales, int64_t rows, int64_t C,
                       int64_t ldx, int dtype, void *stream)
{
    return guarded([&] {
        return norm_impl(x, nullptr, nullptr, true, nullptr, q, scales, nullptr, rows, C, ldx, 0.0,
                         dtype, stream, true);
    });
}

int whtmix_dequantize_mx(const void *q, const uint8_t *scales, void *y, int64_t rows, int64_t C,
                         int dtype, void *stream)
{
    return guarded([&]() -> int {
        int st = check_dtype(dtype);
        if (st == WHTMIX_SUCCESS) st = check_sizes(rows, {C}, C, C);
        if (st != WHTMIX_SUCCESS) return st;
        if (rows == 0) return WHTMIX_SUCCESS;
        if (!q || !scales || !y) return WHTMIX_ERROR_INVALID_VALUE;
        if (!aligned({y}, elt(dtype)) || !aligned({q}, 16)) return WHTMIX_ERROR_MISALIGNED;
        if (!apart({y, span(rows, C, C, elt(dtype))},
                   {{q, (uint64_t)rows * mx_width(C)},
                    {scales, (uint64_t)rows * (mx_width(C) / whtmix::kMxBlock)}}))
            return WHTMIX_ERROR_INVALID_VALUE;
        return done(whtmix::launch_dequantize(q, scales, y, rows, C, dtype,
                                              static_cast<hipStream_t>(stream)),
                    "dequantise");
    });
}

int whtmix_norm_backward(const void *h, const float *weight, const void *dy, const void *dh,
                         void *dx, float *dweight, int64_t rows, int64_t C, double eps, int dtype,
                         void *stream)
{
    return guarded([&]() -> int {
        int st = check_dtype(dtype);
        if (st == WHTMIX_SUCCESS) st = check_sizes(rows, {C}, C, C);
        if (st != WHTMIX_SUCCESS) return st;
        if (bad_eps(eps)) return WHTMIX_ERROR_INVALID_VALUE;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        const uint64_t e = elt(dtype);
        if (!aligned({h, dy, dh, dx}, e) || !aligned({weight, dweight}, 4))
            return WHTMIX_ERROR_MISALIGNED;
        if (rows == 0)
            return dweight ? done(whtmix::launch_zero(dweight, (uint64_t)C * 4, s), "norm backward")
                           : WHTMIX_SUCCESS;
        if (!h || !weight || !dy || !dx) return WHTMIX_ERROR_INVALID_VALUE;
        const uint64_t n = span(rows, C, C, e);
        const Range rx{dx, n}, rw{dweight, (uint64_t)C * 4}, rh{h, n}, ry{dy, n}, rd{dh, n},
            rg{weight, (uint64_t)C * 4};
        if (!apart(rx, {rh, rg, rw}) || (dx != dy && overlap(rx, ry)) ||
            (dx != dh && overlap(rx, rd)) || !apart(rw, {rh, ry, rd, rg}))
            return WHTMIX_ERROR_INVALID_VALUE;
        const uint64_t floats = whtmix::norm_backward_floats(rows, C, dtype, dweight != nullptr);
        return with_workspace(stream, floats * 4, "norm backward", [&](float *ws) {
            const whtmix::NormBackwardArgs a{h, weight, dy, dh, dx, dweight, ws, rows, C,
                                             (float)eps, dtype, s};
            return whtmix::launch_norm_backward(a);
        });
    });
}

int whtmix_linear_forward(const void *x, const void *w, const float *bias, const void *residual,
                          void *y, void *z, int64_t M, int64_t K, int64_t N, int64_t ldx,
                          int activation, int dtype, void *stream)
{
    return guarded([&]() -> int {
        int st = check_dtype(dtype);
        if (st == WHTMIX_SUCCESS) st = check_sizes(M, {K, N}, ldx, K);
        if (st == WHTMIX_SUCCESS) st = check_act(activation);
        if (st != WHTMIX_SUCCESS || M == 0) return st;
        if (!x || !w || !y) return WHTMIX_ERROR_INVALID_VALUE;
        const uint64_t e = elt(dtype);
        if (!aligned({x, w, residual, y, z}, e) || !aligned({bias}, 4))
            return WHTMIX_ERROR_MISALIGNED;
        const uint64_t out = span(M, N, N, e);
        const Range rx{x, span(M, K, ldx, e)}, rw{w, span(K, N, N, e)},
            rb{bias, (uint64_t)N * 4}, rr{residual, out}, ry{y, out}, rz{z, out};
        if (!apart(ry, {rx, rw, rb, rz}) || (y != residual && overlap(ry, rr)) ||
            !apart(rz, {rx, rw, rb, rr}))
            return WHTMIX_ERROR_INVALID_VALUE;
        whtmix::LinearArgs a{x, w, bias, residual, y, z, M, K, N, ldx, activation, dtype, nullptr,
                             static_cast<hipStream_t>(stream)};
        return with_workspace(stream, whtmix::linear_bytes(a), "linear", [&](float *ws) {
            a.ws = ws;
            return whtmix::launch_linear(a);
        });
    });
}

int whtmix_linear_backward(const void *x, const void *w, const void *dy, const void *z, void *dx,
                           void *dw, float *dbias, int64_t M, int64_t K, int64_t N, int64_t ldx,
                           int activation, int dtype, void *stream)
{
    return guarded([&]() -> int {
        int st = check_dtype(dtype);
        if (st == WHTMIX_SUCCESS) st = check_sizes(M, {K, N}, ldx, K);
        if (st == WHTMIX_SUCCESS) st = check_act(activation);
        if (st != WHTMIX_SUCCESS) return st;
        if (!dx && !dw && !dbias) return WHTMIX_ERROR_INVALID_VALUE;
        const uint64_t e = elt(dtype);
        if (!aligned({x, w, dy, z, dx, dw}, e) || !aligned({dbias}, 4))
            return WHTMIX_ERROR_MISALIGNED;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        if (M == 0) {
            hipError_t er = hipSuccess;
            if (dw) er = whtmix::launch_zero(dw, (uint64_t)K * N * e, s);
            if (dbias && er == hipSuccess) er = whtmix::launch_zero(dbias, (uint64_t)N * 4, s);
            return done(er, "linear backward");
        }
        if (!dy || (dx && !w) || (dw && !x) || (activation != WHTMIX_ACT_NONE && !z))
            return WHTMIX_ERROR_INVALID_VALUE;
        const uint64_t out = span(M, N, N, e);
        const Range rx{x, span(M, K, ldx, e)}, rw{w, span(K, N, N, e)}, ry{dy, out}, rz{z, out},
            ox{dx, span(M, K, K, e)}, ow{dw, span(K, N, N, e)}, ob{dbias, (uint64_t)N * 4};
        if (!apart(ox, {rx, rw, ry, rz, ow, ob}) || !apart(ow, {rx, rw, ry, rz, ob}) ||
            !apart(ob, {rx, rw, ry, rz}))
            return WHTMIX_ERROR_INVALID_VALUE;
        whtmix::LinearBackwardArgs a{x, w, dy, z, dx, dw, dbias, M, K, N, ldx, activation, dtype,
                                     nullptr, s};
        return with_workspace(stream, whtmix::linear_backward_bytes(a), "linear backward",
                              [&](float *ws) {
                                  a.ws = ws;
                                  return whtmix::launch_linear_backward(a);
                              });
    });
}

int whtmix_linear_mx_forward(const void *xq, const uint8_t *xs, const void *wq, const uint8_t *ws,
                             const float *bias, const void *residual, void *y, void *yq,
                             uint8_t *ys, int64_t M, int64_t K, int64_t N, int activation,
                             int dtype, void *stream)
{
    return guarded([&]() -> int {
        int st = check_dtype(dtype);
        if (st == WHTMIX_SUCCESS) st = check_sizes(M, {K, N}, K, K);
        if (st == WHTMIX_SUCCESS) st = check_act(activation);
        if (st != WHTMIX_SUCCESS || M == 0) return st;
        if (!xq || !xs || !wq || !ws || (y ? yq || ys : !yq || !ys))
            return WHTMIX_ERROR_INVALID_VALUE;
        const uint64_t e = elt(dtype);
        if (!aligned({residual, y}, e) || !aligned({bias}, 4) || !aligned({xq, wq, yq}, 16))
            return WHTMIX_ERROR_MISALIGNED;
        const uint64_t kw = mx_width(K), nw = mx_width(N), kb = kw / whtmix::kMxBlock;
        const Range ra{xq, M * kw}, rb{xs, M * kb}, rc{wq, N * kw}, rd{ws, N * kb},
            rbias{bias, (uint64_t)N * 4}, rr{residual, span(M, N, N, e)},
            ry{y, span(M, N, N, e)}, rq{yq, M * nw}, rs{ys, M * (nw / whtmix::kMxBlock)};
        if (!apart(ry, {ra, rb, rc, rd, rbias}) || (y != residual && overlap(ry, rr)) ||
            !apart(rq, {ra, rb, rc, rd, rbias, rr, rs}) ||
            !apart(rs, {ra, rb, rc, rd, rbias, rr}))
            return WHTMIX_ERROR_INVALID_VALUE;
        whtmix::LinearMxArgs a{xq, xs, wq, ws, bias, residual, y, yq, ys, M, K, N, activation,
                               dtype, nullptr, static_cast<hipStream_t>(stream)};
        return with_workspace(stream, whtmix::linear_mx_bytes(a), "linear in 8 bits",
                              [&](float *p) {
                                  a.ws = p;
                                  return whtmix::launch_linear_mx(a);
                              });
    });
}

}  // extern "C"
