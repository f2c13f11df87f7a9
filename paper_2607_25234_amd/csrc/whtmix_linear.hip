// Matrix products with bias, activation and residual in the epilogue, and
// their gradients.
//
//   z = x w + bias,  y = act(z) + residual
//   dz = dy act'(z),  dx = dz w^T,  dw = x^T dz,  dbias = column sums of dz
//
// Here what a call is made of: dz, and the products by element type (whtmix_linear_bf16.hip,
// whtmix_linear_f32.hip, whtmix_linear_mx.hip).
#include "whtmix_gemm.h"

#include <algorithm>

namespace whtmix {
namespace {

// dz = dy act'(z), with the columns' sums of the unrounded values: 32 threads across
// 256 columns, 8 rows at a time, four of them in flight a thread; the workgroup's 8
// sums of a column are added in order.  dz is rounded to the type of dy: bf16 is what the matrix
// cores read, and half the bytes for both products.  Bound by memory and, with gelu in bf16, by its
// vector instructions as much: 262144 x 512 bf16 192 us (805 MB at 4.2 TB/s; wide products of
// it follow, narrow ones are formed in launch_dzx's pass), float32 3001 x 2003 21 us.
constexpr int kDzRows = 8, kDzCols = 256;

template <typename T>
__global__ void __launch_bounds__(256) dz_kernel(const T *dy, const T *z, T *dz, float *part,
                                                 int64_t M, int64_t N, int64_t per, int act)
{
    __shared__ float sums[kDzRows][kDzCols + 8];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int64_t n = (int64_t)blockIdx.x * kDzCols + tx * 8;
    const int cnt = (int)min((int64_t)8, N - n);
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 0.f;
    const int64_t end = min(M, ((int64_t)blockIdx.y + 1) * per);
    if (cnt > 0)
        with_act(act, [&](auto tag) {
            constexpr int ACT = decltype(tag)::value;
            constexpr int U = 4;
            for (int64_t m = (int64_t)blockIdx.y * per + ty; m < end; m += U * kDzRows) {
                float d[U][8], v[U][8];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t r = m + u * kDzRows;
                    const int c = r < end ? cnt : 0;
                    const int64_t at = (r < end ? r : m) * N + n;
                    load8(dy + at, c, d[u]);
                    if (ACT != ACT_NONE) load8(z + at, c, v[u]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t r = m + u * kDzRows;
                    if (r >= end) break;
                    if (ACT != ACT_NONE) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) d[u][i] *= act_grad<ACT>(v[u][i]);
                        if (dz) store8(dz + r * N + n, cnt, d[u]);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[i] += d[u][i];
                }
            }
        });
    if (!part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[ty][tx * 8 + i] = s[i];
    __syncthreads();
    const int64_t c = (int64_t)blockIdx.x * kDzCols + threadIdx.x;
    if (c >= N) return;
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < kDzRows; ++r) t += sums[r][threadIdx.x];
    part[(int64_t)blockIdx.y * N + c] = t;
}

// Workgroups down the rows: about 1024 in all, 32 rows or more each.
int64_t dz_parts(int64_t M, int64_t N)
{
    const int64_t cols = (N + kDzCols - 1) / kDzCols;
    return std::max<int64_t>(1, std::min<int64_t>((M + 31) / 32, 1024 / cols));
}

uint64_t align256(uint64_t v) { return (v + 255) / 256 * 256; }

template <typename T>
hipError_t product(const GemmArgs &g, Layout la, Layout lb, void *ws, hipStream_t stream)
{
    if constexpr (std::is_same_v<T, __bf16>) return gemm_bf16(g, la, lb, ws, stream);
    else return gemm_f32(g, la, lb, ws, stream);
}

uint64_t product_bytes(const GemmArgs &g, Layout la, Layout lb, int dtype)
{
    return dtype == DTYPE_BF16 ? gemm_bf16_bytes(g, la, lb) : gemm_f32_bytes(g);
}

GemmArgs forward_args(const LinearArgs &a)
{
    GemmArgs g{};
    g.a = a.x, g.lda = a.ldx, g.b = a.w, g.ldb = a.N;
    g.M = a.M, g.N = a.N, g.K = a.K;
    g.bias = a.bias, g.residual = a.residual, g.y = a.y, g.z = a.z, g.act = a.act;
    return g;
}

GemmArgs dx_args(const LinearBackwardArgs &a, const void *dz)
{
    GemmArgs g{};
    g.a = dz, g.lda = a.N, g.b = a.w, g.ldb = a.N;
    g.M = a.M, g.N = a.K, g.K = a.N, g.y = a.dx;
    return g;
}

GemmArgs dw_args(const LinearBackwardArgs &a, const void *dz)
{
    GemmArgs g{};
    g.a = a.x, g.lda = a.ldx, g.b = dz, g.ldb = a.N;
    g.M = a.K, g.N = a.N, g.K = a.M, g.y = a.dw;
    return g;
}

struct BackwardLayoutBytes {
    uint64_t dz = 0, part = 0, product = 0;
};
BackwardLayoutBytes backward_bytes(const LinearBackwardArgs &a)
{
    BackwardLayoutBytes l;
    const int e = a.dtype == DTYPE_BF16 ? 2 : 4;
    // what a product reads: dz, where it is not dy itself
    if (a.act != ACT_NONE && (a.dw || (a.dx && !dzx_takes(a))))
        l.dz = align256((uint64_t)a.M * a.N * e);
    if (a.dbias)
        l.part = align256((uint64_t)(dzx_takes(a) ? dzx_parts(a.M) : dz_parts(a.M, a.N)) * a.N * 4);
    const void *dz = a.act != ACT_NONE ? nullptr : a.dy;    // a workspace's address is aligned
    if (a.dx && !dzx_takes(a))
        l.product = product_bytes(dx_args(a, dz), K_CONTIGUOUS, K_CONTIGUOUS, a.dtype);
    if (a.dw)
        l.product = std::max(l.product, product_bytes(dw_args(a, dz), K_STRIDED, K_STRIDED, a.dtype));
    return l;
}

template <typename T> hipError_t linear_backward(const LinearBackwardArgs &a)
{
    const BackwardLayoutBytes l = backward_bytes(a);
    char *ws = (char *)a.ws;
    T *dz = l.dz ? (T *)ws : nullptr;
    float *part = (float *)(ws + l.dz);
    void *rest = ws + l.dz + l.part;
    hipError_t e;
    const bool together = dzx_takes(a);
    if (together) {
        if ((e = launch_dzx(a, dz, a.dbias ? part : nullptr)) != hipSuccess) return e;
        if (a.dbias && (e = launch_column_sum(part, dzx_parts(a.M), a.N, a.dbias, a.stream)) !=
                           hipSuccess)
            return e;
    } else if (a.act != ACT_NONE || a.dbias) {
        const int64_t parts = dz_parts(a.M, a.N);
        const int64_t per = (a.M + parts - 1) / parts;
        const dim3 grid((uint32_t)((a.N + kDzCols - 1) / kDzCols),
                        (uint32_t)((a.M + per - 1) / per));
        dz_kernel<T><<<grid, dim3(256), 0, a.stream>>>(
            (const T *)a.dy, (const T *)a.z, dz, a.dbias ? part : nullptr, a.M, a.N, per, a.act);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (a.dbias && (e = launch_column_sum(part, grid.y, a.N, a.dbias, a.stream)) != hipSuccess)
            return e;
    }
    const void *d = a.act != ACT_NONE ? (const void *)dz : a.dy;
    if (a.dx && !together &&
        (e = product<T>(dx_args(a, d), K_CONTIGUOUS, K_CONTIGUOUS, rest, a.stream)) != hipSuccess)
        return e;
    if (a.dw) return product<T>(dw_args(a, d), K_STRIDED, K_STRIDED, rest, a.stream);
    return hipSuccess;
}

GemmArgs mx_args(const LinearMxArgs &a)
{
    GemmArgs g{};
    g.a = a.xq, g.as = a.xs, g.b = a.wq, g.bs = a.ws8;
    g.lda = g.ldb = g.K = mx_width(a.K);
    g.M = a.M, g.N = a.N;
    g.bias = a.bias, g.residual = a.residual, g.act = a.act;
    g.y = a.y, g.yq = (uint8_t *)a.yq, g.ys = a.ys;
    return g;
}

}  // namespace

uint64_t linear_bytes(const LinearArgs &a)
{
    return product_bytes(forward_args(a), K_CONTIGUOUS, K_STRIDED, a.dtype);
}

hipError_t launch_linear(const LinearArgs &a)
{
    const GemmArgs g = forward_args(a);
    return a.dtype == DTYPE_BF16 ? product<__bf16>(g, K_CONTIGUOUS, K_STRIDED, a.ws, a.stream)
                                 : product<float>(g, K_CONTIGUOUS, K_STRIDED, a.ws, a.stream);
}

uint64_t linear_backward_bytes(const LinearBackwardArgs &a)
{
    const BackwardLayoutBytes l = backward_bytes(a);
    return l.dz + l.part + l.product;
}

hipError_t launch_linear_backward(const LinearBackwardArgs &a)
{
    return a.dtype == DTYPE_BF16 ? linear_backward<__bf16>(a) : linear_backward<float>(a);
}

uint64_t linear_mx_bytes(const LinearMxArgs &a) { return gemm_mx_bytes(mx_args(a)); }

hipError_t launch_linear_mx(const LinearMxArgs &a)
{
    return gemm_mx(mx_args(a), a.dtype, a.ws, a.stream);
}

}  // namespace whtmix
