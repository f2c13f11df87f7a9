// The gated feed-forward product and its gradients.
//
//   zg = x wg + bg,  zu = x wu + bu,  y = act(zg) o zu
//   dzg = dy zu act'(zg),  dzu = dy act(zg)
//   dx = dzg wg^T + dzu wu^T,  dwg = x^T dzg,  dwu = x^T dzu,  dbg, dbu = column sums of dzg, dzu
//
// Forward both products run in one tile kernel (FORM GATED of the products), so that x is read
// once and neither sum leaves the registers.  Backward dzg and dzu are the halves of one matrix
// [M][2 Np]: dx is one product over its 2 Np columns, the weights' gradients one product with its
// 2 Np columns (forms TWO_K and HALVES), one launch each in place of two.  Narrow inputs form dx
// in the pass that forms dzg and dzu (whtmix_gated_dzx.hip).
//
// 8192 x 4096 x 2 x 12288 bf16: forward 1315 us (1.25 PFLOP/s, the matrix cores 70%
// busy), dz 211 (4.8 TB/s), dx 1256, the weights' gradients 1245 (1.31 and 1.32 PFLOP/s).  262144 x
// 128 x 2 x 344: forward 184 us (608 MB), the weights' gradients 127 + 8.  3001 x 1000 x 2 x 2003
// float32, kernel by kernel: forward 137-145 us, dz 29, dx 145-152 + 12, the weights' gradients 122-128
// + 13, splits 3 x 30.
#include "whtmix_gemm.h"
#include "whtmix_row.h"

#include <algorithm>

namespace whtmix {
namespace {

template <typename T> __device__ __forceinline__ void load_eight(const T *p, int n, float (&v)[8])
{
    constexpr int N = Chunk<T>::N;
#pragma unroll
    for (int i = 0; i < 8; i += N)
        load_row<T>(p + i, max(0, n - i), *(float(*)[N])(v + i));
}

// dzg and dzu with the columns' sums of the unrounded values.  `across` threads take a row's
// chunks of 8 columns, the workgroup's other threads the rows below: with whole rows the memory
// it touches is contiguous whatever their width.  The threads' sums of a column are added in
// order.  The values are rounded to the type of dy, what the matrix cores read; columns N .. width -
// 1 of each half are zeros.
template <typename T>
__global__ void __launch_bounds__(256)
    gated_dz_kernel(const T *dy, const T *zg, const T *zu, T *dz, float *part, int64_t M, int64_t N,
                    int64_t width, int64_t per, int across, int act)
{
    __shared__ float sums[256 * 9];
    const int down = 256 / across, tx = threadIdx.x % across, ty = threadIdx.x / across;
    const int64_t n = ((int64_t)blockIdx.x * across + tx) * 8;
    const int cnt = (int)max((int64_t)0, min((int64_t)8, N - n));
    float sg[8], su[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sg[i] = su[i] = 0.f;
    const int64_t end = min(M, ((int64_t)blockIdx.y + 1) * per);
    if (n < width && ty < down)
        with_act(act, [&](auto tag) {
            constexpr int ACT = decltype(tag)::value;
            constexpr int U = 2;
            for (int64_t m = (int64_t)blockIdx.y * per + ty; m < end; m += U * down) {
                float d[U][8], g[U][8], u[U][8];
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const int64_t r = m + k * down;
                    const int c = r < end ? cnt : 0;
                    const int64_t at = c ? r * N + n : 0;
                    load_eight(dy + at, c, d[k]);
                    load_eight(zg + at, c, g[k]);
                    load_eight(zu + at, c, u[k]);
                }
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const int64_t r = m + k * down;
                    if (r >= end) break;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float a, da;
                        act_both<ACT>(g[k][i], a, da);
                        g[k][i] = d[k][i] * u[k][i] * da;
                        u[k][i] = d[k][i] * a;
                        if (i >= cnt) g[k][i] = u[k][i] = 0.f;
                        sg[i] += g[k][i];
                        su[i] += u[k][i];
                    }
                    if (dz) {
                        store8(dz + r * 2 * width + n, 8, g[k]);
                        store8(dz + r * 2 * width + width + n, 8, u[k]);
                    }
                }
            }
        });
    if (!part) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[threadIdx.x * 9 + i] = h ? su[i] : sg[i];
        __syncthreads();
        for (int c = threadIdx.x; c < 8 * across; c += 256) {
            const int64_t col = (int64_t)blockIdx.x * 8 * across + c;
            if (col >= N) continue;
            float t = 0.f;
            for (int r = 0; r < down; ++r) t += sums[(r * across + c / 8) * 9 + c % 8];
            part[((int64_t)blockIdx.y * 2 + h) * N + col] = t;
        }
    }
}

// Threads across the columns of `width`: whole rows of up to 64 chunks where that leaves at
// most a quarter of the workgroup idle (262144 x 344: 237 us, 298 by 16 threads), else the most of 32,
// 16 and 8 that cover the width to an eighth (3001 x 2003 float32: 29 us, 56 by whole rows).
int dz_across(int64_t width)
{
    const int64_t chunks = width / 8;
    if (chunks <= 64 && 256 / chunks * chunks >= 192) return (int)chunks;
    for (int t = 32; t > 8; t /= 2)
        if ((chunks + t - 1) / t * t * 8 <= chunks * 9) return t;
    return 8;
}

// Workgroups down the rows: about 1024 in all, 32 rows or more each.
int64_t dz_parts(int64_t M, int64_t width)
{
    const int64_t across = 8 * dz_across(width), cols = (width + across - 1) / across;
    return std::max<int64_t>(1, std::min<int64_t>((M + 31) / 32, 1024 / cols));
}

template <typename T>
hipError_t launch_dz(const GatedBackwardArgs &a, int64_t width, T *dz, float *sums, int64_t &rows)
{
    const int across = dz_across(width);
    const int64_t parts = dz_parts(a.M, width), per = (a.M + parts - 1) / parts;
    rows = (a.M + per - 1) / per;
    const dim3 grid((uint32_t)((width + 8 * across - 1) / (8 * across)), (uint32_t)rows);
    gated_dz_kernel<T><<<grid, dim3(256), 0, a.stream>>>((const T *)a.dy, (const T *)a.zg,
                                                         (const T *)a.zu, dz, sums, a.M, a.N, width,
                                                         per, across, a.act);
    return hipGetLastError();
}

// Both weights' rows side by side, [K][2 width], with zeros past N: B of one product over both.
template <typename T>
__global__ void __launch_bounds__(256) join_weights_kernel(const T *wg, const T *wu, T *out,
                                                           int64_t K, int64_t N, int64_t width)
{
    const int64_t per = width / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < K * 2 * per;
         i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / (2 * per), c = i - r * 2 * per;
        const int64_t n = (c < per ? c : c - per) * 8;
        float v[8];
        load8((c < per ? wg : wu) + r * N + n, (int)min((int64_t)8, N - n), v);
        store8(out + r * 2 * width + c * 8, 8, v);
    }
}

uint64_t align256(uint64_t v) { return (v + 255) / 256 * 256; }

// What a backward call is made of.
struct Parts {
    int64_t width;          // Np: of each half of dz
    int64_t pitch;          // between dz's rows
    bool together;          // dz, its sums and dx in one pass
    bool two_k;             // dx reads both weights where they lie
    uint64_t dz, sums, weights, product;    // bytes
};

GemmArgs dx_args(const GatedBackwardArgs &a, const Parts &p, const void *dz, const void *joined)
{
    GemmArgs g{};
    g.a = dz, g.lda = 2 * p.width;
    g.M = a.M, g.N = a.K, g.K = 2 * p.width, g.y = a.dx;
    if (p.two_k) g.b = a.wg, g.b2 = a.wu, g.ldb = a.N, g.half = a.N;
    else g.b = joined, g.ldb = 2 * p.width;
    return g;
}

GemmArgs dw_args(const GatedBackwardArgs &a, const Parts &p, const void *dz)
{
    GemmArgs g{};
    g.a = a.x, g.lda = a.ldx, g.b = dz, g.ldb = p.pitch;
    g.M = a.K, g.N = 2 * p.width, g.K = a.M;
    g.y = a.dwg, g.y2 = a.dwu, g.half = p.width, g.half_n = a.N;
    return g;
}

Parts parts_of(const GatedBackwardArgs &a)
{
    Parts p{};
    const bool bf16 = a.dtype == DTYPE_BF16;
    const int e = bf16 ? 2 : 4;
    auto aligned = [](const void *q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
    // bf16: whole cache lines, float32: whole chunks of the stores
    p.width = bf16 ? (a.N + 63) / 64 * 64 : (a.N + 7) / 8 * 8;
    p.together = gated_dzx_takes(a);
    p.pitch = p.together ? gated_dzx_pitch(a.N, p.width) : 2 * p.width;
    p.two_k = bf16 && a.N % 64 == 0 && aligned(a.wg) && aligned(a.wu);
    if (a.dwg || (a.dx && !p.together)) p.dz = align256((uint64_t)a.M * p.pitch * e);
    if (a.dbg)
        p.sums = align256((uint64_t)(p.together ? gated_dzx_parts(a) : dz_parts(a.M, p.width)) * 2 *
                          a.N * 4);
    // a workspace's address is aligned: null stands for it
    const bool product = a.dx && !p.together;
    if (product && !p.two_k) p.weights = align256((uint64_t)a.K * 2 * p.width * e);
    if (product) {
        const GemmArgs g = dx_args(a, p, nullptr, nullptr);
        p.product = !bf16     ? gemm_f32_bytes(g)
                    : p.two_k ? gemm_bf16_bytes(g, TWO_K)
                              : gemm_bf16_bytes(g, K_CONTIGUOUS, K_CONTIGUOUS);
    }
    if (a.dwg) {
        const GemmArgs g = dw_args(a, p, nullptr);
        p.product = std::max(p.product, bf16 ? gemm_bf16_bytes(g, HALVES) : gemm_f32_bytes(g, HALVES));
    }
    return p;
}

template <typename T> hipError_t backward(const GatedBackwardArgs &a)
{
    const Parts p = parts_of(a);
    char *ws = (char *)a.ws;
    T *dz = p.dz ? (T *)ws : nullptr;
    float *sums = p.sums ? (float *)(ws + p.dz) : nullptr;
    T *joined = (T *)(ws + p.dz + p.sums);
    void *rest = ws + p.dz + p.sums + p.weights;
    int64_t parts = p.together ? gated_dzx_parts(a) : 0;
    hipError_t e = p.together ? launch_gated_dzx(a, p.width, dz, sums)
                              : launch_dz<T>(a, p.width, dz, sums, parts);
    if (e != hipSuccess) return e;
    if (sums && (e = launch_column_sums(sums, parts, a.N, a.dbg, a.dbu, a.stream)) != hipSuccess)
        return e;
    constexpr bool kBf16 = std::is_same_v<T, __bf16>;
    if (a.dx && !p.together) {
        if (!p.two_k) {
            const int64_t blocks = std::min<int64_t>((a.K * 2 * (p.width / 8) + 255) / 256, 1 << 16);
            join_weights_kernel<T><<<dim3((uint32_t)blocks), dim3(256), 0, a.stream>>>(
                (const T *)a.wg, (const T *)a.wu, joined, a.K, a.N, p.width);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        const GemmArgs g = dx_args(a, p, dz, joined);
        if constexpr (kBf16)
            e = p.two_k ? gemm_bf16(g, TWO_K, rest, a.stream)
                        : gemm_bf16(g, K_CONTIGUOUS, K_CONTIGUOUS, rest, a.stream);
        else
            e = gemm_f32(g, K_CONTIGUOUS, K_CONTIGUOUS, rest, a.stream);
        if (e != hipSuccess) return e;
    }
    if (!a.dwg) return hipSuccess;
    const GemmArgs g = dw_args(a, p, dz);
    if constexpr (kBf16) return gemm_bf16(g, HALVES, rest, a.stream);
    else return gemm_f32(g, HALVES, rest, a.stream);
}

GemmArgs forward_args(const GatedArgs &a)
{
    GemmArgs g{};
    g.a = a.x, g.lda = a.ldx, g.b = a.wg, g.b2 = a.wu, g.ldb = g.ldb2 = a.N;
    g.M = a.M, g.N = a.N, g.K = a.K;
    g.bias = a.bg, g.bias2 = a.bu, g.y = a.y, g.z = a.zg, g.z2 = a.zu, g.act = a.act;
    return g;
}

GemmArgs mx_args(const GatedMxArgs &a)
{
    GemmArgs g{};
    g.a = a.xq, g.as = a.xs, g.b = a.wgq, g.bs = a.wgs, g.b2 = a.wuq, g.bs2 = a.wus;
    g.lda = g.ldb = g.ldb2 = g.K = mx_width(a.K);
    g.M = a.M, g.N = a.N;
    g.bias = a.bg, g.bias2 = a.bu, g.act = a.act;
    g.y = a.y, g.yq = (uint8_t *)a.yq, g.ys = a.ys;
    return g;
}

}  // namespace

uint64_t gated_bytes(const GatedArgs &a)
{
    const GemmArgs g = forward_args(a);
    return a.dtype == DTYPE_BF16 ? gemm_bf16_bytes(g, GATED) : gemm_f32_bytes(g, GATED);
}

hipError_t launch_gated(const GatedArgs &a)
{
    const GemmArgs g = forward_args(a);
    return a.dtype == DTYPE_BF16 ? gemm_bf16(g, GATED, a.ws, a.stream)
                                 : gemm_f32(g, GATED, a.ws, a.stream);
}

uint64_t gated_backward_bytes(const GatedBackwardArgs &a)
{
    const Parts p = parts_of(a);
    return p.dz + p.sums + p.weights + p.product;
}

hipError_t launch_gated_backward(const GatedBackwardArgs &a)
{
    return a.dtype == DTYPE_BF16 ? backward<__bf16>(a) : backward<float>(a);
}

uint64_t gated_mx_bytes(const GatedMxArgs &a) { return gated_mx_gemm_bytes(mx_args(a)); }

hipError_t launch_gated_mx(const GatedMxArgs &a)
{
    return gated_mx_gemm(mx_args(a), a.dtype, a.ws, a.stream);
}

}  // namespace whtmix
