// Matrix products with bias, activation and residual in the epilogue, and
// their gradients.
//
//   z = x w + bias,  y = act(z) + residual
//   dz = dy act'(z),  dx = dz w^T,  dw = x^T dz,  dbias = column sums of dz
//
// bf16 and block-scaled 8 bits go to the tile kernel of whtmix_gemm_tile.h; float32 has its
// own here: a 128 x 128 tile of four waves, operands split into three bf16 terms on
// their way to LDS, products on v_mfma_f32_32x32x16_bf16, sums in float32.
#include "whtmix_gemm.h"

#include <algorithm>

namespace whtmix {
namespace {

constexpr int kTile = 128, kStep = 32;
constexpr int kRowBytes = 80;      // K_CONTIGUOUS: 32 bf16 and 16 bytes of padding
constexpr int kKBytes = 320;       // K_STRIDED: 128 bf16 and 64 bytes of padding
constexpr int kPlane = 10240;      // either way
constexpr int kF32Row = kTile + 4; // float32 staging: floats of one k
// Three bf16 terms hold a float32 below 2^128 - 2^119 (above, the first rounds to Inf) and from
// 2^-100 up (below, the last is subnormal); rows mixed with smaller values lose less than 2^-128.
constexpr float kSplitMax = 0x1.ffp127f, kSplitMin = 0x1p-95f;
static_assert(kTile * kRowBytes == kPlane && kStep * kKBytes == kPlane, "planes");

constexpr int P = 3;               // bf16 terms of a float32

// Sixteen elements of an operand in a thread's registers, four times four along memory: a
// row's chunks are neighbouring lanes'.
template <Layout L> struct Stage {
    float v[4][4];
    // Chunk i of the thread: (row, k) of its first element.
    static __device__ __forceinline__ void place(int i, int &row, int &k)
    {
        const int c = i * 256 + threadIdx.x;
        if (L == K_CONTIGUOUS) row = c >> 3, k = (c & 7) * 4;
        else k = c >> 5, row = (c & 31) * 4;
    }
    __device__ __forceinline__ void load(const void *p, int64_t ld, int64_t R, int64_t K,
                                         int64_t r0, int64_t k0)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int row, k;
            place(i, row, k);
            const int64_t outer = L == K_CONTIGUOUS ? r0 + row : k0 + k,
                          inner = L == K_CONTIGUOUS ? k0 + k : r0 + row;
            const int64_t left = outer < (L == K_CONTIGUOUS ? R : K)
                                     ? (L == K_CONTIGUOUS ? K : R) - inner : 0;
            const int n = (int)min((int64_t)4, max((int64_t)0, left));
            Chunk<float>::load((const float *)p + (n ? outer * ld + inner : 0), n, v[i]);
        }
    }
    // As float32, [k][row], for operands that do not split.
    __device__ __forceinline__ void store_f32(float *lds) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int row, k;
            place(i, row, k);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                lds[(k + (L == K_CONTIGUOUS ? j : 0)) * kF32Row + row +
                    (L == K_CONTIGUOUS ? 0 : j)] = v[i][j];
        }
    }
    // The largest magnitudes staged so far by chunk.  (A NaN is passed over: it makes its
    // row's sums NaN either way.)
    __device__ __forceinline__ void largest(float (&top)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top[i] = fmaxf(fmaxf(top[i], fabsf(v[i][0])), fabsf(v[i][1]));
            top[i] = fmaxf(fmaxf(top[i], fabsf(v[i][2])), fabsf(v[i][3]));
        }
    }
    __device__ __forceinline__ void store(char *lds)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int row, k;
            place(i, row, k);
            char *p = lds + (L == K_CONTIGUOUS ? row * kRowBytes + k * 2 : k * kKBytes + row * 2);
#pragma unroll
            for (int s = 0; s < P; ++s) {
                const uint32_t w0 = pack_bf16(v[i][0], v[i][1]), w1 = pack_bf16(v[i][2], v[i][3]);
                *(u32x2 *)(p + s * kPlane) = (u32x2){w0, w1};
                if (s + 1 < P) {
                    v[i][0] -= bits_f32(w0 << 16);
                    v[i][1] -= bits_f32(w0 & 0xffff0000u);
                    v[i][2] -= bits_f32(w1 << 16);
                    v[i][3] -= bits_f32(w1 & 0xffff0000u);
                }
            }
        }
    }
};

// The operand of a 32x32x16 product: lane l holds row l % 32, k 8 (l / 32) + 0..7.
// K_STRIDED planes are read through the transposing LDS load: a group of 16
// lanes reads 4 k of 16 rows and each lane gets one row's 4 k.
template <Layout L> __device__ __forceinline__ bf16x8 fragment(const char *plane, int row0, int k0)
{
    const int lane = threadIdx.x & 63;
    if constexpr (L == K_CONTIGUOUS) {
        return *(const bf16x8 *)(plane + (row0 + (lane & 31)) * kRowBytes +
                                 (k0 + (lane >> 5) * 8) * 2);
    } else {
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s4 lds_s4;
        const int k = k0 + (lane >> 5) * 8 + ((lane >> 2) & 3);
        const int r = row0 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
        const char *p = plane + k * kKBytes + r * 2;
        union {
            s4 h[2];
            bf16x8 f;
        } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)p);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(p + 4 * kKBytes));
        return u.f;
    }
}

// The tile again with float32 products (v_mfma_f32_32x32x2_f32).
template <Layout LA, Layout LB>
__device__ __forceinline__ void float32_tile(const GemmArgs &g, Stage<LA> &sa,
                                          Stage<LB> &sb, float *lds, int64_t m0, int64_t n0,
                                          int64_t kbeg, int64_t kend, int wm, int wn,
                                          f32x16 (&acc)[2][2])
{
    const int lane = threadIdx.x & 63;
    float *la = lds, *lb = lds + kStep * kF32Row;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    for (int64_t k = kbeg; k < kend; k += kStep) {
        sa.load(g.a, g.lda, g.M, kend, m0, k);
        sb.load(g.b, g.ldb, g.N, kend, n0, k);
        __syncthreads();
        sa.store_f32(la);
        sb.store_f32(lb);
        __syncthreads();
        for (int kk = 0; kk < kStep; kk += 2) {
            const float *pa = la + (kk + (lane >> 5)) * kF32Row + wm + (lane & 31);
            const float *pb = lb + (kk + (lane >> 5)) * kF32Row + wn + (lane & 31);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(pb[32 * j], pa[32 * i],
                                                                     acc[i][j], 0, 0, 0);
        }
    }
}

template <Layout LA, Layout LB>
__global__ void __launch_bounds__(256) gemm_kernel(GemmArgs g)
{
    __shared__ __attribute__((aligned(16))) char lds[2 * P * kPlane > 4 * kEpilogueFloats * 4
                                                         ? 2 * P * kPlane
                                                         : 4 * kEpilogueFloats * 4];
    const int wave = threadIdx.x >> 6;
    const int64_t m0 = (int64_t)blockIdx.x * kTile, n0 = (int64_t)blockIdx.y * kTile;
    const int64_t kbeg = (int64_t)blockIdx.z * g.k_per, kend = min(g.K, kbeg + g.k_per);
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    char *la = lds, *lb = lds + P * kPlane;
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    Stage<LA> sa;
    Stage<LB> sb;
    float top_a[4] = {0.f, 0.f, 0.f, 0.f}, top_b[4] = {0.f, 0.f, 0.f, 0.f};  // of the splits
    sa.load(g.a, g.lda, g.M, kend, m0, kbeg);
    sb.load(g.b, g.ldb, g.N, kend, n0, kbeg);
    for (int64_t k = kbeg; k < kend; k += kStep) {
        __syncthreads();
        sa.largest(top_a);
        sb.largest(top_b);
        sa.store(la);
        sb.store(lb);
        if (k + kStep < kend) {
            sa.load(g.a, g.lda, g.M, kend, m0, k + kStep);
            sb.load(g.b, g.ldb, g.N, kend, n0, k + kStep);
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kStep; kk += 16) {
            bf16x8 fa[P][2], fb[P][2];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    fa[p][i] = fragment<LA>(la + p * kPlane, wm + 32 * i, kk);
                    fb[p][i] = fragment<LB>(lb + p * kPlane, wn + 32 * i, kk);
                }
            // Of the nine products of three terms the six largest: what is left
            // out is below 2^-24 of |x| |w|.
#pragma unroll
            for (int s = P - 1; s >= 0; --s)
#pragma unroll
                for (int p = 0; p <= s; ++p)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                                fb[s - p][j], fa[p][i], acc[i][j], 0, 0, 0);
        }
    }
    auto bad = [](float top) { return top >= kSplitMax || (top != 0.f && top < kSplitMin); };
    // A chunk's elements along k are of one row (or four); one that does not split sends the
    // whole tile through float32 products.
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) any = any || bad(top_a[i]) || bad(top_b[i]);
    if (__syncthreads_or(any))
        float32_tile(g, sa, sb, (float *)lds, m0, n0, kbeg, kend, wm, wn, acc);
    __syncthreads();
    float *out = (float *)lds + wave * kEpilogueFloats;
    finish_wave<float>(g, out, m0 + wm, n0 + wn, blockIdx.z, acc);
}

// How many parts k is split into: enough workgroups for the device where the
// output has few tiles, each with at least 8 steps of k.
int64_t splits_of(int64_t M, int64_t N, int64_t K)
{
    const int64_t tiles = ((M + kTile - 1) / kTile) * ((N + kTile - 1) / kTile);
    const int64_t steps = (K + kStep - 1) / kStep;
    return std::max<int64_t>(1, std::min<int64_t>(512 / std::max<int64_t>(1, tiles), steps / 8));
}

uint64_t gemm_bytes(int64_t M, int64_t N, int64_t K)
{
    const int64_t s = splits_of(M, N, K);
    return s > 1 ? (uint64_t)s * M * N * 4 : 0;
}

template <Layout LA, Layout LB>
hipError_t run_gemm(GemmArgs g, float *ws, hipStream_t stream)
{
    const int64_t s = splits_of(g.M, g.N, g.K);
    const int64_t steps = (g.K + kStep - 1) / kStep;
    g.k_per = (steps + s - 1) / s * kStep;
    const int64_t splits = (g.K + g.k_per - 1) / g.k_per;
    g.part = splits > 1 ? ws : nullptr;
    const dim3 grid((uint32_t)((g.M + kTile - 1) / kTile), (uint32_t)((g.N + kTile - 1) / kTile),
                    (uint32_t)splits);
    gemm_kernel<LA, LB><<<grid, dim3(256), 0, stream>>>(g);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    return launch_split_sum<float>(g, (int)splits, stream);
}

// dz = dy act'(z), with the columns' sums of the unrounded values: 32 threads across
// 256 columns, 8 rows at a time, four of them in flight a thread; the workgroup's 8
// sums of a column are added in order.
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
    if constexpr (std::is_same_v<T, __bf16>) {
        return gemm_bf16(g, la, lb, ws, stream);
    } else {
        float *w = (float *)ws;
        if (la == K_CONTIGUOUS && lb == K_STRIDED)
            return run_gemm<K_CONTIGUOUS, K_STRIDED>(g, w, stream);
        if (la == K_CONTIGUOUS) return run_gemm<K_CONTIGUOUS, K_CONTIGUOUS>(g, w, stream);
        return run_gemm<K_STRIDED, K_STRIDED>(g, w, stream);
    }
}

uint64_t product_bytes(const GemmArgs &g, Layout la, Layout lb, int dtype)
{
    return dtype == DTYPE_BF16 ? gemm_bf16_bytes(g, la, lb) : gemm_bytes(g.M, g.N, g.K);
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
    if (a.act != ACT_NONE) l.dz = align256((uint64_t)a.M * a.N * e);
    if (a.dbias) l.part = align256((uint64_t)dz_parts(a.M, a.N) * a.N * 4);
    const void *dz = a.act != ACT_NONE ? nullptr : a.dy;    // a workspace's address is aligned
    if (a.dx) l.product = product_bytes(dx_args(a, dz), K_CONTIGUOUS, K_CONTIGUOUS, a.dtype);
    if (a.dw)
        l.product = std::max(l.product, product_bytes(dw_args(a, dz), K_STRIDED, K_STRIDED, a.dtype));
    return l;
}

template <typename T> hipError_t linear_backward(const LinearBackwardArgs &a)
{
    const BackwardLayoutBytes l = backward_bytes(a);
    char *ws = (char *)a.ws;
    T *dz = (T *)ws;
    float *part = (float *)(ws + l.dz);
    void *rest = ws + l.dz + l.part;
    hipError_t e;
    if (a.act != ACT_NONE || a.dbias) {
        const int64_t parts = dz_parts(a.M, a.N);
        const int64_t per = (a.M + parts - 1) / parts;
        const dim3 grid((uint32_t)((a.N + kDzCols - 1) / kDzCols),
                        (uint32_t)((a.M + per - 1) / per));
        dz_kernel<T><<<grid, dim3(256), 0, a.stream>>>(
            (const T *)a.dy, (const T *)a.z, a.dx || a.dw ? dz : nullptr,
            a.dbias ? part : nullptr, a.M, a.N, per, a.act);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (a.dbias && (e = launch_column_sum(part, grid.y, a.N, a.dbias, a.stream)) != hipSuccess)
            return e;
    }
    const void *d = a.act != ACT_NONE ? (const void *)dz : a.dy;
    if (a.dx && (e = product<T>(dx_args(a, d), K_CONTIGUOUS, K_CONTIGUOUS, rest, a.stream)) !=
                    hipSuccess)
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
