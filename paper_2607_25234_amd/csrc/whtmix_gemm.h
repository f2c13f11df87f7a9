// Matrix products on the matrix cores: what the kernels of the three element
// types share, the epilogue first.
#pragma once

#include "whtmix_vec.h"

namespace whtmix {

// How an operand lies in memory: k contiguous, or its rows (the output's
// dimension) contiguous.
enum Layout { K_CONTIGUOUS = 0, K_STRIDED = 1 };

// out [M][N] = act(A B + bias) + residual with A [M][K] and B [K][N].
struct GemmArgs {
    const void *a, *b;
    const uint8_t *as, *bs;     // block scales (8-bit operands)
    int64_t as_ld, bs_ld;       // bytes between their rows, whole dwords
    int64_t lda, ldb;           // elements between k rows or between output rows
    int64_t a_rows, a_k, b_rows, b_k;   // what the operands' memory holds (packed ones: padded)
    int64_t M, N, K;
    const float *bias;          // [N] or null
    const void *residual;       // [M][N] of the output's type, or null
    void *y;                    // [M][N], or null with yq
    void *z;                    // [M][N] before the activation, or null
    uint8_t *yq, *ys;           // 8-bit output and its scales
    int act;
    float *part;                // split: [splits][M][N] partial sums, or null
    int64_t k_per;              // k of one split
};

template <typename T>
__device__ __forceinline__ void load8(const T *p, int n, float (&v)[8])
{
    if constexpr (Chunk<T>::N == 8) {
        Chunk<T>::load(p, n, v);
    } else {
        Chunk<T>::load(p, n, *(float(*)[4])v);
        Chunk<T>::load(p + 4, n - 4, *(float(*)[4])(v + 4));
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, int n, const float (&v)[8])
{
    if constexpr (Chunk<T>::N == 8) {
        Chunk<T>::store(p, n, v);
    } else {
        Chunk<T>::store(p, n, *(const float(*)[4])v);
        Chunk<T>::store(p + 4, n - 4, *(const float(*)[4])(v + 4));
    }
}

// Eight values of row m from column n on, the first cnt of them real, in block-scaled 8 bits;
// four neighbouring lanes hold a block of 32 columns and call this together.
__device__ __forceinline__ void store_mx8(float (&v)[8], int cnt, bool live, int64_t m, int64_t n,
                                          int64_t width, uint8_t *q, uint8_t *scales)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= cnt) v[i] = 0.f;
        top = max(top, mx_magnitude(v[i]));
    }
    top = max(top, quad_xor<0>(top));
    top = max(top, quad_xor<1>(top));
    const uint32_t byte = mx_scale_byte(top);
    const float inv = mx_inverse(byte);
    if (live && n < width) {
        *(u32x2 *)(q + m * width + n) =
            (u32x2){mx_pack(v[0], v[1], v[2], v[3], inv), mx_pack(v[4], v[5], v[6], v[7], inv)};
        if (n % kMxBlock == 0) scales[m * (width / kMxBlock) + n / kMxBlock] = (uint8_t)byte;
    }
}

// Eight sums of row m from column n on, to the outputs.  With 8-bit output
// four neighbouring lanes hold a block of 32 columns and call this together.
template <typename T>
__device__ __forceinline__ void finish8(const GemmArgs &g, int64_t m, int64_t n, float (&v)[8])
{
    const int cnt = m < g.M ? (int)min((int64_t)8, max((int64_t)0, g.N - n)) : 0;
    const int64_t at = m * g.N + n;
    if (g.bias) {
        float b[8];
        load8(g.bias + n, (int)min((int64_t)8, g.N - n), b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += b[i];
    }
    if (g.z && cnt > 0) store8((T *)g.z + at, cnt, v);
    with_act(g.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = act_of<decltype(act)::value>(v[i]);
    });
    if (g.residual) {
        float r[8];
        load8((const T *)g.residual + at, cnt, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    if (!g.yq) {
        if (cnt > 0) store8((T *)g.y + at, cnt, v);
        return;
    }
    store_mx8(v, cnt, m < g.M, m, n, (g.N + kMxBlock - 1) / kMxBlock * kMxBlock, g.yq, g.ys);
}

// A pointer that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const char *uniform(const char *p)
{
    const uint64_t v = (uint64_t)p;
    return (const char *)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) |
                          (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32);
}

// 16 bytes a lane from memory to LDS (lane order from the wave's address `lds`), counted by
// vmcnt.  In assembler, because the compiler would have every later LDS read wait for the
// copies in flight; the kernel waits for them itself, a step later.  No registers but m0 are
// written, which the compiler reserves (it may not be named as clobbered) and uses nowhere else
// in these kernels.
__device__ __forceinline__ void copy16(const char *base, uint32_t off, uint32_t lds)
{
    base = uniform(base);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds),
                 "v"(off), "s"(base)
                 : "memory");
}
__device__ __forceinline__ void copy4(const char *src, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds),
                 "v"(src)
                 : "memory");
}
__device__ __forceinline__ void copy16(const char *src, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds),
                 "v"(src)
                 : "memory");
}
// Until at most LEFT of the wave's copies (and loads) are in flight.
template <int LEFT> __device__ __forceinline__ void wait_copies()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}

// Workgroup -> tile and part of k.  Consecutive workgroups go round the 8 XCDs, each with its
// own L2: an XCD's are neighbours in the order below (a part's tiles together, in groups
// of 4 rows of tiles), so that those it holds at a time share operands.
__device__ __forceinline__ void place_tile(uint32_t id, uint32_t total, uint32_t tiles_m,
                                           uint32_t tiles_n, uint32_t &tm, uint32_t &tn,
                                           uint32_t &split)
{
    const uint32_t x = id % 8, tiles = tiles_m * tiles_n;
    const uint32_t s = x * (total / 8) + min(x, total % 8) + id / 8;
    split = s / tiles;
    const uint32_t t = s - split * tiles;
    const uint32_t group = t / (4 * tiles_n), first = group * 4;
    const uint32_t rows = min(4u, tiles_m - first), in = t - group * 4 * tiles_n;
    tm = first + in % rows;
    tn = in / rows;
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Orders a wave's own LDS accesses (no other wave touches them).
__device__ __forceinline__ void wave_lds_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int N, typename F, int I = 0> __device__ __forceinline__ void static_for(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<N, F, I + 1>(f);
    }
}

// A wave's 32 WM x 64 sums to the outputs, 32 rows at a time: from the matrix instructions'
// layout (lane: row l % 32, columns 8 (r / 4) + 4 (l / 32) + r % 4 of each 32)
// through the wave's LDS (kEpilogueFloats) to rows of 64, eight lanes a row, so that
// stores and the residual's loads are 16 bytes a lane and whole cache lines a row.  A lane's
// columns stay the same: their bias is read once.
constexpr int kEpilogueStride = 68;      // floats: rows 4 banks apart
constexpr int kEpilogueFloats = 32 * kEpilogueStride;

template <typename T, int WM>
__device__ __forceinline__ void finish_wave(const GemmArgs &g, float *lds, int64_t m0, int64_t n0,
                                            int64_t split, const f32x16 (&acc)[WM][2])
{
    const int lane = threadIdx.x & 63;
    float *w = lds + (lane & 31) * kEpilogueStride + (lane >> 5) * 4;
    const float *p = lds + (lane >> 3) * kEpilogueStride + (lane & 7) * 8;
    const int64_t n = n0 + (lane & 7) * 8;
    const int cnt = (int)max((int64_t)0, min((int64_t)8, g.N - n));
    const int rows = (int)min((int64_t)(32 * WM), g.M - m0) - (lane >> 3);   // left for this lane
    // Rows 32 i .. 32 i + 31, of which the lane takes every eighth: f(row of the tile, sums).
    auto each = [&](auto f) __attribute__((always_inline)) {
        static_for<WM>([&](auto part) __attribute__((always_inline)) {
            constexpr int I = decltype(part)::value;
            wave_lds_fence();
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *(f32x4 *)(w + 32 * j + 8 * r) =
                        (f32x4){acc[I][j][4 * r], acc[I][j][4 * r + 1], acc[I][j][4 * r + 2],
                                acc[I][j][4 * r + 3]};
            wave_lds_fence();
            float v[4][8];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                *(f32x4 *)v[r] = *(const f32x4 *)(p + 8 * r * kEpilogueStride);
                *(f32x4 *)(v[r] + 4) = *(const f32x4 *)(p + 8 * r * kEpilogueStride + 4);
            }
            f(32 * I, v);
        });
    };
    if (g.part) {
        float *to = g.part + (split * g.M + m0 + (lane >> 3)) * g.N + n;
        each([&](int i, float (&v)[4][8]) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (i + 8 * r < rows) store8(to + (int64_t)(i + 8 * r) * g.N, cnt, v[r]);
        });
        return;
    }
    float b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (g.bias) load8(g.bias + n, cnt, b);
    const int64_t at = (m0 + (lane >> 3)) * g.N + n;
    const T *res = (const T *)g.residual + at;
    T *y = (T *)g.y + at, *z = (T *)g.z + at;
    const int64_t width = (g.N + kMxBlock - 1) / kMxBlock * kMxBlock;
    with_act(g.act, [&](auto act) __attribute__((always_inline)) {
        constexpr int ACT = decltype(act)::value;
        each([&](int i, float (&v)[4][8]) __attribute__((always_inline)) {
            float e[4][8];
            if (g.residual) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    load8(res + (int64_t)(i + 8 * r) * g.N, i + 8 * r < rows ? cnt : 0, e[r]);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[r][k] += b[k];
                if (g.z && i + 8 * r < rows) store8(z + (int64_t)(i + 8 * r) * g.N, cnt, v[r]);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[r][k] = act_of<ACT>(v[r][k]);
                    if (g.residual) v[r][k] += e[r][k];
                }
                if (g.y) {
                    if (i + 8 * r < rows) store8(y + (int64_t)(i + 8 * r) * g.N, cnt, v[r]);
                } else if (n < width) {     // the four lanes of a block of 32 columns together
                    store_mx8(v[r], cnt, i + 8 * r < rows, m0 + (lane >> 3) + i + 8 * r, n, width,
                              g.yq, g.ys);
                }
            }
        });
    });
}

// Adds the parts' partial sums and finishes them: eight columns a thread, and where the parts
// are many, the workgroup's threads in GROUPS that take every GROUPS-th part, whose sums are
// then added in order.  A launch and the parts' loads: 4-5 us for one row of 16384 or 17 of 4096,
// 10 us for 3001 x 1000 float32.
template <typename T, int GROUPS>
__global__ void __launch_bounds__(256) split_sum_kernel(GemmArgs g, int splits)
{
    constexpr int kChunks = 256 / GROUPS;
    __shared__ float sums[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? kChunks : 1][9];
    const int64_t width = g.yq ? (g.N + kMxBlock - 1) / kMxBlock * kMxBlock : (g.N + 7) / 8 * 8;
    const int c = threadIdx.x % kChunks, first = threadIdx.x / kChunks;
    const int64_t i = ((int64_t)blockIdx.x * kChunks + c) * 8;
    const int64_t m = i / width, n = i - m * width;
    const int cnt = m < g.M ? (int)max((int64_t)0, min((int64_t)8, g.N - n)) : 0;
    const float *from = g.part + (m < g.M ? m * g.N + n : 0);
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.f;
    for (int s = first; s < splits; s += 4 * GROUPS) {       // four parts' loads in flight
        float p[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            load8(from + (int64_t)min(s + u * GROUPS, splits - 1) * g.M * g.N,
                  s + u * GROUPS < splits ? cnt : 0, p[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += p[u][k];
    }
    if constexpr (GROUPS > 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k) sums[first][c][k] = v[k];
        __syncthreads();
        if (first > 0) return;
#pragma unroll
        for (int f = 1; f < GROUPS; ++f)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += sums[f][c][k];
    }
    if (m < g.M) finish8<T>(g, m, n, v);    // 8-bit output: the four lanes of a block together
}

template <typename T> hipError_t launch_split_sum(const GemmArgs &g, int splits, hipStream_t stream)
{
    const int64_t width = g.yq ? mx_width(g.N) : (g.N + 7) / 8 * 8, chunks = g.M * width / 8;
    // 16 parts and more of an output that does not fill the device: 8 threads a chunk
    // (65536 sums of 128 parts: 33 us with one)
    if (splits >= 16 && chunks <= 1 << 16)
        split_sum_kernel<T, 8><<<dim3((uint32_t)((chunks + 31) / 32)), dim3(256), 0, stream>>>(g, splits);
    else
        split_sum_kernel<T, 1><<<dim3((uint32_t)((chunks + 255) / 256)), dim3(256), 0, stream>>>(g, splits);
    return hipGetLastError();
}

// Products of bf16 operands (whtmix_linear_bf16.hip), float32 ones (whtmix_linear_f32.hip)
// and block-scaled 8-bit ones (whtmix_linear_mx.hip), with `*_bytes` of workspace.
uint64_t gemm_bf16_bytes(const GemmArgs &g, Layout la, Layout lb);
hipError_t gemm_bf16(GemmArgs g, Layout la, Layout lb, void *ws, hipStream_t stream);
uint64_t gemm_f32_bytes(const GemmArgs &g);
hipError_t gemm_f32(const GemmArgs &g, Layout la, Layout lb, void *ws, hipStream_t stream);
// dz, its columns' partial sums (dzx_parts rows, or null) and dx in one kernel
// (whtmix_linear_dzx.hip), for calls that it takes.
bool dzx_takes(const LinearBackwardArgs &a);
int64_t dzx_parts(int64_t M);
hipError_t launch_dzx(const LinearBackwardArgs &a, void *dz, float *part);
uint64_t gemm_mx_bytes(const GemmArgs &g);
hipError_t gemm_mx(GemmArgs g, int dtype, void *ws, hipStream_t stream);

}  // namespace whtmix
