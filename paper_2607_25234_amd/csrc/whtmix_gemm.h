// Matrix products on the matrix cores: what the kernels of the three element
// types share, the epilogue first.
#pragma once

#include "whtmix_vec.h"

namespace whtmix {

// How an operand lies in memory: k contiguous, or its rows (the output's
// dimension) contiguous.
enum Layout { K_CONTIGUOUS = 0, K_STRIDED = 1 };

// What a product is beside the plain one:
//   GATED   two products of the same A, act(A B + bias) o (A B2 + bias2): a tile's columns are the
//           first's and the second's of the same n, 32 of each a wave, which has both sums of an
//           output in its registers
//   HALVES  the columns from `half` on are those of another output, y2; both have half_n
//   TWO_K   the k from `half` on are those of another B, b2, whose k starts at 0 again
enum Form { PLAIN = 0, GATED = 1, HALVES = 2, TWO_K = 3 };

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
    const void *b2;             // GATED: like b, bs, ldb, bias and z; TWO_K
    const uint8_t *bs2;
    int64_t ldb2, bs2_ld;
    const float *bias2;
    void *z2;
    void *y2;                   // HALVES
    int64_t half, half_n;
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

template <typename T, int FORM, int WM>
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
    if constexpr (FORM == HALVES) {     // whole chunks of 8 columns on either side
        const bool second = n >= g.half;
        const int64_t in = second ? n - g.half : n;
        const int own = (int)max((int64_t)0, min((int64_t)cnt, g.half_n - in));
        T *to = (T *)(second ? g.y2 : g.y) + (m0 + (lane >> 3)) * g.half_n + in;
        each([&](int i, float (&v)[4][8]) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (i + 8 * r < rows) store8(to + (int64_t)(i + 8 * r) * g.half_n, own, v[r]);
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

// Eight sums of both products of row m from column n on, to the outputs of a gated product.
template <typename T, int ACT>
__device__ __forceinline__ void finish_gated8(const GemmArgs &g, int64_t m, int64_t n, int cnt,
                                              bool live, float (&v)[8], float (&u)[8])
{
    const int64_t at = m * g.N + n;
    if (live && cnt > 0) {
        if (g.z) store8((T *)g.z + at, cnt, v);
        if (g.z2) store8((T *)g.z2 + at, cnt, u);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = act_of<ACT>(v[k]) * u[k];
    if (g.y) {
        if (live && cnt > 0) store8((T *)g.y + at, cnt, v);
    } else {
        const int64_t width = (g.N + kMxBlock - 1) / kMxBlock * kMxBlock;
        store_mx8(v, cnt, live, m, n, width, g.yq, g.ys);
    }
}

// A wave's 32 WM x 32 pairs of sums to the outputs of a gated product: as finish_wave, but four
// lanes a row, each with 8 columns of both.  n0: of the wave's columns.
template <typename T, int WM>
__device__ __forceinline__ void finish_gated_wave(const GemmArgs &g, float *lds, int64_t m0,
                                                  int64_t n0, int64_t split,
                                                  const f32x16 (&acc)[WM][2])
{
    const int lane = threadIdx.x & 63;
    float *w = lds + (lane & 31) * kEpilogueStride + (lane >> 5) * 4;
    // 16 lanes, a cycle of an LDS read, take rows 0, 1, 8 and 9 of 16 (and so on): 16 different
    // groups of 4 banks.
    const int row = (lane >> 2 & 1) | (lane >> 4) << 1 | (lane >> 3 & 1) << 3;
    const float *p = lds + row * kEpilogueStride + (lane & 3) * 8;
    const int64_t n = n0 + (lane & 3) * 8;
    const int cnt = (int)max((int64_t)0, min((int64_t)8, g.N - n));
    const int rows = (int)min((int64_t)(32 * WM), g.M - m0) - row;     // left for this lane
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
            float v[2][8], u[2][8];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float *q = p + 16 * r * kEpilogueStride;
                *(f32x4 *)v[r] = *(const f32x4 *)q;
                *(f32x4 *)(v[r] + 4) = *(const f32x4 *)(q + 4);
                *(f32x4 *)u[r] = *(const f32x4 *)(q + 32);
                *(f32x4 *)(u[r] + 4) = *(const f32x4 *)(q + 36);
            }
            f(32 * I, v, u);
        });
    };
    if (g.part) {       // [splits][2][M][N]
        float *to = g.part + (2 * split * g.M + m0 + row) * g.N + n;
        each([&](int i, float (&v)[2][8], float (&u)[2][8]) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (i + 16 * r < rows) {
                    store8(to + (int64_t)(i + 16 * r) * g.N, cnt, v[r]);
                    store8(to + (i + 16 * r + g.M) * g.N, cnt, u[r]);
                }
        });
        return;
    }
    float b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float b2[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (g.bias) load8(g.bias + n, cnt, b);
    if (g.bias2) load8(g.bias2 + n, cnt, b2);
    if (n0 >= (g.N + kMxBlock - 1) / kMxBlock * kMxBlock) return;
    with_act(g.act, [&](auto act) __attribute__((always_inline)) {
        constexpr int ACT = decltype(act)::value;
        each([&](int i, float (&v)[2][8], float (&u)[2][8]) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[r][k] += b[k], u[r][k] += b2[k];
                finish_gated8<T, ACT>(g, m0 + row + i + 16 * r, n, cnt, i + 16 * r < rows, v[r],
                                      u[r]);
            }
        });
    });
}

// Adds the parts' partial sums and finishes them: eight columns a thread, and where the parts
// are many, the workgroup's threads in GROUPS that take every GROUPS-th part, whose sums are
// then added in order.  A launch and the parts' loads: 4-5 us for one row of 16384 or 17 of 4096,
// 10 us for 3001 x 1000 float32.
template <typename T, int FORM, int GROUPS>
__global__ void __launch_bounds__(256) split_sum_kernel(GemmArgs g, int splits)
{
    constexpr int kChunks = 256 / GROUPS, P = FORM == GATED ? 2 : 1;
    __shared__ float sums[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? kChunks : 1][8 * P + 1];
    const int64_t width = g.yq ? (g.N + kMxBlock - 1) / kMxBlock * kMxBlock : (g.N + 7) / 8 * 8;
    const int c = threadIdx.x % kChunks, first = threadIdx.x / kChunks;
    const int64_t i = ((int64_t)blockIdx.x * kChunks + c) * 8;
    const int64_t m = i / width, n = i - m * width;
    const int cnt = m < g.M ? (int)max((int64_t)0, min((int64_t)8, g.N - n)) : 0;
    const float *from = g.part + (m < g.M ? m * g.N + n : 0);
    float v[P][8];
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[q][k] = 0.f;
    for (int s = first; s < splits; s += 4 * GROUPS) {       // four parts' loads in flight
        float p[4][P][8];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int q = 0; q < P; ++q)
                load8(from + (int64_t)(min(s + u * GROUPS, splits - 1) * P + q) * g.M * g.N,
                      s + u * GROUPS < splits ? cnt : 0, p[u][q]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[q][k] += p[u][q][k];
    }
    if constexpr (GROUPS > 1) {
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) sums[first][c][8 * q + k] = v[q][k];
        __syncthreads();
        if (first > 0) return;
#pragma unroll
        for (int f = 1; f < GROUPS; ++f)
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[q][k] += sums[f][c][8 * q + k];
    }
    if (m >= g.M) return;
    // 8-bit output: the four lanes of a block together
    if constexpr (FORM == GATED) {
        float b[8], b2[8];
        load8(g.bias ? g.bias + n : g.part, g.bias ? cnt : 0, b);
        load8(g.bias2 ? g.bias2 + n : g.part, g.bias2 ? cnt : 0, b2);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[0][k] += b[k], v[1][k] += b2[k];
        with_act(g.act, [&](auto act) {
            finish_gated8<T, decltype(act)::value>(g, m, n, cnt, true, v[0], v[1]);
        });
    } else if constexpr (FORM == HALVES) {
        const bool second = n >= g.half;
        const int64_t in = second ? n - g.half : n;
        store8((T *)(second ? g.y2 : g.y) + m * g.half_n + in,
               (int)max((int64_t)0, min((int64_t)cnt, g.half_n - in)), v[0]);
    } else {
        finish8<T>(g, m, n, v[0]);
    }
}

template <typename T, int FORM>
hipError_t launch_split_sum(const GemmArgs &g, int splits, hipStream_t stream)
{
    const int64_t width = g.yq ? mx_width(g.N) : (g.N + 7) / 8 * 8, chunks = g.M * width / 8;
    // 16 parts and more of an output that does not fill the device: 8 threads a chunk
    // (65536 sums of 128 parts: 33 us with one)
    if (splits >= 16 && chunks <= 1 << 16)
        split_sum_kernel<T, FORM, 8><<<dim3((uint32_t)((chunks + 31) / 32)), dim3(256), 0, stream>>>(g, splits);
    else
        split_sum_kernel<T, FORM, 1><<<dim3((uint32_t)((chunks + 255) / 256)), dim3(256), 0, stream>>>(g, splits);
    return hipGetLastError();
}

// Products of bf16 operands (whtmix_linear_bf16.hip), float32 ones (whtmix_linear_f32.hip)
// and block-scaled 8-bit ones (whtmix_linear_mx.hip), with `*_bytes` of workspace.
uint64_t gemm_bf16_bytes(const GemmArgs &g, Layout la, Layout lb);
hipError_t gemm_bf16(GemmArgs g, Layout la, Layout lb, void *ws, hipStream_t stream);
uint64_t gemm_f32_bytes(const GemmArgs &g);
hipError_t gemm_f32(const GemmArgs &g, Layout la, Layout lb, void *ws, hipStream_t stream);
// The other forms (whtmix_gated_bf16.hip, whtmix_linear_f32.hip, whtmix_gated_mx.hip): GATED with
// K_CONTIGUOUS a and K_STRIDED b, HALVES with both K_STRIDED, TWO_K (bf16, whole steps of k and
// aligned operands) with both K_CONTIGUOUS.
uint64_t gemm_bf16_bytes(const GemmArgs &g, Form form);
hipError_t gemm_bf16(GemmArgs g, Form form, void *ws, hipStream_t stream);
uint64_t gemm_f32_bytes(const GemmArgs &g, Form form);
hipError_t gemm_f32(const GemmArgs &g, Form form, void *ws, hipStream_t stream);
uint64_t gated_mx_gemm_bytes(const GemmArgs &g);
hipError_t gated_mx_gemm(GemmArgs g, int dtype, void *ws, hipStream_t stream);
// dz, its columns' partial sums (dzx_parts rows, or null) and dx in one kernel
// (whtmix_linear_dzx.hip), for calls that it takes.
bool dzx_takes(const LinearBackwardArgs &a);
int64_t dzx_parts(int64_t M);
hipError_t launch_dzx(const LinearBackwardArgs &a, void *dz, float *part);
// The same of a gated product (whtmix_gated_dzx.hip): dz [M] rows a pitch apart, its second half
// `width` columns on, or null; part [parts][2][N].
bool gated_dzx_takes(const GatedBackwardArgs &a);
int64_t gated_dzx_parts(const GatedBackwardArgs &a);
int64_t gated_dzx_pitch(int64_t N, int64_t width);
hipError_t launch_gated_dzx(const GatedBackwardArgs &a, int64_t width, void *dz, float *part);
uint64_t gemm_mx_bytes(const GemmArgs &g);
hipError_t gemm_mx(GemmArgs g, int dtype, void *ws, hipStream_t stream);

}  // namespace whtmix
