// Root-mean-square norm with the residual's addition, its backward pass, and
// the block-scaled 8-bit form (quantise, dequantise).
//
//   t = x + residual          (float32; h = t rounded to the stream's type)
//   y = t * rstd * w,         rstd = 1 / sqrt(mean(t^2) + eps)
//   dx = dh + rstd * (g - n * mean(g n)),   n = h rstd, g = dy w
//   dw = sum over rows of dy n
//
// All of it is bound by memory: a row is read once into the registers of G
// lanes (R chunks of 16 bytes each), its sum of squares goes over the lanes,
// and y and h leave from the registers.  Sums are float32: a lane's over its
// own values, then a fixed tree, so results do not change from run to run.
#include "whtmix_row.h"

#include <algorithm>

namespace whtmix {
namespace {

enum Mode { MODE_NORM = 0, MODE_NORM_MX = 1, MODE_QUANT = 2 };

// Sum over the G lanes that hold a row; `part` is a float of LDS for each wave of the
// workgroup, for rows wider than a wave.
template <int G> __device__ __forceinline__ float row_sum(float v, float *part)
{
#pragma unroll
    for (int d = 1; d < (G < 64 ? G : 64); d <<= 1) v += __shfl_xor(v, d);
    if constexpr (G > 64) {
        part += threadIdx.x / G * (G / 64);
        __syncthreads();   // the reads of the sum before
        if ((threadIdx.x & 63) == 0) part[threadIdx.x % G >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < G / 64; ++i) v += part[i];
    }
    return v;
}

// Two sums over a row's lanes at once; `part` is another one (2 * G / 64 floats) than in
// the call before, whose reads may still be under way.
template <int G> __device__ __forceinline__ void row_sums(float &u, float &v, float *part)
{
    static_assert(G <= 64 || G >= 256, "a workgroup's waves hold one row");
#pragma unroll
    for (int d = 1; d < (G < 64 ? G : 64); d <<= 1) u += __shfl_xor(u, d), v += __shfl_xor(v, d);
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0)
            part[threadIdx.x >> 6] = u, part[G / 64 + (threadIdx.x >> 6)] = v;
        __syncthreads();
        u = v = 0.f;
#pragma unroll
        for (int i = 0; i < G / 64; ++i) u += part[i], v += part[G / 64 + i];
    }
}

struct NormKernelArgs {
    const void *x, *residual;
    const float *weight;
    void *y, *h, *q;
    uint8_t *scales;
    int64_t rows, C, ldx;
    float eps;
};

// One row on G lanes.  R chunks a lane stay in registers; with R = 0 (rows
// wider than that) the row is read twice.  Bound by memory, and narrow rows share a workgroup.
// Measured (x, residual, y and h): 262144 x 128 bf16 45 us, 268 MB at 6.0 TB/s; 16384 x 4096 99 us,
// 537 MB at 5.4 TB/s; 8192 x 4096 with 8-bit output 50-54 us, 237 MB at 4.4-4.7 TB/s; float32 32768 x 128
// 13 us (67 MB, the caches' rate); one row of 4096 2.6 us, the latency of its loads and of
// one sum.
template <typename T, int G, int R, int MODE>
__global__ void __launch_bounds__(G > 256 ? G : 256) norm_kernel(NormKernelArgs a)
{
    constexpr int N = Chunk<T>::N;
    constexpr int kRows = G > 256 ? 1 : 256 / G;
    __shared__ float part[16];
    const int lane = threadIdx.x % G;
    const int64_t width = MODE == MODE_NORM ? a.C : (a.C + kMxBlock - 1) / kMxBlock * kMxBlock;
    for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows;
         base += (int64_t)gridDim.x * kRows) {
        const int64_t row = base + threadIdx.x / G;
        // Rows past the end go through the exchanges with zeros and store nothing.
        const bool live = row < a.rows;
        const T *x = (const T *)a.x + (live ? row * a.ldx : 0);
        const T *r = a.residual ? (const T *)a.residual + (live ? row * a.C : 0) : nullptr;
        T *y = MODE == MODE_NORM ? (T *)a.y + (live ? row * a.C : 0) : nullptr;
        T *h = a.h ? (T *)a.h + (live ? row * a.C : 0) : nullptr;
        uint8_t *q = MODE == MODE_NORM ? nullptr : (uint8_t *)a.q + (live ? row * width : 0);
        uint8_t *sc = MODE == MODE_NORM ? nullptr
                                        : a.scales + (live ? row * (width / kMxBlock) : 0);

        auto load = [&](int64_t c, float (&v)[N]) {
            const int n = live ? (int)min((int64_t)N, max((int64_t)0, a.C - c)) : 0;
            Chunk<T>::load(x + c, n, v);
            if (r) {
                float e[N];
                Chunk<T>::load(r + c, n, e);
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += e[i];
            }
        };
        auto emit = [&](int64_t c, float (&v)[N], float rstd) {
            const int n = (int)min((int64_t)N, a.C - c);
            if (h && live && n > 0) Chunk<T>::store(h + c, n, v);
            if (MODE != MODE_QUANT) {
                float w[N];
                Chunk<float>::load(a.weight + c, n, *(float(*)[4])w);
                if constexpr (N == 8)
                    Chunk<float>::load(a.weight + c + 4, n - 4, *(float(*)[4])(w + 4));
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = v[i] * rstd * w[i];
            }
            if (MODE == MODE_NORM) {
                if (live && n > 0) Chunk<T>::store(y + c, n, v);
            } else if (live) {
                store_mx<T>(v, q, sc, c);
            }
        };

        if constexpr (R > 0) {
            float v[R][N];
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < R; ++j) load(((int64_t)j * G + lane) * N, v[j]);
            if (MODE != MODE_QUANT) {
#pragma unroll
                for (int j = 0; j < R; ++j)
#pragma unroll
                    for (int i = 0; i < N; ++i) s = fmaf(v[j][i], v[j][i], s);
                s = rsqrtf(row_sum<G>(s, part) / (float)a.C + a.eps);
            }
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int64_t c = ((int64_t)j * G + lane) * N;
                if (c < width) emit(c, v[j], s);
            }
        } else {
            float s = 0.f;
            if (MODE != MODE_QUANT) {
                for (int64_t c = (int64_t)lane * N; c < a.C; c += (int64_t)G * N) {
                    float v[N];
                    load(c, v);
#pragma unroll
                    for (int i = 0; i < N; ++i) s = fmaf(v[i], v[i], s);
                }
                s = rsqrtf(row_sum<G>(s, part) / (float)a.C + a.eps);
            }
            // A block's lanes are in the loop together: `width` is a multiple of 32.
            for (int64_t c = (int64_t)lane * N; c < width; c += (int64_t)G * N) {
                float v[N];
                load(c, v);
                emit(c, v, s);
            }
        }
    }
}

template <typename T, int G, int R, int MODE>
hipError_t run_norm(const NormArgs &a)
{
    constexpr int kRows = G > 256 ? 1 : 256 / G;
    const NormKernelArgs k{a.x, a.residual, a.weight, a.y, a.h, a.q, a.scales,
                           a.rows, a.C, a.ldx, a.eps};
    const int64_t blocks = std::min<int64_t>((a.rows + kRows - 1) / kRows, kMaxBlocks);
    norm_kernel<T, G, R, MODE><<<dim3((uint32_t)blocks), dim3(G > 256 ? G : 256), 0, a.stream>>>(k);
    return hipGetLastError();
}

// Chunks of a row -> lanes and chunks a lane: one chunk a lane up to 512 lanes.  With two or
// more on fewer lanes: 65536 x 512 float32 114 and 95 us (64 x 2, 128 x 1), 16384 x 4096 bf16 102
// and 99, 3001 x 1111 float32 14 and 11 (256 x 2, 512 x 1), 8192 x 8192 bf16 110 and 103 us (256
// x 4, 512 x 2); 8-bit output of 8192 x 8192 124 and 100 us (1024 x 1, 512 x 2).
template <typename T, int MODE> hipError_t pick_norm(const NormArgs &a)
{
    const int64_t width = MODE == MODE_NORM ? a.C : mx_width(a.C);
    const int64_t n = (width + Chunk<T>::N - 1) / Chunk<T>::N;
    if (n <= 8) return run_norm<T, 8, 1, MODE>(a);
    if (n <= 16) return run_norm<T, 16, 1, MODE>(a);
    if (n <= 32) return run_norm<T, 32, 1, MODE>(a);
    if (n <= 64) return run_norm<T, 64, 1, MODE>(a);
    if (n <= 128) return run_norm<T, 128, 1, MODE>(a);
    if (n <= 256) return run_norm<T, 256, 1, MODE>(a);
    if (n <= 512) return run_norm<T, 512, 1, MODE>(a);
    if (n <= 1024) return run_norm<T, 512, 2, MODE>(a);
    if (n <= 2048) return run_norm<T, 1024, 2, MODE>(a);
    if (n <= 4096) return run_norm<T, 1024, 4, MODE>(a);
    return run_norm<T, 1024, 0, MODE>(a);
}

template <typename T> hipError_t pick_mode(const NormArgs &a)
{
    if (!a.q) return pick_norm<T, MODE_NORM>(a);
    return a.weight ? pick_norm<T, MODE_NORM_MX>(a) : pick_norm<T, MODE_QUANT>(a);
}

// ---- dequantise ----
// 16 bytes of output a lane, whose block's scale is one exponent: bound by memory (8192 x
// 4096 to bf16 18 us, 102 MB at 5.7 TB/s).  A product with a power of two is exact, so the
// store's rounding is the only one.
template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t *q, const uint8_t *scales,
                                                         T *y, int64_t rows, int64_t C,
                                                         uint32_t chunks)
{
    constexpr int N = Chunk<T>::N;
    const int64_t width = (C + kMxBlock - 1) / kMxBlock * kMxBlock;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * chunks;
         i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / chunks, c = (i - row * chunks) * N;
        uint32_t w[N / 4];
        __builtin_memcpy(w, __builtin_assume_aligned(q + row * width + c, N), N);
        const uint32_t byte = scales[row * (width / kMxBlock) + c / kMxBlock];
        // 2^(byte - 127); byte 0 is the subnormal 2^-127, 255 is NaN
        const float s = byte == 0     ? bits_f32(0x00400000u)
                        : byte == 255 ? bits_f32(0x7fc00000u)
                                      : bits_f32(byte << 23);
        float v[N];
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            v[4 * k] = __builtin_amdgcn_cvt_f32_fp8((int)w[k], 0) * s;
            v[4 * k + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[k], 1) * s;
            v[4 * k + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[k], 2) * s;
            v[4 * k + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[k], 3) * s;
        }
        Chunk<T>::store(y + row * C + c, (int)min((int64_t)N, C - c), v);
    }
}

// ---- backward ----
struct NormBackwardKernelArgs {
    const void *h, *dy, *dh;
    const float *weight;
    void *dx;
    float *part;            // [gridDim.x][C] or null
    int64_t rows, C;
    float eps;
};

// Waves a SIMD that the registers of `values` values a lane leave room for (h, dy, the sums
// of dw, and what is computed from them).
constexpr int backward_waves(int lanes, int values)
{
    return values <= 8 ? (lanes > 64 ? 5 : 6) : values <= 16 ? 4 : 2;
}

// Rows go round the grid; a lane keeps its columns' sums of dy n.  The groups
// of a workgroup add theirs in order through LDS.  One pass: h and dy stay in registers
// between a row's two sums (which go over the lanes together) and its dx.  Bound by memory:
// 262144 x 128 bf16 48 us, 65536 x 2048 186 us (805 MB at 4.3 TB/s; 360 us with 64 lanes of four
// chunks a row, two waves a SIMD), 16384 x 4096 107 us, float32 32768 x 1000 87 us.
template <typename T, int G, int R>
__global__ void __launch_bounds__(G > 256 ? G : 256, backward_waves(G, Chunk<T>::N *R))
    norm_backward_kernel(NormBackwardKernelArgs a)
{
    constexpr int N = Chunk<T>::N;
    constexpr int kRows = G > 256 ? 1 : 256 / G;
    __shared__ float parts[2][32];
    __shared__ float sums[kRows > 1 ? 256 * R * N : 1];
    const int lane = threadIdx.x % G, grp = threadIdx.x / G;
    float dw[R][N];
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) dw[j][i] = 0.f;

    int turn = 0;
    for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows;
         base += (int64_t)gridDim.x * kRows, turn ^= 1) {
        const int64_t row = base + grp;
        const bool live = row < a.rows;
        const int64_t at = live ? row * a.C : 0;
        float h[R][N], dy[R][N];
        float s = 0.f, p = 0.f;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t c = ((int64_t)j * G + lane) * N;
            const int n = live ? (int)min((int64_t)N, max((int64_t)0, a.C - c)) : 0;
            Chunk<T>::load((const T *)a.h + at + c, n, h[j]);
            Chunk<T>::load((const T *)a.dy + at + c, n, dy[j]);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t c = ((int64_t)j * G + lane) * N;
            const int n = (int)min((int64_t)N, max((int64_t)0, a.C - c));
            float w[N];
            Chunk<float>::load(a.weight + c, n, *(float(*)[4])w);
            if constexpr (N == 8)
                Chunk<float>::load(a.weight + c + 4, n - 4, *(float(*)[4])(w + 4));
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s = fmaf(h[j][i], h[j][i], s);
                p = fmaf(h[j][i], dy[j][i] * w[i], p);
            }
        }
        row_sums<G>(s, p, parts[turn]);
        const float rstd = rsqrtf(s / (float)a.C + a.eps);
        const float k = p * rstd * rstd / (float)a.C;   // mean(g n) * rstd
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t c = ((int64_t)j * G + lane) * N;
            const int n = live ? (int)min((int64_t)N, max((int64_t)0, a.C - c)) : 0;
            if (n <= 0) continue;
            float w[N], o[N];
            Chunk<float>::load(a.weight + c, n, *(float(*)[4])w);
            if constexpr (N == 8)
                Chunk<float>::load(a.weight + c + 4, n - 4, *(float(*)[4])(w + 4));
            if (a.dh) Chunk<T>::load((const T *)a.dh + at + c, n, o);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = rstd * (dy[j][i] * w[i] - h[j][i] * k);
                o[i] = a.dh ? o[i] + d : d;
                dw[j][i] = fmaf(dy[j][i], h[j][i] * rstd, dw[j][i]);
            }
            Chunk<T>::store((T *)a.dx + at + c, n, o);
        }
    }
    if (!a.part) return;
    float *out = a.part + (int64_t)blockIdx.x * a.C;
    if constexpr (kRows > 1) {
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) sums[grp * (G * R * N) + (j * G + lane) * N + i] = dw[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < G * R * N && c < a.C; c += 256) {
            float t = 0.f;
#pragma unroll
            for (int g = 0; g < kRows; ++g) t += sums[g * (G * R * N) + c];
            out[c] = t;
        }
    } else {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t c = ((int64_t)j * G + lane) * N;
            const int n = (int)min((int64_t)N, max((int64_t)0, a.C - c));
            Chunk<float>::store(out + c, n, *(float(*)[4])dw[j]);
            if constexpr (N == 8) Chunk<float>::store(out + c + 4, n - 4, *(float(*)[4])(dw[j] + 4));
        }
    }
}

// Rows too wide for registers: the two sums of each row first (stat [rows][2]:
// rstd and mean(g n) rstd), then dx and the columns' sums by column chunks.
template <typename T>
__global__ void __launch_bounds__(1024) norm_backward_stats(NormBackwardKernelArgs a, float *stat)
{
    constexpr int N = Chunk<T>::N;
    __shared__ float part[16];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = row * a.C;
        float s = 0.f, p = 0.f;
        for (int64_t c = (int64_t)threadIdx.x * N; c < a.C; c += 1024 * N) {
            const int n = (int)min((int64_t)N, a.C - c);
            float h[N], dy[N];
            Chunk<T>::load((const T *)a.h + at + c, n, h);
            Chunk<T>::load((const T *)a.dy + at + c, n, dy);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s = fmaf(h[i], h[i], s);
                p = fmaf(h[i], i < n ? dy[i] * a.weight[c + i] : 0.f, p);
            }
        }
        const float rstd = rsqrtf(row_sum<1024>(s, part) / (float)a.C + a.eps);
        const float k = row_sum<1024>(p, part) * rstd * rstd / (float)a.C;
        if (threadIdx.x == 0) {
            stat[2 * row] = rstd;
            stat[2 * row + 1] = k;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) norm_backward_columns(NormBackwardKernelArgs a,
                                                             const float *stat, int64_t per)
{
    constexpr int N = Chunk<T>::N;
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N;
    const int n = (int)min((int64_t)N, a.C - c);
    if (n <= 0) return;
    float dw[N], w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) dw[i] = 0.f, w[i] = i < n ? a.weight[c + i] : 0.f;
    const int64_t end = min(a.rows, ((int64_t)blockIdx.y + 1) * per);
    for (int64_t row = (int64_t)blockIdx.y * per; row < end; ++row) {
        const float rstd = stat[2 * row], k = stat[2 * row + 1];
        const int64_t at = row * a.C + c;
        float h[N], dy[N], o[N];
        Chunk<T>::load((const T *)a.h + at, n, h);
        Chunk<T>::load((const T *)a.dy + at, n, dy);
        if (a.dh) Chunk<T>::load((const T *)a.dh + at, n, o);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = rstd * (dy[i] * w[i] - h[i] * k);
            o[i] = a.dh ? o[i] + d : d;
            dw[i] = fmaf(dy[i], h[i] * rstd, dw[i]);
        }
        Chunk<T>::store((T *)a.dx + at, n, o);
    }
    if (a.part) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) a.part[(int64_t)blockIdx.y * a.C + c + i] = dw[i];
    }
}

// Chunks of a row that stay in the backward kernel's registers, at most (a lane of 1024
// threads has 128 of them).
constexpr int64_t wide_chunks(int per) { return per == 8 ? 2048 : 4096; }
// Lanes and chunks a lane of the backward kernel for rows of n chunks.
struct BackwardShape {
    int lanes, chunks;
    int threads() const { return lanes > 256 ? lanes : 256; }
};
BackwardShape backward_shape(int64_t n)
{
    if (n <= 64) return {n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : 64, 1};
    if (n <= 128) return {64, 2};
    if (n <= 256) return {256, 1};
    if (n <= 1024) return {256, n <= 512 ? 2 : 4};
    return {1024, n <= 2048 ? 2 : 4};
}

int64_t backward_parts(int64_t rows, int64_t C, int dtype)
{
    const int per = dtype == DTYPE_BF16 ? 8 : 4;
    const int64_t n = (C + per - 1) / per;
    if (n > wide_chunks(per)) return rows < 64 ? rows : 64;
    // As many workgroups as the 256 compute units hold at a time, each of the same count of
    // rows: with half as many again the last ones ran alone (262144 x 128 bf16: 61 us with 2048,
    // 48 us with 1536).
    const BackwardShape s = backward_shape(n);
    const int64_t in_block = s.threads() / s.lanes, blocks = (rows + in_block - 1) / in_block;
    return std::min<int64_t>(
        blocks, 256 * (backward_waves(s.lanes, per * s.chunks) * 4 / (s.threads() / 64)));
}

template <typename T, int G, int R>
hipError_t run_backward(const NormBackwardArgs &a, uint32_t blocks)
{
    const NormBackwardKernelArgs k{a.h, a.dy, a.dh, a.weight, a.dx,
                                   a.dweight ? a.ws : nullptr, a.rows, a.C, a.eps};
    norm_backward_kernel<T, G, R><<<dim3(blocks), dim3(G > 256 ? G : 256), 0, a.stream>>>(k);
    return hipGetLastError();
}

template <typename T> hipError_t pick_backward(const NormBackwardArgs &a)
{
    const int64_t n = (a.C + Chunk<T>::N - 1) / Chunk<T>::N;
    const int64_t parts = backward_parts(a.rows, a.C, a.dtype);
    const uint32_t b = (uint32_t)parts;
    hipError_t e;
    if (n > wide_chunks(Chunk<T>::N)) {
        float *stat = a.ws + (a.dweight ? parts * a.C : 0);
        const NormBackwardKernelArgs k{a.h, a.dy, a.dh, a.weight, a.dx,
                                       a.dweight ? a.ws : nullptr, a.rows, a.C, a.eps};
        norm_backward_stats<T><<<dim3((uint32_t)std::min<int64_t>(a.rows, 1 << 16)), dim3(1024), 0,
                                 a.stream>>>(k, stat);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        const int64_t per = (a.rows + parts - 1) / parts;
        norm_backward_columns<T><<<dim3((uint32_t)((n + 255) / 256), b), dim3(256), 0, a.stream>>>(
            k, stat, per);
        e = hipGetLastError();
    } else if (n <= 8) e = run_backward<T, 8, 1>(a, b);
    else if (n <= 16) e = run_backward<T, 16, 1>(a, b);
    else if (n <= 32) e = run_backward<T, 32, 1>(a, b);
    else if (n <= 64) e = run_backward<T, 64, 1>(a, b);
    else if (n <= 128) e = run_backward<T, 64, 2>(a, b);
    else if (n <= 256) e = run_backward<T, 256, 1>(a, b);
    else if (n <= 512) e = run_backward<T, 256, 2>(a, b);
    else if (n <= 1024) e = run_backward<T, 256, 4>(a, b);
    else if (n <= 2048) e = run_backward<T, 1024, 2>(a, b);
    else if constexpr (Chunk<T>::N == 4) e = run_backward<T, 1024, 4>(a, b);
    else e = hipErrorInvalidValue;
    if (e != hipSuccess || !a.dweight) return e;
    return launch_column_sum(a.ws, parts, a.C, a.dweight, a.stream);
}

// Column sums of partial rows, to `out` and those from `half` on to `out2`: COLS columns a workgroup,
// 1024 / COLS rows at a time, each thread's rows in order and then their sums in order.  2048 x
// 128: 5-7 us, a launch and its loads' latency; 2048 x 688 11 us, 8 with 8 columns.
template <int COLS>
__global__ void __launch_bounds__(1024) column_sum_kernel(const float *part, int64_t n, int64_t C,
                                                          float *out, int64_t half, float *out2)
{
    constexpr int kDown = 1024 / COLS;
    __shared__ float s[kDown][COLS + 1];
    const int cx = threadIdx.x % COLS, ry = threadIdx.x / COLS;
    const int64_t c = (int64_t)blockIdx.x * COLS + cx;
    float t = 0.f;
    for (int64_t r = ry; r < n; r += 8 * kDown) {      // eight loads in flight
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            v[u] = c < C && r + u * kDown < n ? part[(r + u * kDown) * C + c] : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) t += v[u];
    }
    s[ry][cx] = t;
    __syncthreads();
    if constexpr (kDown > 32) {         // 32 sums of a column again
        constexpr int kFold = kDown / 32;
        float u = 0.f;
#pragma unroll
        for (int r = 0; r < kFold; ++r) u += ry < 32 ? s[ry * kFold + r][cx] : 0.f;
        __syncthreads();
        if (ry < 32) s[ry][cx] = u;
        __syncthreads();
    }
    if (ry == 0 && c < C) {
        float u = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) u += s[r][cx];
        float *to = c < half ? out : out2;
        if (to) to[c < half ? c : c - half] = u;
    }
}

// 16 bytes a thread round the grid; the first workgroup takes what lies before and after them, in
// 2-byte words.
__global__ void __launch_bounds__(256) zero_kernel(char *p, uint64_t bytes)
{
    const uint64_t before = min(bytes, (16 - (uint64_t)(uintptr_t)p % 16) % 16);
    const uint64_t wide = (bytes - before) / 16;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < wide;
         i += (uint64_t)gridDim.x * 256)
        *(u32x4 *)(p + before + 16 * i) = (u32x4){0, 0, 0, 0};
    if (blockIdx.x > 0 || threadIdx.x >= 8) return;
    const uint64_t at = 2 * threadIdx.x, end = before + 16 * wide;
    if (at < before) *(uint16_t *)(p + at) = 0;
    if (end + at < bytes) *(uint16_t *)(p + end + at) = 0;
}

}  // namespace

hipError_t launch_zero(void *p, uint64_t bytes, hipStream_t stream)
{
    const uint64_t blocks = std::min<uint64_t>(bytes / 4096 + 1, kMaxBlocks);
    zero_kernel<<<dim3((uint32_t)blocks), dim3(256), 0, stream>>>((char *)p, bytes);
    return hipGetLastError();
}

hipError_t launch_norm(const NormArgs &a)
{
    return a.dtype == DTYPE_BF16 ? pick_mode<__bf16>(a) : pick_mode<float>(a);
}

uint64_t norm_backward_floats(int64_t rows, int64_t C, int dtype, bool dweight)
{
    const int per = dtype == DTYPE_BF16 ? 8 : 4;
    // the partial sums, and two numbers a row where rows are too wide for registers
    return (dweight ? (uint64_t)backward_parts(rows, C, dtype) * C : 0) +
           ((C + per - 1) / per > wide_chunks(per) ? 2 * (uint64_t)rows : 0);
}

hipError_t launch_norm_backward(const NormBackwardArgs &a)
{
    return a.dtype == DTYPE_BF16 ? pick_backward<__bf16>(a) : pick_backward<float>(a);
}

hipError_t launch_dequantize(const void *q, const uint8_t *scales, void *y, int64_t rows,
                             int64_t C, int dtype, hipStream_t stream)
{
    const int n = dtype == DTYPE_BF16 ? 8 : 4;
    const int64_t chunks = (C + n - 1) / n;
    const dim3 grid((uint32_t)std::min<int64_t>((rows * chunks + 255) / 256, kMaxBlocks));
    if (dtype == DTYPE_BF16)
        dequantize_kernel<<<grid, dim3(256), 0, stream>>>((const uint8_t *)q, scales, (__bf16 *)y,
                                                          rows, C, (uint32_t)chunks);
    else
        dequantize_kernel<<<grid, dim3(256), 0, stream>>>((const uint8_t *)q, scales, (float *)y,
                                                          rows, C, (uint32_t)chunks);
    return hipGetLastError();
}

hipError_t launch_column_sum(const float *part, int64_t n, int64_t C, float *out,
                             hipStream_t stream)
{
    column_sum_kernel<32><<<dim3((uint32_t)((C + 31) / 32)), dim3(1024), 0, stream>>>(
        part, n, C, out, C, nullptr);
    return hipGetLastError();
}

hipError_t launch_column_sums(const float *part, int64_t n, int64_t C, float *first, float *second,
                              hipStream_t stream)
{
    // Many rows of few columns: narrower workgroups, more of them.
    if (n >= 512 && C <= 1024)
        column_sum_kernel<8><<<dim3((uint32_t)((2 * C + 7) / 8)), dim3(1024), 0, stream>>>(
            part, n, 2 * C, first, C, second);
    else
        column_sum_kernel<32><<<dim3((uint32_t)((2 * C + 31) / 32)), dim3(1024), 0, stream>>>(
            part, n, 2 * C, first, C, second);
    return hipGetLastError();
}

}  // namespace whtmix
