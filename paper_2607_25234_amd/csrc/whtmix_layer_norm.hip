// Layer norm with the residual's addition, and its backward pass.
//
//   t = x + residual          (float32; h = t rounded to the stream's type)
//   mu = mean(t),  v = mean((t - mu)^2),  n = (t - mu) / sqrt(v + eps),  y = n w + b
//   from h:  g = dy w,  dx = dh + (g - mean(g) - n mean(g n)) / sqrt(v + eps)
//            dw = sum over rows of dy n,   db = sum over rows of dy
//
// Bound by memory: a row is read once into the registers of G lanes (R chunks of 16 bytes each)
// and all that is formed of it leaves from there.  The mean comes first and the squares are of
// the distances from it, because mean(t^2) - mu^2 cancels where the mean is large beside the
// spread.  The float32 mean is itself off by some 2^-24 |mu|, so distances are taken from a pivot p
// near it, and their own mean d, summed with their squares, gives both (v = mean((t - p)^2) - d^2,
// mu = p + d, kept as two floats).  Rows of bf16 lie on a coarse grid, of which every t - p would
// drop the same low bits of a p that has all 24: a bias that d would take for its own.  p is
// therefore rounded to 2^-12 of the spread, which makes such distances and their sums exact
// (error of mu in units of 2^-24 of the spread, root mean square, 512 rows of 4096 values in bf16 of mean 0
// and deviation 1: 0.006, 0.28 about the mean with all its bits; of mean 1: 0.005 and 0.31).
// Sums are float32 in a fixed order: a lane's over its own values, then a fixed tree.
//
// 8192 x 4096 bf16 to 8 bits 50 us (4.7 TB/s of 235 MB), 262144 x 128 bf16 45 us forward and 48
// backward (5.9 and 5.6 TB/s, in part out of the caches), 5003 x 1111 float32 14 and 17 us; one row of
// 4096 2.8 us, the latency of its loads and of two sums.  Rows that the registers do not hold are read
// once for each sum and once more, in part out of the caches: 2000 x 40000 bf16 121 and 218 us.
#include "whtmix_row.h"

#include <algorithm>

namespace whtmix {
namespace {

struct LayerNormKernelArgs {
    const void *x, *residual;
    const float *weight, *bias;
    void *y, *h, *q;
    uint8_t *scales;
    int64_t rows, C, ldx;
    float eps;
};

// What distances are taken from, by a row's mean m and the mean of its squares: m to 2^-12 of the
// spread or down to half of that (the next power of two).  Of a mean beyond 16 spreads all bits are
// kept: values are near it there, and their distances exact; and where squares overflow or
// cancel to nothing.
__device__ __forceinline__ float row_pivot(float m, float squares)
{
    const float q = fmaxf(fmaf(-m, m, squares), 0.f);
    const uint32_t spread = ((f32_bits(q) >> 23) + 127) >> 1;       // its exponent
    const float on = bits_f32((spread + 11) << 23 | 0x400000u);     // 1.5 * 2^11 of it
    return m * m <= 256.f * q && q < bits_f32(0x7f800000u) ? (m + on) - on : m;
}

// What a row's sums give: of the distances from its pivot p their sum t0 and their squares' t1.
// The mean p + d is kept as hi + lo: t - hi - lo rounds once where the mean is moderate, and
// still holds where it is far larger than the spread.
struct RowStats {
    float hi, lo, rstd;
};
__device__ __forceinline__ RowStats row_stats(float p, float t0, float t1, float C, float eps)
{
    const float d = t0 / C, v = fmaxf(fmaf(-d, d, t1 / C), 0.f) + eps;
    RowStats r;
    r.hi = p + d;
    r.lo = (p - r.hi) + d;
    // The hardware's reciprocal root to its last bit, by a step of Newton's.
    const float e = rsqrtf(v);
    const float c = fmaf(0.5f * e, fmaf(-v * e, e, 1.f), e);
    r.rstd = c == c ? c : e;        // (v = 0, or Inf)
    return r;
}

// Workgroups that a unit holds at a time, by the waves a SIMD that their registers leave room for.
constexpr int forward_waves(int chunks) { return chunks == 1 ? 6 : 4; }
constexpr int threads_of(int G) { return G > 256 ? G : 256; }

// One row on G lanes, R chunks a lane; with R = 0 (rows wider than the registers hold) the row
// is read three times.  With one chunk a lane rows go round the grid and the next one is on its
// way while this one is formed (8192 x 4096 to 8 bits 50 us; 62 with a workgroup a row).  Values for
// the 8-bit form keep the parts that roundings on the
// way would leave out: off by a few 2^-24, one value in 10^5 moves to the next of the 8-bit ones.
template <typename T, int G, int R, bool MX>
__global__ void __launch_bounds__(threads_of(G), forward_waves(R))
    layer_norm_kernel(LayerNormKernelArgs a)
{
    constexpr int N = Chunk<T>::N;
    constexpr int kRows = threads_of(G) / G;
    __shared__ float part[2][48];
    const int lane = threadIdx.x % G;
    const int64_t width = MX ? (a.C + kMxBlock - 1) / kMxBlock * kMxBlock : a.C;
    const float C = (float)a.C, inv = 1.f / C;
    auto count = [&](int64_t c) { return (int)min((int64_t)N, max((int64_t)0, a.C - c)); };
    auto vectors = [&](int64_t c, float (&w)[N], float (&b)[N]) {
        const int n = count(c);
        load_floats(a.weight + (n ? c : 0), n, w);
        load_floats(a.bias ? a.bias + (n ? c : 0) : a.weight, a.bias ? n : 0, b);
    };
    // The values (zeros past the row's end) into their sum and squares.
    auto total = [&](const float (&v)[N], float (&s)[2]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[0] += v[i];
            s[1] = fmaf(v[i], v[i], s[1]);
        }
    };
    // The distances from the pivot, of the elements there are, likewise.
    auto spread = [&](int n, const float (&v)[N], float p, float (&t)[2]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = i < n ? v[i] - p : 0.f;
            t[0] += d;
            t[1] = fmaf(d, d, t[1]);
        }
    };
    auto emit = [&](int64_t row, int64_t c, float (&v)[N], const float (&w)[N],
                    const float (&b)[N], const RowStats &r) {
        const int n = count(c);
        if (a.h && n > 0) store_row<T>((T *)a.h + row * a.C + c, n, v);
        if constexpr (MX) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                // the distance and its product with rstd, each with what its rounding left out
                const float d = v[i] - r.hi, z = d - v[i], p = d * r.rstd;
                const float dl = ((v[i] - (d - z)) - (r.hi + z)) - r.lo;
                const float pl = fmaf(dl, r.rstd, fmaf(d, r.rstd, -p));
                v[i] = i < n ? fmaf(p, w[i], fmaf(pl, w[i], b[i])) : 0.f;
            }
            store_mx<T>(v, (uint8_t *)a.q + row * width, a.scales + row * (width / kMxBlock), c);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = fmaf((v[i] - r.hi - r.lo) * r.rstd, w[i], b[i]);
            if (n > 0) store_row<T>((T *)a.y + row * a.C + c, n, v);
        }
    };

    if constexpr (R == 1) {
        const int64_t c = (int64_t)lane * N;
        const int n = count(c);
        RawChunk<T> x, r;
        auto load = [&](int64_t row) {
            const bool live = row < a.rows && n > 0;
            x.load((const T *)a.x + (live ? row * a.ldx + c : 0), live ? n : 0);
            if (a.residual)
                r.load((const T *)a.residual + (live ? row * a.C + c : 0), live ? n : 0);
        };
        int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
        const int64_t step = (int64_t)gridDim.x * kRows;
        load(row);
        float w[N], b[N];
        vectors(c, w, b);
        // Rows past the end go through the exchanges with zeros and store nothing.
        for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows; base += step, row += step) {
            float v[N], s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = x[i];
                if (a.residual) v[i] += r[i];
            }
            if (base + step < a.rows) load(row + step);
            total(v, s);
            row_sums<G>(s, part[0]);
            const float p = row_pivot(s[0] * inv, s[1] * inv);
            spread(n, v, p, t);
            row_sums<G>(t, part[1]);
            const RowStats st = row_stats(p, t[0], t[1], C, a.eps);
            if (row < a.rows && c < width) emit(row, c, v, w, b, st);
        }
    } else {
        // A workgroup a row.
        for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
            const T *x = (const T *)a.x + row * a.ldx;
            const T *r = a.residual ? (const T *)a.residual + row * a.C : nullptr;
            auto load = [&](int64_t c, float (&v)[N]) {
                const int n = count(c);
                load_row<T>(x + (n ? c : 0), n, v);
                if (r) {
                    float e[N];
                    load_row<T>(r + (n ? c : 0), n, e);
#pragma unroll
                    for (int i = 0; i < N; ++i) v[i] += e[i];
                }
            };
            float s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};
            if constexpr (R > 0) {
                float v[R][N];
#pragma unroll
                for (int j = 0; j < R; ++j) load(((int64_t)j * G + lane) * N, v[j]);
#pragma unroll
                for (int j = 0; j < R; ++j) total(v[j], s);
                row_sums<G>(s, part[0]);
                const float p = row_pivot(s[0] * inv, s[1] * inv);
#pragma unroll
                for (int j = 0; j < R; ++j)
                    spread(count(((int64_t)j * G + lane) * N), v[j], p, t);
                row_sums<G>(t, part[1]);
                const RowStats st = row_stats(p, t[0], t[1], C, a.eps);
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    const int64_t c = ((int64_t)j * G + lane) * N;
                    if (c >= width) continue;
                    float w[N], b[N];
                    vectors(c, w, b);
                    emit(row, c, v[j], w, b, st);
                }
            } else {
                for (int64_t c = (int64_t)lane * N; c < a.C; c += (int64_t)G * N) {
                    float v[N];
                    load(c, v);
                    total(v, s);
                }
                row_sums<G>(s, part[0]);
                const float p = row_pivot(s[0] * inv, s[1] * inv);
                for (int64_t c = (int64_t)lane * N; c < a.C; c += (int64_t)G * N) {
                    float v[N];
                    load(c, v);
                    spread(count(c), v, p, t);
                }
                row_sums<G>(t, part[1]);
                const RowStats st = row_stats(p, t[0], t[1], C, a.eps);
                // A block's lanes are in the loop together: `width` is a multiple of 32.
                for (int64_t c = (int64_t)lane * N; c < width; c += (int64_t)G * N) {
                    float v[N], w[N], b[N];
                    load(c, v);
                    vectors(c, w, b);
                    emit(row, c, v, w, b, st);
                }
            }
        }
    }
}

template <typename T, int G, int R, bool MX> hipError_t run_forward(const LayerNormArgs &a)
{
    constexpr int kRows = threads_of(G) / G;
    const LayerNormKernelArgs k{a.x, a.residual, a.weight, a.bias, a.y, a.h, a.q, a.scales,
                                a.rows, a.C, a.ldx, a.eps};
    const int64_t at_once = 256 * (forward_waves(R) * 4 / (threads_of(G) / 64));
    const int64_t blocks =
        std::min<int64_t>((a.rows + kRows - 1) / kRows, R == 1 ? at_once : kMaxBlocks);
    layer_norm_kernel<T, G, R, MX>
        <<<dim3((uint32_t)blocks), dim3(threads_of(G)), 0, a.stream>>>(k);
    return hipGetLastError();
}

// Chunks of a row -> lanes and chunks a lane.  384 lanes for rows that leave a third of 512 idle: 8192
// x 2560 bf16 28 us, 31 on 512, to 8 bits 34 and 38, 5003 x 1111 float32 14 and 16; one row 2.9 on either.
template <typename T, bool MX> hipError_t pick_forward(const LayerNormArgs &a)
{
    const int64_t width = MX ? mx_width(a.C) : a.C;
    const int64_t n = (width + Chunk<T>::N - 1) / Chunk<T>::N;
    if (n <= 8) return run_forward<T, 8, 1, MX>(a);
    if (n <= 16) return run_forward<T, 16, 1, MX>(a);
    if (n <= 32) return run_forward<T, 32, 1, MX>(a);
    if (n <= 64) return run_forward<T, 64, 1, MX>(a);
    if (n <= 128) return run_forward<T, 128, 1, MX>(a);
    if (n <= 256) return run_forward<T, 256, 1, MX>(a);
    if (n <= 384) return run_forward<T, 384, 1, MX>(a);
    if (n <= 512) return run_forward<T, 512, 1, MX>(a);
    if (n <= 1024) return run_forward<T, 512, 2, MX>(a);
    if (n <= 2048) return run_forward<T, 1024, 2, MX>(a);
    if (n <= 4096) return run_forward<T, 1024, 4, MX>(a);
    return run_forward<T, 1024, 0, MX>(a);
}

// ---- backward ----
struct LayerNormBackwardKernelArgs {
    const void *h, *dy, *dh;
    const float *weight;
    void *dx;
    float *part;            // [gridDim.x][2][C]: the sums of dy n, then of dy; or null
    float *dweight, *dbias; // with part null: [C] or null
    int64_t rows, C;
    float eps;
};

// Waves a SIMD that the registers of `values` values a lane leave room for (h, dy, weight, both
// vectors' sums, and what is computed from them); a workgroup of 1024 takes four.
constexpr int backward_waves(int lanes, int values)
{
    return lanes == 1024 ? 4 : values <= 4 ? 6 : values <= 8 ? 4 : 2;
}

// Rows go round the grid; a lane keeps its columns' sums of dy n and of dy.  The groups of a
// workgroup add theirs in order through LDS.
template <typename T, int G, int R>
__global__ void __launch_bounds__(G > 256 ? G : 256, backward_waves(G, Chunk<T>::N *R))
    layer_norm_backward_kernel(LayerNormBackwardKernelArgs a)
{
    constexpr int N = Chunk<T>::N;
    constexpr int kRows = G > 256 ? 1 : 256 / G;
    __shared__ float parts[2][48];
    __shared__ float sums[kRows > 1 ? 256 * R * N : 1];
    const int lane = threadIdx.x % G, grp = threadIdx.x / G;
    const float inv = 1.f / (float)a.C;
    float dw[R][N], db[R][N], w0[N];
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) dw[j][i] = db[j][i] = 0.f;
    auto count = [&](int j) {
        return (int)min((int64_t)N, max((int64_t)0, a.C - ((int64_t)j * G + lane) * N));
    };
    auto weights = [&](int j, float (&w)[N]) {
        const int n = count(j);
        load_floats(a.weight + (n ? ((int64_t)j * G + lane) * N : 0), n, w);
    };
    if constexpr (R == 1) weights(0, w0);

    for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows;
         base += (int64_t)gridDim.x * kRows) {
        const int64_t row = base + grp;
        const bool live = row < a.rows;
        const int64_t at = live ? row * a.C : 0;
        float h[R][N], dy[R][N];
        float s[3] = {0.f, 0.f, 0.f};   // of h, of g, of h's squares
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int n = live ? count(j) : 0;
            const int64_t c = at + (n ? ((int64_t)j * G + lane) * N : 0);
            load_row<T>((const T *)a.h + c, n, h[j]);
            load_row<T>((const T *)a.dy + c, n, dy[j]);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            float w[N];
            if constexpr (R > 1) weights(j, w);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s[0] += h[j][i];
                s[1] = fmaf(dy[j][i], R == 1 ? w0[i] : w[i], s[1]);
                s[2] = fmaf(h[j][i], h[j][i], s[2]);
            }
        }
        row_sums<G>(s, parts[0]);
        const float pivot = row_pivot(s[0] * inv, s[2] * inv);
        float t[3] = {0.f, 0.f, 0.f};   // of the distances d, their squares, g d
#pragma unroll
        for (int j = 0; j < R; ++j) {
            float w[N];
            if constexpr (R > 1) weights(j, w);
            const int n = count(j);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = i < n ? h[j][i] - pivot : 0.f;
                h[j][i] = d;
                t[0] += d;
                t[1] = fmaf(d, d, t[1]);
                t[2] = fmaf(d, dy[j][i] * (R == 1 ? w0[i] : w[i]), t[2]);
            }
        }
        row_sums<G>(t, parts[1]);
        const float off = t[0] * inv;
        const float rstd = rsqrtf(fmaxf(fmaf(-off, off, t[1] * inv), 0.f) + a.eps);
        const float gm = s[1] * inv;                            // mean(g)
        const float k = fmaf(-off, s[1], t[2]) * rstd * inv;    // mean(g n)
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int n = live ? count(j) : 0;
            if (n <= 0) continue;
            const int64_t c = at + ((int64_t)j * G + lane) * N;
            float w[N], o[N];
            if constexpr (R > 1) weights(j, w);
            if (a.dh) load_row<T>((const T *)a.dh + c, n, o);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float nn = (h[j][i] - off) * rstd;
                const float d = rstd * (fmaf(dy[j][i], R == 1 ? w0[i] : w[i], -gm) - nn * k);
                o[i] = a.dh ? o[i] + d : d;
                dw[j][i] = fmaf(dy[j][i], nn, dw[j][i]);
                db[j][i] += dy[j][i];
            }
            store_row<T>((T *)a.dx + c, n, o);
        }
    }
    // To this workgroup's partial sums, or where it is the only one to the gradients.
    auto emit = [&](const float (&v)[R][N], float *to) {
        if (!to) return;
        if constexpr (kRows > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < R; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    sums[grp * (G * R * N) + (j * G + lane) * N + i] = v[j][i];
            __syncthreads();
            for (int c = threadIdx.x; c < G * R * N && c < a.C; c += 256) {
                float u = 0.f;
#pragma unroll
                for (int g = 0; g < kRows; ++g) u += sums[g * (G * R * N) + c];
                to[c] = u;
            }
        } else {
#pragma unroll
            for (int j = 0; j < R; ++j)
                store_floats(to + ((int64_t)j * G + lane) * N, count(j), v[j]);
        }
    };
    float *out = a.part ? a.part + (int64_t)blockIdx.x * 2 * a.C : nullptr;
    emit(dw, out ? out : a.dweight);
    emit(db, out ? out + a.C : a.dbias);
}

// Rows too wide for registers: what each row's sums give first (stat: [rows][4] of the pivot, the
// mean's distance from it, 1 / sqrt(v + eps) and mean(g), then [rows] of mean(g n)), then dx and the columns'
// sums by column chunks.
template <typename T>
__global__ void __launch_bounds__(1024) layer_norm_backward_stats(LayerNormBackwardKernelArgs a,
                                                                  float *stat)
{
    constexpr int N = Chunk<T>::N;
    __shared__ float parts[2][48];
    const float inv = 1.f / (float)a.C;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = row * a.C;
        auto each = [&](auto f) {
            for (int64_t c = (int64_t)threadIdx.x * N; c < a.C; c += 1024 * N) {
                const int n = (int)min((int64_t)N, a.C - c);
                float h[N], dy[N], w[N];
                load_row<T>((const T *)a.h + at + c, n, h);
                load_row<T>((const T *)a.dy + at + c, n, dy);
                load_floats(a.weight + c, n, w);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i < n) f(h[i], dy[i] * w[i]);
            }
        };
        float s[3] = {0.f, 0.f, 0.f}, t[3] = {0.f, 0.f, 0.f};
        each([&](float h, float g) {
            s[0] += h;
            s[1] += g;
            s[2] = fmaf(h, h, s[2]);
        });
        row_sums<1024>(s, parts[0]);
        const float pivot = row_pivot(s[0] * inv, s[2] * inv);
        each([&](float h, float g) {
            const float d = h - pivot;
            t[0] += d;
            t[1] = fmaf(d, d, t[1]);
            t[2] = fmaf(d, g, t[2]);
        });
        row_sums<1024>(t, parts[1]);
        const float off = t[0] * inv;
        const float rstd = rsqrtf(fmaxf(fmaf(-off, off, t[1] * inv), 0.f) + a.eps);
        if (threadIdx.x == 0) {
            stat[4 * row] = pivot;
            stat[4 * row + 1] = off;
            stat[4 * row + 2] = rstd;
            stat[4 * row + 3] = s[1] * inv;
            stat[4 * a.rows + row] = fmaf(-off, s[1], t[2]) * rstd * inv;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256)
    layer_norm_backward_columns(LayerNormBackwardKernelArgs a, const float *stat, int64_t per)
{
    constexpr int N = Chunk<T>::N;
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N;
    const int n = (int)min((int64_t)N, a.C - c);
    if (n <= 0) return;
    float dw[N], db[N], w[N];
    load_floats(a.weight + c, n, w);
#pragma unroll
    for (int i = 0; i < N; ++i) dw[i] = db[i] = 0.f;
    const int64_t end = min(a.rows, ((int64_t)blockIdx.y + 1) * per);
    for (int64_t row = (int64_t)blockIdx.y * per; row < end; ++row) {
        const float pivot = stat[4 * row], off = stat[4 * row + 1], rstd = stat[4 * row + 2],
                    gm = stat[4 * row + 3], k = stat[4 * a.rows + row];
        const int64_t at = row * a.C + c;
        float h[N], dy[N], o[N];
        load_row<T>((const T *)a.h + at, n, h);
        load_row<T>((const T *)a.dy + at, n, dy);
        if (a.dh) load_row<T>((const T *)a.dh + at, n, o);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float nn = (h[i] - pivot - off) * rstd;
            const float d = rstd * (fmaf(dy[i], w[i], -gm) - nn * k);
            o[i] = a.dh ? o[i] + d : d;
            dw[i] = fmaf(dy[i], nn, dw[i]);
            db[i] += dy[i];
        }
        store_row<T>((T *)a.dx + at, n, o);
    }
    if (a.part) {
        float *out = a.part + (int64_t)blockIdx.y * 2 * a.C + c;
        store_floats(out, n, dw);
        store_floats(out + a.C, n, db);
    }
}

// Chunks of a row that stay in the backward kernel's registers, at most.
constexpr int64_t wide_chunks(int per) { return per == 8 ? 2048 : 4096; }
constexpr int kWideFloats = 5;          // of a row that does not

struct BackwardShape {
    int lanes, chunks;
    int threads() const { return lanes > 256 ? lanes : 256; }
};
BackwardShape backward_shape(int64_t n)
{
    if (n <= 64) return {n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : 64, 1};
    if (n <= 128) return {128, 1};
    if (n <= 256) return {256, 1};
    if (n <= 512) return {512, 1};
    return {1024, n <= 1024 ? 1 : n <= 2048 ? 2 : 4};
}

int64_t backward_parts(int64_t rows, int64_t C, int dtype)
{
    const int per = dtype == DTYPE_BF16 ? 8 : 4;
    const int64_t n = (C + per - 1) / per;
    if (n > wide_chunks(per)) return std::min<int64_t>(rows, 64);
    // As many workgroups as the 256 compute units hold at a time, each of the same count of rows.
    const BackwardShape s = backward_shape(n);
    const int64_t in_block = s.threads() / s.lanes, blocks = (rows + in_block - 1) / in_block;
    // One workgroup and no launch more: calls of 8 x 1024 bf16 (four) 7 us, 9 to 10 in parts; of 17 x
    // 1024 (nine) 11 in one, 9 to 10 in parts.
    if (blocks <= 4) return 1;
    const int at_once = std::max(1, backward_waves(s.lanes, per * s.chunks) * 4 / (s.threads() / 64));
    return std::min<int64_t>(blocks, 256 * at_once);
}

template <typename T, int G, int R>
hipError_t run_backward(const LayerNormBackwardKernelArgs &k, uint32_t blocks, hipStream_t stream)
{
    layer_norm_backward_kernel<T, G, R><<<dim3(blocks), dim3(G > 256 ? G : 256), 0, stream>>>(k);
    return hipGetLastError();
}

template <typename T> hipError_t backward(const LayerNormBackwardArgs &a)
{
    const int64_t n = (a.C + Chunk<T>::N - 1) / Chunk<T>::N;
    const int64_t parts = backward_parts(a.rows, a.C, a.dtype);
    const bool sums = a.dweight || a.dbias;
    const uint32_t b = (uint32_t)parts;
    const bool wide = n > wide_chunks(Chunk<T>::N), joined = sums && (wide || parts > 1);
    const LayerNormBackwardKernelArgs k{a.h, a.dy, a.dh, a.weight, a.dx, joined ? a.ws : nullptr,
                                        a.dweight, a.dbias, a.rows, a.C, a.eps};
    hipError_t e;
    if (wide) {
        float *stat = a.ws + (sums ? parts * 2 * a.C : 0);
        layer_norm_backward_stats<T><<<dim3((uint32_t)std::min<int64_t>(a.rows, 1 << 16)),
                                       dim3(1024), 0, a.stream>>>(k, stat);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        const int64_t per = (a.rows + parts - 1) / parts;
        layer_norm_backward_columns<T>
            <<<dim3((uint32_t)((n + 255) / 256), b), dim3(256), 0, a.stream>>>(k, stat, per);
        e = hipGetLastError();
    } else if (n <= 8) e = run_backward<T, 8, 1>(k, b, a.stream);
    else if (n <= 16) e = run_backward<T, 16, 1>(k, b, a.stream);
    else if (n <= 32) e = run_backward<T, 32, 1>(k, b, a.stream);
    else if (n <= 64) e = run_backward<T, 64, 1>(k, b, a.stream);
    else if (n <= 128) e = run_backward<T, 128, 1>(k, b, a.stream);
    else if (n <= 256) e = run_backward<T, 256, 1>(k, b, a.stream);
    else if (n <= 512) e = run_backward<T, 512, 1>(k, b, a.stream);
    else if (n <= 1024) e = run_backward<T, 1024, 1>(k, b, a.stream);
    else if (n <= 2048) e = run_backward<T, 1024, 2>(k, b, a.stream);
    else if constexpr (Chunk<T>::N == 4) e = run_backward<T, 1024, 4>(k, b, a.stream);
    else e = hipErrorInvalidValue;
    if (e != hipSuccess || !joined) return e;
    return launch_column_sums(a.ws, parts, a.C, a.dweight, a.dbias, a.stream);
}

}  // namespace

hipError_t launch_layer_norm(const LayerNormArgs &a)
{
    if (a.dtype == DTYPE_BF16)
        return a.q ? pick_forward<__bf16, true>(a) : pick_forward<__bf16, false>(a);
    return a.q ? pick_forward<float, true>(a) : pick_forward<float, false>(a);
}

uint64_t layer_norm_backward_floats(int64_t rows, int64_t C, int dtype, bool sums)
{
    const int per = dtype == DTYPE_BF16 ? 8 : 4;
    const bool wide = (C + per - 1) / per > wide_chunks(per);
    const int64_t parts = backward_parts(rows, C, dtype);
    return (sums && (wide || parts > 1) ? (uint64_t)parts * 2 * C : 0) +
           (wide ? kWideFloats * (uint64_t)rows : 0);
}

hipError_t launch_layer_norm_backward(const LayerNormBackwardArgs &a)
{
    return a.dtype == DTYPE_BF16 ? backward<__bf16>(a) : backward<float>(a);
}

}  // namespace whtmix
