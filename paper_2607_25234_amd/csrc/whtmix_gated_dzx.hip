// dzg = dy zu act'(zg), dzu = dy act(zg), their columns' sums and dx = dzg wg^T + dzu wu^T in one
// pass over dy, zg and zu, for bf16 and inputs of up to 128 columns: there the products are few
// and everything is bound by memory.
//
// A workgroup takes 128 rows through all N in steps of 64: it forms dzg and dzu in registers,
// writes them (rounded to bf16, what the matrix cores read) to memory for the weights' gradients,
// where those are asked for, and to LDS for its own product, and multiplies with both weights'
// step, which copies bring to LDS meanwhile.  The next step's dy, zg and zu are on their way
// during the products.  One set of buffers, 66 KiB, so that two workgroups share a compute unit:
// one's products and barriers pass under the other's loads.
//
// Where rows are not whole cache lines, every `apart`-th one starts at the same place in a line
// (2, 4 or 8, N being a multiple of 8).  A workgroup takes every apart-th row; its steps start that
// many columns before the rows, and dz's rows lie so far apart that they start alike: every access is
// to a whole line.  262144 x 128 x 344 297 us (309 from each row's start on, 351 with dz's rows at
// whole lines), x 336 270 (291, 320), x 352 256 (273, 271); the weights' gradients read such rows
// no slower (127 and 129 us); without dz (no weights' gradients) 160 us for dx, 188 with the sums.
// Of 516 MiB of operands the counters have 982 MiB read from each row's start on and 603 so (scaled
// by what they give for a copy), and 422 written: 3.6 TB/s.  The waves wait for 58% of their time,
// vector instructions take 27%, products 8%.
#include "whtmix_gemm_tile.h"
#include "whtmix_row.h"

namespace whtmix {
namespace {

constexpr int kRows = 128, kCols = 128, kN = 64;   // rows, columns of dx, n of a step

struct GatedDzxArgs {
    const __bf16 *dy, *zg, *zu;
    const void *wg, *wu;
    __bf16 *dz;             // [M] rows `pitch` apart, dzu `width` behind dzg; or null
    float *part;            // [groups * apart][2][N] sums of the unrounded values, or null
    __bf16 *dx;             // [M][K]
    int64_t M, N, K, width, pitch;
    uint32_t groups;        // of kRows * apart rows
    int apart;
};

// Sum of the wave's lanes with the same number within eight, in all of them.
__device__ __forceinline__ float rows_of_eight(float v)
{
    v += lane_move<0x128>(v);       // eight lanes on, in rows of sixteen
    const auto r = __builtin_amdgcn_permlane16_swap(f32_bits(v), f32_bits(v), false, false);
    v = bits_f32((uint32_t)r[0]) + bits_f32((uint32_t)r[1]);
    const auto h = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
    return bits_f32((uint32_t)h[0]) + bits_f32((uint32_t)h[1]);
}

// An activation a kernel: with all of them in one the registers do not hold a step.
template <int ACT>
__global__ void __launch_bounds__(256, 2) gated_dzx_kernel(GatedDzxArgs d)
{
    constexpr int kTileBytes = kRows * kStepBytes;      // of each of four: dzg, dzu, wg, wu
    constexpr int kSums = 2 * 4 * kN * 4;
    __shared__ __attribute__((aligned(1024))) char lds[4 * kTileBytes + kSums];
    float(*sums)[4][kN] = (float(*)[4][kN])(lds + 4 * kTileBytes);      // [half][wave][column]
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // A group's workgroups are on one XCD, whose L2 has the lines that neighbouring rows share.
    const uint32_t nth = blockIdx.x / 8, group = blockIdx.x % 8 + 8 * (nth / d.apart);
    if (group >= d.groups) return;
    const int first = (int)(nth % d.apart);
    const int64_t m0 = (int64_t)group * kRows * d.apart + first;
    const int rows = (int)min((int64_t)kRows, (d.M - m0 + d.apart - 1) / d.apart);  // maybe none
    const int shift = (int)(first * d.N % kN);      // columns of the first step before the rows'
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    const uint32_t lds_wave = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds +
                              (uint32_t)__builtin_amdgcn_readfirstlane(wave) * 1024;
    const int steps = (int)((d.N + shift + kN - 1) / kN);
    // Whether column c of step t is one of the rows'.
    auto column = [&](int t, int c) __attribute__((always_inline)) {
        const int n = t * kN - shift + c;
        return n >= 0 && n < d.N;
    };

    // Four chunks of 8 n (N is a multiple of 8): rows threadIdx.x / 8 + 32 i, the same columns.
    const int row0 = threadIdx.x >> 3, chunk = threadIdx.x & 7;
    u32x4 dy[4], zg[4], zu[4];
    const int64_t row = m0 + row0 * d.apart;
    const int64_t at0 = row * d.N + chunk * 8 - shift;
    const int64_t to0 = row * d.pitch + chunk * 8 - shift;
    auto load = [&](int t) __attribute__((always_inline)) {
        const bool in = column(t, chunk * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool live = in && row0 + 32 * i < rows;
            const int64_t at = at0 + (int64_t)(32 * i * d.apart) * d.N + t * kN;
            dy[i] = live ? *(const u32x4 *)(d.dy + at) : (u32x4){0, 0, 0, 0};
            zg[i] = live ? *(const u32x4 *)(d.zg + at) : (u32x4){0, 0, 0, 0};
            zu[i] = live ? *(const u32x4 *)(d.zu + at) : (u32x4){0, 0, 0, 0};
        }
    };

    // Where chunk i of the thread is in the tile of dzg (and a tile on in dzu's).
    auto place = [&](int i) __attribute__((always_inline)) {
        const int row = row0 + 32 * i;
        return lds + row * kStepBytes +
               Operand<2, K_CONTIGUOUS, kRows, 1>::swizzle(row, chunk) * 16;
    };

    using Weights = Operand<2, K_CONTIGUOUS, kCols, 4>;
    Weights ob[2];
    ob[0].init(d.wg, d.N, d.K, 0, -shift, d.N);
    ob[1].init(d.wu, d.N, d.K, 0, -shift, d.N);
    auto copy = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t to = lds_wave + (2 + h) * kTileBytes;
            if (t > 0 && t + 1 < steps) {
#pragma unroll
                for (int i = 0; i < Weights::kCopies; ++i) ob[h].copy_one(to, i);
            } else {            // zeros before and behind the columns
#pragma unroll
                for (int i = 0; i < Weights::kCopies; ++i) {
                    int outer, at;
                    Weights::place(i, outer, at);
                    copy16(column(t, at * 8) ? ob[h].base + ob[h].off[i] : (const char *)kZero16,
                           to + i * 4096);
                }
            }
            ob[h].copied();
        }
    };

    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    load(0);
    copy(0);
    for (int t = 0; t < steps; ++t) {
        float sg[8], su[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) sg[k] = su[k] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x4 og, ou;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float vg[2], vu[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    auto half = [&](uint32_t w) { return bits_f32(e ? w & 0xffff0000u : w << 16); };
                    float a, da;
                    act_both<ACT>(half(zg[i][k]), a, da);
                    const float y = half(dy[i][k]);
                    vg[e] = y * half(zu[i][k]) * da;
                    vu[e] = y * a;
                    sg[2 * k + e] += vg[e];
                    su[2 * k + e] += vu[e];
                }
                og[k] = pack_bf16(vg[0], vg[1]);
                ou[k] = pack_bf16(vu[0], vu[1]);
            }
            *(u32x4 *)place(i) = og;
            *(u32x4 *)(place(i) + kTileBytes) = ou;
            __builtin_amdgcn_sched_barrier(0);      // chunk by chunk: the registers' sake
        }
        if (d.part) {
            // the wave's eight rows of lanes, then its columns
#pragma unroll
            for (int k = 0; k < 8; ++k) sg[k] = rows_of_eight(sg[k]), su[k] = rows_of_eight(su[k]);
            if (lane < 8) {
                *(f32x4 *)&sums[0][wave][lane * 8] = (f32x4){sg[0], sg[1], sg[2], sg[3]};
                *(f32x4 *)&sums[0][wave][lane * 8 + 4] = (f32x4){sg[4], sg[5], sg[6], sg[7]};
                *(f32x4 *)&sums[1][wave][lane * 8] = (f32x4){su[0], su[1], su[2], su[3]};
                *(f32x4 *)&sums[1][wave][lane * 8 + 4] = (f32x4){su[4], su[5], su[6], su[7]};
            }
        }
        wait_copies<0>();       // step t of the weights (and what was stored a step ago)
        __syncthreads();
        const bool in = column(t, chunk * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d.dz && in && row0 + 32 * i < rows) {
                __bf16 *to = d.dz + to0 + (int64_t)(32 * i * d.apart) * d.pitch + t * kN;
                *(u32x4 *)to = *(const u32x4 *)place(i);
                *(u32x4 *)(to + d.width) = *(const u32x4 *)(place(i) + kTileBytes);
            }
        __builtin_amdgcn_sched_barrier(0);
        if (t + 1 < steps) load(t + 1);
        __builtin_amdgcn_sched_barrier(0);
        if (d.part && threadIdx.x < 2 * kN) {
            const int h = threadIdx.x / kN, c = threadIdx.x % kN;
            const float *p = &sums[h][0][c];
            if (column(t, c))
                d.part[(((int64_t)group * d.apart + first) * 2 + h) * d.N + t * kN - shift + c] =
                    ((p[0] + p[kN]) + p[2 * kN]) + p[3 * kN];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char *z = lds + h * kTileBytes, *w = lds + (2 + h) * kTileBytes;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                bf16x8 fa[2], fb[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    fa[i] = fragment16<K_CONTIGUOUS, kRows>(z, wm + 32 * i, kk);
                    fb[i] = fragment16<K_CONTIGUOUS, kCols>(w, wn + 32 * i, kk);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i],
                                                                            acc[i][j], 0, 0, 0);
                if (kk & 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();        // all have read this step's tiles
        if (t + 1 < steps) copy(t + 1);
    }
    static_assert(4 * kEpilogueFloats * 4 <= sizeof(lds), "the epilogue's rows");
    // The sums to dx, 32 rows of the wave at a time through LDS.
    float *out = (float *)lds + wave * kEpilogueFloats;
    float *w = out + (lane & 31) * kEpilogueStride + (lane >> 5) * 4;
    const float *p = out + (lane >> 3) * kEpilogueStride + (lane & 7) * 8;
    const int64_t n = wn + (lane & 7) * 8;
    const int cnt = (int)max((int64_t)0, min((int64_t)8, d.K - n));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        wave_lds_fence();
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                *(f32x4 *)(w + 32 * j + 8 * r) = (f32x4){acc[i][j][4 * r], acc[i][j][4 * r + 1],
                                                         acc[i][j][4 * r + 2], acc[i][j][4 * r + 3]};
        wave_lds_fence();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float v[8];
            *(f32x4 *)v = *(const f32x4 *)(p + 8 * r * kEpilogueStride);
            *(f32x4 *)(v + 4) = *(const f32x4 *)(p + 8 * r * kEpilogueStride + 4);
            const int m = wm + 32 * i + 8 * r + (lane >> 3);
            if (m < rows) store8(d.dx + (m0 + (int64_t)m * d.apart) * d.K + n, cnt, v);
        }
    }
}

// The rows from one that starts at a cache line's start to the next: N is a multiple of 8.
int rows_apart(int64_t N)
{
    int p = 1;
    while (p * N % kN != 0) p *= 2;
    return p;
}

uint32_t groups_of(int64_t M, int64_t N)
{
    const int64_t rows = (int64_t)kRows * rows_apart(N);
    return (uint32_t)((M + rows - 1) / rows);
}

}  // namespace

int64_t gated_dzx_parts(const GatedBackwardArgs &a)
{
    return (int64_t)groups_of(a.M, a.N) * rows_apart(a.N);
}

// Narrow inputs, whole 16-byte chunks (32-bit offsets of the weights'), and rows enough for the
// device, more of them where a workgroup's rows take long.  The whole backward pass, so and with
// dz and dx apart: 262144 x 128 x 256 235 and 289 us, x 512 440 and 536; 131072 x 64 x 344 195 and
// 197 (with dz's rows at whole lines); at the fewest rows 32768 x 128 x 256 50 and 51, 49152 x 128 x 344
// 101 and 106, x 520 138 and 161.
bool gated_dzx_takes(const GatedBackwardArgs &a)
{
    auto aligned = [](const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    return a.dtype == DTYPE_BF16 && a.dx && a.K <= kCols && a.N % 8 == 0 && a.N >= kN &&
           a.N <= 1024 && a.M >= (a.N <= 256 ? 256 : 384) * kRows && aligned(a.dy) &&
           aligned(a.zg) && aligned(a.zu) && aligned(a.wg) && aligned(a.wu);
}

int64_t gated_dzx_pitch(int64_t N, int64_t width) { return 2 * width + N % kN; }

hipError_t launch_gated_dzx(const GatedBackwardArgs &a, int64_t width, void *dz, float *part)
{
    const int apart = rows_apart(a.N);
    const uint32_t groups = groups_of(a.M, a.N);
    const GatedDzxArgs d{(const __bf16 *)a.dy, (const __bf16 *)a.zg, (const __bf16 *)a.zu, a.wg, a.wu,
                         (__bf16 *)dz, part, (__bf16 *)a.dx, a.M, a.N, a.K, width,
                         gated_dzx_pitch(a.N, width), groups, apart};
    const auto kernel = a.act == ACT_RELU        ? gated_dzx_kernel<ACT_RELU>
                        : a.act == ACT_GELU      ? gated_dzx_kernel<ACT_GELU>
                        : a.act == ACT_GELU_TANH ? gated_dzx_kernel<ACT_GELU_TANH>
                        : a.act == ACT_SILU      ? gated_dzx_kernel<ACT_SILU>
                                                 : gated_dzx_kernel<ACT_NONE>;
    kernel<<<dim3((groups + 7) / 8 * 8 * (uint32_t)apart), dim3(256), 0, a.stream>>>(d);
    return hipGetLastError();
}

}  // namespace whtmix
