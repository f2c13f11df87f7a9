// dz = dy act'(z), its columns' sums and dx = dz w^T in one pass over dy and z, for bf16 and
// inputs of up to 128 columns: there the products are few and everything is bound by memory.
//
// Apart, dz is written by one kernel and read again by dx's: 262144 x 128 x 512 took 192 and 81 us.
// Here a workgroup takes 128 rows through all N in steps of 64: it forms dz in registers, writes
// it (rounded to bf16, what the matrix cores read) to memory for dw's product and to LDS for its own, and multiplies with w's step, which copies
// bring to LDS meanwhile.  The next step's dy and z are on their way during the products.
// Together 197-232 us: 872 MB at 3.8-4.4 TB/s, about what dz alone took.
#include "whtmix_gemm_tile.h"

namespace whtmix {
namespace {

constexpr int kRows = 128, kCols = 128, kN = 64;   // rows, columns of dx, n of a step

struct DzxArgs {
    const __bf16 *dy, *z;
    __bf16 *dz;
    float *part;            // [workgroups][N] sums of the unrounded dz, or null
    int64_t M, N;
    int act;
};

__global__ void __launch_bounds__(256) dzx_kernel(DzxArgs d, GemmArgs g)
{
    constexpr int kTileBytes = kRows * kStepBytes;      // of either operand
    constexpr int kSums = 2 * 4 * kN * 4;
    __shared__ __attribute__((aligned(1024))) char lds[4 * kTileBytes + kSums];
    float(*sums)[4][kN] = (float(*)[4][kN])(lds + 4 * kTileBytes);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t m0 = (int64_t)blockIdx.x * kRows;
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    const uint32_t lds_wave = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds +
                              (uint32_t)__builtin_amdgcn_readfirstlane(wave) * 1024;
    const int steps = (int)((d.N + kN - 1) / kN);

    // Four chunks of 8 n: rows threadIdx.x / 8 + 32 i, the same columns.
    const int row0 = threadIdx.x >> 3, chunk = threadIdx.x & 7;
    u32x4 dy[4], z[4];
    const int64_t at0 = (m0 + row0) * d.N + chunk * 8;
    auto load = [&](int t) __attribute__((always_inline)) {
        const bool in = t * kN + chunk * 8 < d.N;       // whole chunks: N is a multiple of 8
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool live = in && m0 + row0 + 32 * i < d.M;
            const int64_t at = at0 + (int64_t)(32 * i) * d.N + t * kN;
            dy[i] = live ? *(const u32x4 *)(d.dy + at) : (u32x4){0, 0, 0, 0};
            z[i] = live ? *(const u32x4 *)(d.z + at) : (u32x4){0, 0, 0, 0};
        }
    };

    Operand<2, K_CONTIGUOUS, kCols, 4> ob;
    ob.init(g.b, g.ldb, g.N, 0, 0, d.N);
    auto copy = [&](int t) __attribute__((always_inline)) {
        const uint32_t to = lds_wave + (2 + (t & 1)) * kTileBytes;
        if (t + 1 < steps) {
#pragma unroll
            for (int i = 0; i < Operand<2, K_CONTIGUOUS, kCols, 4>::kCopies; ++i) ob.copy_one(to, i);
            ob.copied();
        } else {
            ob.copy_last(to, (int64_t)t * kN);
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
    with_act(d.act, [&](auto tag) __attribute__((always_inline)) {
        constexpr int ACT = decltype(tag)::value;
        for (int t = 0; t < steps; ++t) {
            char *here = lds + (t & 1) * kTileBytes;
            float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            u32x4 out[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float d0 = bits_f32(dy[i][k] << 16) * act_grad<ACT>(bits_f32(z[i][k] << 16));
                    const float d1 = bits_f32(dy[i][k] & 0xffff0000u) *
                                     act_grad<ACT>(bits_f32(z[i][k] & 0xffff0000u));
                    s[2 * k] += d0;
                    s[2 * k + 1] += d1;
                    out[i][k] = pack_bf16(d0, d1);
                }
                const int row = row0 + 32 * i;
                *(u32x4 *)(here + row * kStepBytes +
                           Operand<2, K_CONTIGUOUS, kRows, 1>::swizzle(row, chunk) * 16) = out[i];
            }
            if (d.part) {
                // the wave's eight rows of lanes, then its columns
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    s[k] += __shfl_xor(s[k], 8);
                    s[k] += __shfl_xor(s[k], 16);
                    s[k] += __shfl_xor(s[k], 32);
                }
                if (lane < 8) {
                    *(f32x4 *)&sums[t & 1][wave][lane * 8] = (f32x4){s[0], s[1], s[2], s[3]};
                    *(f32x4 *)&sums[t & 1][wave][lane * 8 + 4] = (f32x4){s[4], s[5], s[6], s[7]};
                }
            }
            wait_copies<0>();       // step t of w (and what was stored a step ago)
            __syncthreads();
            const bool in = t * kN + chunk * 8 < d.N;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (in && m0 + row0 + 32 * i < d.M)
                    *(u32x4 *)(d.dz + at0 + (int64_t)(32 * i) * d.N + t * kN) = out[i];
            if (t + 1 < steps) {
                load(t + 1);
                copy(t + 1);
            }
            if (d.part && threadIdx.x < kN && t * kN + (int)threadIdx.x < d.N) {
                const float *p = &sums[t & 1][0][threadIdx.x];
                d.part[(int64_t)blockIdx.x * d.N + t * kN + threadIdx.x] =
                    ((p[0] + p[kN]) + p[2 * kN]) + p[3 * kN];
            }
            const char *w = lds + (2 + (t & 1)) * kTileBytes;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                bf16x8 fa[2], fb[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    fa[i] = fragment16<K_CONTIGUOUS, kRows>(here, wm + 32 * i, kk);
                    fb[i] = fragment16<K_CONTIGUOUS, kCols>(w, wn + 32 * i, kk);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i], acc[i][j],
                                                                            0, 0, 0);
            }
        }
    });
    __syncthreads();
    static_assert(4 * kEpilogueFloats * 4 <= sizeof(lds), "the epilogue's rows");
    finish_wave<__bf16>(g, (float *)lds + wave * kEpilogueFloats, m0 + wm, wn, 0, acc);
}

}  // namespace

int64_t dzx_parts(int64_t M) { return (M + kRows - 1) / kRows; }

// Narrow inputs, whole 16-byte chunks (32-bit offsets of w's), and rows enough for the device, more
// of them where a workgroup's rows take long.  dx and dbias, together and apart:
//   32768 x 128 x 64 12 and 21 us, x 128 15 and 25, x 256 23 and 26, x 512 37 and 35;
//   49152 x 128 x 512 49 and 51, x 1024 82 and 84; 40960 x 128 x 1024 78 and 74;
//   65536 x 128 x 512 54 and 61, x 2048 240 and 229; 262144 x 128 x 512 195 and 240, and with dw
//   131072 x 128 x 1024 262 and 295, x 2048 588 and 590, x 4096 1105 and 1068;
//   4096 x 128 x 512 28 and 20.
bool dzx_takes(const LinearBackwardArgs &a)
{
    auto aligned = [](const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    return a.dtype == DTYPE_BF16 && a.act != ACT_NONE && a.dx && a.K <= kCols && a.N % 8 == 0 &&
           a.N >= kN && a.N <= 1024 && a.M >= (a.N <= 256 ? 256 : 384) * kRows &&
           aligned(a.dy) && aligned(a.z) && aligned(a.w);
}

hipError_t launch_dzx(const LinearBackwardArgs &a, void *dz, float *part)
{
    GemmArgs g{};
    g.b = a.w, g.ldb = a.N;
    g.M = a.M, g.N = a.K, g.K = a.N, g.y = a.dx;
    const DzxArgs d{(const __bf16 *)a.dy, (const __bf16 *)a.z, (__bf16 *)dz, part, a.M, a.N, a.act};
    dzx_kernel<<<dim3((uint32_t)dzx_parts(a.M)), dim3(256), 0, a.stream>>>(d, g);
    return hipGetLastError();
}

}  // namespace whtmix
