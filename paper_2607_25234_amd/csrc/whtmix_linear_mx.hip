// Products of block-scaled 8-bit rows.
//
// The scaled matrix instructions (twice the rate of bf16) line the products of 64 k up
// with the largest and drop what lies some 2^-15 below it.  Measured error over the sum of
// magnitudes, root mean square: 1e-6 at K = 256 and 7e-7 at 512 for normal values, 1e-5 for values
// spread over 2^6, where float32 sums are off by 5e-9.  Of few k that is more than the float32
// sum's own bound (up to 14 times it at K = 192 and 256), and no rounding to bf16 or 8 bits
// hides it where a sum cancels.  So sums of up to 512 k, and float32 outputs of any K, are formed of
// bf16 products instead (bf16 holds each value, to multiples of 2^-133), whose sums keep
// float32's accuracy.  32768 x K x 2048, bf16 products first: K = 160 56 and 41 us, 256 54 and
// 38, 512 84 and 53; 17 x 512 x 4096 8.9 and 8.5, 17 x 8192 x 4096 14.3 and 13.3 us.
#include "whtmix_gemm_tile.h"

namespace whtmix {

constexpr int64_t kExactK = 512;

// Rows of scales to whole dwords, 1 past the end: the tile kernel copies dwords.  Both
// operands' in one launch.
struct ScalesJob {
    const uint8_t *src;
    uint32_t *dst;
    int64_t rows;
    int width;
    uint32_t blocks;
};

__global__ void __launch_bounds__(256) pack_scales_kernel(ScalesJob a, ScalesJob b)
{
    const bool first = blockIdx.x < a.blocks;
    const ScalesJob &j = first ? a : b;
    const int dwords = (j.width + 3) / 4;
    for (int64_t i = (int64_t)(first ? blockIdx.x : blockIdx.x - a.blocks) * 256 + threadIdx.x;
         i < j.rows * dwords; i += (int64_t)j.blocks * 256) {
        const int64_t row = i / dwords;
        const int at = (int)(i - row * dwords) * 4;
        uint32_t v = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v |= (at + k < j.width ? (uint32_t)j.src[row * j.width + at + k] : 127u) << (8 * k);
        j.dst[i] = v;
    }
}

static bool whole_dwords(const uint8_t *p, int64_t width)
{
    return width % 4 == 0 && reinterpret_cast<uintptr_t>(p) % 4 == 0;
}

static uint64_t packed_bytes(const uint8_t *p, int64_t rows, int64_t width)
{
    return whole_dwords(p, width) ? 0 : (uint64_t)(rows * ((width + 3) / 4 * 4) + 255) / 256 * 256;
}

static ScalesJob place_scales(const uint8_t *&p, int64_t &ld, int64_t rows, int64_t width,
                              char *&ws)
{
    ld = width;
    const uint64_t bytes = packed_bytes(p, rows, width);
    if (!bytes) return ScalesJob{};
    const int64_t n = rows * ((width + 3) / 4), blocks = (n + 255) / 256;
    const ScalesJob j{p, (uint32_t *)ws, rows, (int)width,
                      (uint32_t)(blocks < 65536 ? blocks : 65536)};
    p = (const uint8_t *)ws;
    ws += bytes;
    ld = (width + 3) / 4 * 4;
    return j;
}

uint64_t gemm_mx_bytes(const GemmArgs &g)
{
    return packed_bytes(g.as, g.M, g.K / kMxBlock) + packed_bytes(g.bs, g.N, g.K / kMxBlock) +
           tile_part_bytes(g.M, g.N, g.K, kStepBytes);
}

template <bool EXACT, typename T> static hipError_t run(const GemmArgs &g, void *ws, hipStream_t s)
{
    return run_tiles<1, EXACT, T, K_CONTIGUOUS, K_CONTIGUOUS>(g, (float *)ws, s);
}

hipError_t gemm_mx(GemmArgs g, int dtype, void *ws, hipStream_t stream)
{
    g.a_rows = g.M, g.b_rows = g.N, g.a_k = g.b_k = g.K;
    char *w = (char *)ws;
    const ScalesJob a = place_scales(g.as, g.as_ld, g.M, g.K / kMxBlock, w);
    const ScalesJob b = place_scales(g.bs, g.bs_ld, g.N, g.K / kMxBlock, w);
    if (a.blocks + b.blocks) {
        pack_scales_kernel<<<dim3(a.blocks + b.blocks), dim3(256), 0, stream>>>(a, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    ws = w;
    const bool exact = g.K <= kExactK || (g.y && dtype == DTYPE_F32);
    if (dtype == DTYPE_BF16)
        return exact ? run<true, __bf16>(g, ws, stream) : run<false, __bf16>(g, ws, stream);
    return exact ? run<true, float>(g, ws, stream) : run<false, float>(g, ws, stream);
}

}  // namespace whtmix
