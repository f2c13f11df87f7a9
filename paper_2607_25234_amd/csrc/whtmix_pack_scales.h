// The packing of block scales whose rows are not whole dwords (device code of the file that
// includes it), and the rule for products of 8-bit values as bf16.
#pragma once

#include "whtmix_gemm_tile.h"

namespace whtmix {
namespace {

constexpr int64_t kExactK = 512;    // sums of up to this many k are formed of bf16 products

// Rows of scales to whole dwords, 1 past the end: the tile kernel copies dwords.  Up to three
// operands' in one launch.
struct ScalesJob {
    const uint8_t *src;
    uint32_t *dst;
    int64_t rows;
    int width;
    uint32_t blocks;
};

__global__ void __launch_bounds__(256) pack_scales_kernel(ScalesJob a, ScalesJob b, ScalesJob c)
{
    const bool first = blockIdx.x < a.blocks, last = blockIdx.x >= a.blocks + b.blocks;
    const ScalesJob &j = first ? a : last ? c : b;
    const uint32_t before = first ? 0 : last ? a.blocks + b.blocks : a.blocks;
    const int dwords = (j.width + 3) / 4;
    for (int64_t i = (int64_t)(blockIdx.x - before) * 256 + threadIdx.x; i < j.rows * dwords;
         i += (int64_t)j.blocks * 256) {
        const int64_t row = i / dwords;
        const int at = (int)(i - row * dwords) * 4;
        uint32_t v = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v |= (at + k < j.width ? (uint32_t)j.src[row * j.width + at + k] : 127u) << (8 * k);
        j.dst[i] = v;
    }
}

bool whole_dwords(const uint8_t *p, int64_t width)
{
    return width % 4 == 0 && reinterpret_cast<uintptr_t>(p) % 4 == 0;
}

uint64_t packed_bytes(const uint8_t *p, int64_t rows, int64_t width)
{
    return whole_dwords(p, width) ? 0 : (uint64_t)(rows * ((width + 3) / 4 * 4) + 255) / 256 * 256;
}

ScalesJob place_scales(const uint8_t *&p, int64_t &ld, int64_t rows, int64_t width,
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

hipError_t launch_pack_scales(const ScalesJob &a, const ScalesJob &b, const ScalesJob &c,
                              hipStream_t stream)
{
    const uint32_t blocks = a.blocks + b.blocks + c.blocks;
    if (blocks == 0) return hipSuccess;
    pack_scales_kernel<<<dim3(blocks), dim3(256), 0, stream>>>(a, b, c);
    return hipGetLastError();
}

}  // namespace
}  // namespace whtmix
