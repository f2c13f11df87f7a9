// The packing of bf16 operands whose rows do not start at 16 bytes (device code of the file that
// includes it).
#pragma once

#include "whtmix_gemm_tile.h"

namespace whtmix {
namespace {

// Rows of `inner` elements, ld apart, to rows of `width` (a multiple of 8) with zeros
// past `inner`; eight elements a thread.
struct PackJob {
    const __bf16 *src;
    __bf16 *dst;
    int64_t outer, inner, ld, width;
    uint32_t blocks;
};

// Up to three operands in one launch: the first `a.blocks` workgroups take a, the next b.
__global__ void __launch_bounds__(256) pack_kernel(PackJob a, PackJob b, PackJob c)
{
    const bool first = blockIdx.x < a.blocks, last = blockIdx.x >= a.blocks + b.blocks;
    const PackJob &j = first ? a : last ? c : b;
    const uint32_t before = first ? 0 : last ? a.blocks + b.blocks : a.blocks;
    const int64_t per = j.width / 8, total = j.outer * per;
    for (int64_t i = (int64_t)(blockIdx.x - before) * 256 + threadIdx.x; i < total;
         i += (int64_t)j.blocks * 256) {
        const int64_t r = i / per, c = (i - r * per) * 8;
        float v[8];
        Chunk<__bf16>::load(j.src + r * j.ld + c, (int)min((int64_t)8, j.inner - c), v);
        Chunk<__bf16>::store(j.dst + r * j.width + c, 8, v);
    }
}

// Copies move 16 aligned bytes, and a tile's offsets are 32 bits.  What the packing costs: 3001 x
// 1001 x 2003 30 us (3000 x 1000 x 2000 21), 16384 x 4095 x 4095 494 (4096s 437), 1 x 4095 x
// 4095 32 (11).
bool needs_packing(const void *p, int64_t inner, int64_t ld)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) != 0 || inner % 8 != 0 || ld % 8 != 0 ||
           ld > (int64_t(1) << 22);
}

struct Side {
    int64_t outer, inner, width;
    bool pack;
    uint64_t bytes() const { return pack ? ((uint64_t)outer * width * 2 + 255) / 256 * 256 : 0; }
};

Side side(const void *p, Layout l, int64_t rows, int64_t k, int64_t ld)
{
    Side s{l == K_CONTIGUOUS ? rows : k, l == K_CONTIGUOUS ? k : rows, 0, false};
    s.width = (s.inner + 7) / 8 * 8;
    s.pack = needs_packing(p, s.inner, ld);
    return s;
}

// Where the tile kernel finds an operand, and the packing that puts it there.
PackJob place(const void *&p, int64_t &ld, int64_t &rows, int64_t &k, Layout l, const Side &s,
              char *&ws)
{
    PackJob j{};
    int64_t width = s.inner;
    if (s.pack) {
        const int64_t blocks = (s.outer * (s.width / 8) + 255) / 256;
        j = {(const __bf16 *)p, (__bf16 *)ws, s.outer, s.inner, ld, s.width,
             (uint32_t)(blocks < 65536 ? blocks : 65536)};
        p = ws;
        ws += s.bytes();
        ld = width = s.width;
    }
    rows = l == K_CONTIGUOUS ? s.outer : width;
    k = l == K_CONTIGUOUS ? width : s.outer;
    return j;
}

// The packing of the operands that need it.
hipError_t launch_pack(const PackJob &a, const PackJob &b, const PackJob &c, hipStream_t stream)
{
    const uint32_t blocks = a.blocks + b.blocks + c.blocks;
    if (blocks == 0) return hipSuccess;
    pack_kernel<<<dim3(blocks), dim3(256), 0, stream>>>(a, b, c);
    return hipGetLastError();
}

}  // namespace
}  // namespace whtmix
