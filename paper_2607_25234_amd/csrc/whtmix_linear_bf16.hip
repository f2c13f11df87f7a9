// Products of bf16 operands: the tile kernel, and the packing of operands whose rows do not
// start at 16 bytes.
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

// Both operands in one launch: the first `a.blocks` workgroups take a, the others b.
__global__ void __launch_bounds__(256) pack_kernel(PackJob a, PackJob b)
{
    const bool first = blockIdx.x < a.blocks;
    const PackJob &j = first ? a : b;
    const int64_t per = j.width / 8, total = j.outer * per;
    for (int64_t i = (int64_t)(first ? blockIdx.x : blockIdx.x - a.blocks) * 256 + threadIdx.x;
         i < total; i += (int64_t)j.blocks * 256) {
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

}  // namespace

uint64_t gemm_bf16_bytes(const GemmArgs &g, Layout la, Layout lb)
{
    return side(g.a, la, g.M, g.K, g.lda).bytes() + side(g.b, lb, g.N, g.K, g.ldb).bytes() +
           tile_part_bytes(g.M, g.N, g.K, kStepBytes / 2);
}

hipError_t gemm_bf16(GemmArgs g, Layout la, Layout lb, void *ws, hipStream_t stream)
{
    char *w = (char *)ws;
    const PackJob a = place(g.a, g.lda, g.a_rows, g.a_k, la, side(g.a, la, g.M, g.K, g.lda), w);
    const PackJob b = place(g.b, g.ldb, g.b_rows, g.b_k, lb, side(g.b, lb, g.N, g.K, g.ldb), w);
    if (a.blocks + b.blocks) {
        pack_kernel<<<dim3(a.blocks + b.blocks), dim3(256), 0, stream>>>(a, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (la == K_CONTIGUOUS && lb == K_STRIDED)
        return run_tiles<2, false, __bf16, K_CONTIGUOUS, K_STRIDED>(g, (float *)w, stream);
    if (la == K_CONTIGUOUS)
        return run_tiles<2, false, __bf16, K_CONTIGUOUS, K_CONTIGUOUS>(g, (float *)w, stream);
    return run_tiles<2, false, __bf16, K_STRIDED, K_STRIDED>(g, (float *)w, stream);
}

}  // namespace whtmix
