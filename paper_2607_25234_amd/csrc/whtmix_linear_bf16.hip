// Products of bf16 operands on the tile kernel.
#include "whtmix_pack.h"

namespace whtmix {

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
    const hipError_t e = launch_pack(a, b, PackJob{}, stream);
    if (e != hipSuccess) return e;
    if (la == K_CONTIGUOUS && lb == K_STRIDED)
        return run_tiles<2, false, __bf16, K_CONTIGUOUS, K_STRIDED>(g, (float *)w, stream);
    if (la == K_CONTIGUOUS)
        return run_tiles<2, false, __bf16, K_CONTIGUOUS, K_CONTIGUOUS>(g, (float *)w, stream);
    return run_tiles<2, false, __bf16, K_STRIDED, K_STRIDED>(g, (float *)w, stream);
}

}  // namespace whtmix
