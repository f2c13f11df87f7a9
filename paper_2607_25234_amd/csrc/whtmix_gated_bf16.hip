// The other forms of bf16 products on the tile kernel: two products of the same rows whose sums
// meet in the epilogue, one whose columns are of two outputs, one whose k is of two operands.
// One row, 1 x 4096 x 2 x 12288: 38 us for the weights' 201 MB (5.3 TB/s) and 5 for the sum of the
// parts of k; a kernel of multiply-adds on the weights as they stream took 48 in all.
#include "whtmix_pack.h"

namespace whtmix {

uint64_t gemm_bf16_bytes(const GemmArgs &g, Form form)
{
    const int64_t columns = form == GATED ? 2 * g.N : g.N;
    const uint64_t parts = tile_part_bytes(g.M, columns, g.K, kStepBytes / 2, form != PLAIN);
    if (form == TWO_K) return parts;
    if (form == HALVES)
        return parts + side(g.a, K_STRIDED, g.M, g.K, g.lda).bytes() +
               side(g.b, K_STRIDED, g.N, g.K, g.ldb).bytes();
    return parts + side(g.a, K_CONTIGUOUS, g.M, g.K, g.lda).bytes() +
           side(g.b, K_STRIDED, g.N, g.K, g.ldb).bytes() +
           side(g.b2, K_STRIDED, g.N, g.K, g.ldb2).bytes();
}

hipError_t gemm_bf16(GemmArgs g, Form form, void *ws, hipStream_t stream)
{
    char *w = (char *)ws;
    if (form == TWO_K) {
        g.a_rows = g.M, g.b_rows = g.N, g.a_k = g.b_k = g.K;
        return run_tiles<2, false, __bf16, K_CONTIGUOUS, K_CONTIGUOUS, TWO_K>(g, (float *)w, stream);
    }
    const Layout la = form == HALVES ? K_STRIDED : K_CONTIGUOUS;
    const PackJob a = place(g.a, g.lda, g.a_rows, g.a_k, la, side(g.a, la, g.M, g.K, g.lda), w);
    const PackJob b = place(g.b, g.ldb, g.b_rows, g.b_k, K_STRIDED,
                            side(g.b, K_STRIDED, g.N, g.K, g.ldb), w);
    PackJob c{};
    if (form == GATED)      // of b's width too, whichever of them is packed
        c = place(g.b2, g.ldb2, g.b_rows, g.b_k, K_STRIDED, side(g.b2, K_STRIDED, g.N, g.K, g.ldb2), w);
    const hipError_t e = launch_pack(a, b, c, stream);
    if (e != hipSuccess) return e;
    if (form == HALVES)
        return run_tiles<2, false, __bf16, K_STRIDED, K_STRIDED, HALVES>(g, (float *)w, stream);
    return run_tiles<2, false, __bf16, K_CONTIGUOUS, K_STRIDED, GATED>(g, (float *)w, stream);
}

}  // namespace whtmix
