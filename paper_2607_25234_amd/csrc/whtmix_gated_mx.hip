// The gated product of block-scaled 8-bit rows: both products in one tile, as of bf16.  The same
// rule as for a single product says which are formed of the scaled matrix instructions.  17 x 4096 x 2 x
// 16384: 27 us for the weights' 138 MB (5.1 TB/s) and 5 for the sum of the parts.
#include "whtmix_pack_scales.h"

namespace whtmix {

uint64_t gated_mx_gemm_bytes(const GemmArgs &g)
{
    return packed_bytes(g.as, g.M, g.K / kMxBlock) + packed_bytes(g.bs, g.N, g.K / kMxBlock) +
           packed_bytes(g.bs2, g.N, g.K / kMxBlock) + tile_part_bytes(g.M, 2 * g.N, g.K, kStepBytes);
}

template <bool EXACT, typename T> static hipError_t run(const GemmArgs &g, void *ws, hipStream_t s)
{
    return run_tiles<1, EXACT, T, K_CONTIGUOUS, K_CONTIGUOUS, GATED>(g, (float *)ws, s);
}

hipError_t gated_mx_gemm(GemmArgs g, int dtype, void *ws, hipStream_t stream)
{
    g.a_rows = g.M, g.b_rows = g.N, g.a_k = g.b_k = g.K;
    char *w = (char *)ws;
    const int64_t width = g.K / kMxBlock;
    const ScalesJob a = place_scales(g.as, g.as_ld, g.M, width, w);
    const ScalesJob b = place_scales(g.bs, g.bs_ld, g.N, width, w);
    const ScalesJob c = place_scales(g.bs2, g.bs2_ld, g.N, width, w);
    const hipError_t e = launch_pack_scales(a, b, c, stream);
    if (e != hipSuccess) return e;
    const bool exact = g.K <= kExactK || (g.y && dtype == DTYPE_F32);
    if (dtype == DTYPE_BF16)
        return exact ? run<true, __bf16>(g, w, stream) : run<false, __bf16>(g, w, stream);
    return exact ? run<true, float>(g, w, stream) : run<false, float>(g, w, stream);
}

}  // namespace whtmix
