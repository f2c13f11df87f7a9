// Products of block-scaled 8-bit rows.
//
// The scaled matrix instructions (twice the rate of bf16) line the products of 64 k up
// with the largest and drop what lies some 2^-15 below it: 2e-6 of the sum of magnitudes,
// root mean square, measured on normal values.  A rounding to bf16 or 8 bits hides that but
// where a sum cancels.  A float32 output, and sums of few k, are formed of bf16
// products instead (bf16 holds each value), whose sums keep float32's accuracy:
// with K <= 512 a product is bound by memory either way.
#include "whtmix_gemm_tile.h"

namespace whtmix {

constexpr int64_t kExactK = 512;

uint64_t gemm_mx_bytes(const GemmArgs &g) { return tile_part_bytes(g.M, g.N, g.K, kStepBytes); }

template <bool EXACT, typename T> static hipError_t run(const GemmArgs &g, void *ws, hipStream_t s)
{
    return run_tiles<1, EXACT, T, K_CONTIGUOUS, K_CONTIGUOUS>(g, (float *)ws, s);
}

hipError_t gemm_mx(GemmArgs g, int dtype, void *ws, hipStream_t stream)
{
    g.a_rows = g.M, g.b_rows = g.N, g.a_k = g.b_k = g.K;
    const bool exact = g.K <= kExactK || (g.y && dtype == DTYPE_F32);
    if (dtype == DTYPE_BF16)
        return exact ? run<true, __bf16>(g, ws, stream) : run<false, __bf16>(g, ws, stream);
    return exact ? run<true, float>(g, ws, stream) : run<false, float>(g, ws, stream);
}

}  // namespace whtmix
