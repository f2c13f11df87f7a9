// The tile kernel of bf16 and block-scaled 8-bit products.
//
// A workgroup forms BM x BN sums.  Each step of 128 bytes of k (64 bf16, 128
// 8-bit values) is copied to LDS without passing registers (16 bytes a lane), two
// buffers deep: the copies of the next step are in flight while the matrix
// instructions run on this one.  LDS takes a wave's copies in lane order, so what
// keeps the fragments' reads free of bank conflicts is which 16 bytes each lane
// fetches: chunks of a row are permuted by the row (K_CONTIGUOUS) or the k
// (K_STRIDED).
//
// Each wave holds 32 WM x 64 sums.  The matrix instructions take the second operand's
// columns as their rows, so that a lane's sums run along the output's row.
//
// Measured:
//   8192 x 8192 x 8192 bf16 1.30-1.33 PFLOP/s, 8 bits 2.3-2.4;
//   16384 x 4096 x 16384 bf16 with gelu 1750-1790 us, 1.23-1.26 PFLOP/s: the matrix cores are
//   70% busy at the 1.5-1.7 GHz that the power limit leaves;
//   8192 x 4096 x 16384 8 bits with MX output 620-690 us, 8192 x 16384 x 4096 540-550 us: 43%
//   and 54% busy at 1.8 GHz, the rest the fragments' LDS reads (the registers, 226 of 256
//   taken, hold one set of them) and the epilogue;
//   16384 x 4096 x 4096 bf16 with gelu and z 495 us, its dx 450 and dw 411;
//   1 x 4096 x 16384 bf16 22 us: the second operand's 134 MB at 6.1 TB/s;
//   17 x 8192 x 4096 8 bits 11 us: 34 MB, the latency of a part's few steps.
#pragma once

#include "whtmix_gemm.h"

namespace whtmix {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// What copies fetch past the end of k.
static __device__ __attribute__((aligned(16))) const uint32_t kZero16[4] = {0, 0, 0, 0};

constexpr int kStepBytes = 128;

// One operand's tile: R rows of output (or k-strided columns), NW waves copying.
template <int EB, Layout L, int R, int NW> struct Operand {
    static constexpr int kStepK = kStepBytes / EB;
    static constexpr int kCopies = R / 8 / NW;          // a wave's copies of a step
    static_assert(R % (8 * NW) == 0, "whole copies");
    static constexpr int kRowChunks = L == K_CONTIGUOUS ? 8 : R * EB / 16;

    const char *base;       // of the tile at the next step to copy (uniform)
    uint32_t off[kCopies];  // of this lane's chunks from there
    int64_t ahead;          // bytes from a step to the next
    int64_t k_end;          // of the operand: chunks from there on are zeros

    static __device__ __forceinline__ int swizzle(int outer, int chunk)
    {
        // A cycle of an LDS read serves 16 lanes: 16 rows of 128 bytes fall on all 64 banks
        // when every second row's chunks are permuted alike.
        if constexpr (L == K_CONTIGUOUS) return chunk ^ ((outer >> 1) & 7);
        else return chunk ^ ((4 * (outer & 3)) & (kRowChunks - 1));
    }
    // The (row or k, chunk) that copy i of this lane fetches.
    static __device__ __forceinline__ void place(int i, int &outer, int &chunk)
    {
        const int c = (i * NW + (int)(threadIdx.x >> 6)) * 64 + (int)(threadIdx.x & 63);
        outer = c / kRowChunks;
        chunk = swizzle(outer, c % kRowChunks);
    }
    // rows: of the operand; every chunk that starts before k_end (K_CONTIGUOUS) or
    // rows (K_STRIDED) is whole.
    __device__ __forceinline__ void init(const void *p, int64_t ld_elements, int64_t rows,
                                         int64_t r0, int64_t k0, int64_t kend)
    {
        const int64_t ld = ld_elements * EB;
        k_end = kend;
        ahead = L == K_CONTIGUOUS ? kStepBytes : kStepK * ld;
        base = (const char *)p + (L == K_CONTIGUOUS ? r0 * ld + k0 * EB : k0 * ld + r0 * EB);
        const uint32_t ld32 = (uint32_t)ld, last = (uint32_t)min((int64_t)R, rows - r0);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            int outer, chunk;
            place(i, outer, chunk);
            if constexpr (L == K_CONTIGUOUS)     // rows past the end repeat the last one
                off[i] = min((uint32_t)outer, last - 1) * ld32 + (uint32_t)chunk * 16;
            else                                 // columns likewise
                off[i] = (uint32_t)outer * ld32 + min((uint32_t)chunk * 16, last * EB - 16);
        }
    }
    // The next step, to the LDS address of this wave's part: copy by copy, then on.
    __device__ __forceinline__ void copy_one(uint32_t lds, int i)
    {
        copy16(base, off[i], lds + i * NW * 1024);
    }
    __device__ __forceinline__ void copied() { base += ahead; }
    // The last step, at k, with zeros from k_end on.
    __device__ __forceinline__ void copy_last(uint32_t lds, int64_t k)
    {
        const int left = (int)min(k_end - k, (int64_t)kStepK);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            int outer, chunk;
            place(i, outer, chunk);
            const int at = L == K_CONTIGUOUS ? chunk * (16 / EB) : outer;
            copy16(at < left ? base + off[i] : (const char *)kZero16, lds + i * NW * 1024);
        }
    }
};

// A 32-row fragment of 16 bf16 of k (step kk of 4).
template <Layout L, int R>
__device__ __forceinline__ bf16x8 fragment16(const char *lds, int row0, int kk)
{
    const int lane = threadIdx.x & 63;
    if constexpr (L == K_CONTIGUOUS) {
        const int row = row0 + (lane & 31), chunk = kk * 2 + (lane >> 5);
        return *(const bf16x8 *)(lds + row * kStepBytes +
                                 Operand<2, L, R, 1>::swizzle(row, chunk) * 16);
    } else {
        // The transposing read: 16 lanes read 4 k of 16 rows, each gets one row's 4 k.
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s4 lds_s4;
        const int k = kk * 16 + (lane >> 5) * 8 + ((lane >> 2) & 3);
        const int r = row0 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
        const char *p = lds + k * (R * 2) + Operand<2, L, R, 1>::swizzle(k, r >> 3) * 16 +
                        (r & 7) * 2;
        union {
            s4 h[2];
            bf16x8 f;
        } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)p);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(p + 4 * R * 2));
        return u.f;
    }
}

// A 32-row fragment of 64 8-bit values of k (step kk of 2): lane l holds k
// 16 (l / 32) + 0..15 and 32 more.
template <int R> __device__ __forceinline__ i32x8 fragment64(const char *lds, int row0, int kk)
{
    const int lane = threadIdx.x & 63;
    const int row = row0 + (lane & 31), chunk = kk * 4 + (lane >> 5);
    union {
        u32x4 h[2];
        i32x8 f;
    } u;
    u.h[0] = *(const u32x4 *)(lds + row * kStepBytes +
                              Operand<1, K_CONTIGUOUS, R, 1>::swizzle(row, chunk) * 16);
    u.h[1] = *(const u32x4 *)(lds + row * kStepBytes +
                              Operand<1, K_CONTIGUOUS, R, 1>::swizzle(row, chunk + 2) * 16);
    return u.f;
}

// A 32-row fragment of 16 k (step kk of 8) of block-scaled values as bf16, which holds each
// value: 4 significant bits, from scale byte 3 on (below, multiples of 2^-133).  s: the row's
// scales of the step.
template <int R>
__device__ __forceinline__ bf16x8 fragment_exact(const char *lds, uint32_t s, int row0, int kk)
{
    const int lane = threadIdx.x & 63, row = row0 + (lane & 31);
    const u32x2 q = *(const u32x2 *)(lds + row * kStepBytes +
                                     Operand<1, K_CONTIGUOUS, R, 1>::swizzle(row, kk) * 16 +
                                     (lane >> 5) * 8);
    const uint32_t byte = (s >> (kk / 2 * 8)) & 255u;
    const float scale = bits_f32(byte == 0 ? 0x00400000u : byte == 255u ? 0x7fc00000u : byte << 23);
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    union {
        b2 h[4];
        bf16x8 f;
    } u;
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[0], scale, false);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[0], scale, true);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[1], scale, false);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[1], scale, true);
    return u.f;
}

// Block scales of a step, a dword a row (bytes of 32 k each), copied to LDS like the rest:
// the tile's rows of both operands in order, 64 a wave's copy.  Rows of scales are whole
// dwords, and those past the operands' ends repeat the last.
template <int BM, int BN, int NT> struct Scales {
    static constexpr int kCopies = (BM + BN + NT - 1) / NT;
    static constexpr int kBytes = kCopies * NT * 4;
    const char *p[kCopies];
    __device__ __forceinline__ void init(const GemmArgs &g, int64_t m0, int64_t n0, int64_t k0)
    {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int r = i * NT + (int)threadIdx.x;
            const bool b = r >= BM;
            const int64_t row = b ? min(n0 + r - BM, g.N - 1) : min(m0 + r, g.M - 1);
            p[i] = (const char *)(b ? g.bs + row * g.bs_ld : g.as + row * g.as_ld) + k0 / kMxBlock;
        }
    }
    __device__ __forceinline__ void copy(uint32_t lds)
    {
        const uint32_t to = lds + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 256;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            copy4(p[i], to + i * NT * 4);
            p[i] += 4;
        }
    }
};

// EXACT: block-scaled values multiplied as bf16 (see gemm_mx).
template <int EB, bool EXACT, typename T, Layout LA, Layout LB, int BM, int BN, int WAVES_M,
          int WAVES_N>
__global__ void __launch_bounds__(64 * WAVES_M *WAVES_N)
    gemm_tile_kernel(GemmArgs g, uint32_t tiles_m, uint32_t tiles_n)
{
    constexpr int NW = WAVES_M * WAVES_N, NT = 64 * NW;
    constexpr int WM = BM / WAVES_M / 32, WN = BN / WAVES_N / 32;
    static_assert(WN == 2, "a wave's epilogue takes 64 columns");
    constexpr int kA = BM * kStepBytes, kB = BN * kStepBytes;
    constexpr int kScales = EB == 1 ? Scales<BM, BN, NT>::kBytes : 0;
    constexpr int kBuffer = kA + kB + kScales;
    constexpr int kEpilogue = NW * kEpilogueFloats * 4;
    __shared__ __attribute__((aligned(1024))) char lds[2 * kBuffer > kEpilogue ? 2 * kBuffer
                                                                               : kEpilogue];
    constexpr int kStepK = kStepBytes / EB;

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    uint32_t tm, tn, split;
    place_tile(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn, split);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int64_t kbeg = (int64_t)split * g.k_per, kend = min(g.K, kbeg + g.k_per);
    const int wm = (wave % WAVES_M) * (WM * 32), wn = (wave / WAVES_M) * (WN * 32);

    f32x16 acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    Operand<EB, LA, BM, NW> oa;
    Operand<EB, LB, BN, NW> ob;
    oa.init(g.a, g.lda, g.a_rows, m0, kbeg, LA == K_CONTIGUOUS ? min(kend, g.a_k) : min(kend, g.K));
    ob.init(g.b, g.ldb, g.b_rows, n0, kbeg, LB == K_CONTIGUOUS ? min(kend, g.b_k) : min(kend, g.K));
    Scales<BM, BN, NT> sc;
    const int steps = (int)((kend - kbeg + kStepK - 1) / kStepK);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const uint32_t lds_wave = lds_base + (uint32_t)__builtin_amdgcn_readfirstlane(wave) * 1024;
    // Step t's copies in kCopies pieces (the scales' loads with the first).
    constexpr int kCopiesA = Operand<EB, LA, BM, NW>::kCopies;
    constexpr int kCopies = kCopiesA + Operand<EB, LB, BN, NW>::kCopies;
    auto copy_piece = [&](int t, int i) __attribute__((always_inline)) {
        const uint32_t to = lds_wave + (t & 1) * kBuffer;
        if (EB == 1 && i == 0) sc.copy(lds_base + (t & 1) * kBuffer + kA + kB);
        if (i < kCopiesA) oa.copy_one(to, i);
        else ob.copy_one(to + kA, i - kCopiesA);
        if (i == kCopies - 1) oa.copied(), ob.copied();
    };
    auto copy = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy_piece(t, i);
    };
    auto copy_last = [&](int t) __attribute__((always_inline)) {
        const uint32_t to = lds_wave + (t & 1) * kBuffer;
        const int64_t k = kbeg + (int64_t)t * kStepK;
        if constexpr (EB == 1) sc.copy(lds_base + (t & 1) * kBuffer + kA + kB);
        oa.copy_last(to, k);
        ob.copy_last(to + kA, k);
    };
    constexpr int kParts = EB == 2 ? 4 : EXACT ? 8 : 2;
    using Fragment = std::conditional_t<EB == 1 && !EXACT, i32x8, bf16x8>;
    // Two sets of fragments where the registers hold them: a part's products run on one while
    // the other is read.
    constexpr int kSets = EB == 2 ? 2 : 1;
    Fragment fa[kSets][WM], fb[kSets][WN];
    uint32_t sa[WM], sb[WN], ua[WM], ub[WN];    // scales of the fragments read, and in use
    auto read_scales = [&](int t) __attribute__((always_inline)) {
        if constexpr (EB == 1) {
            // EXACT: the row's four scales.  Else a lane's scale is of the 32 k its half of
            // the wave stands for: byte 2 kk + lane / 32.
            const uint32_t *s = (const uint32_t *)(lds + (t & 1) * kBuffer + kA + kB);
            const int shift = EXACT ? 0 : (lane >> 5) * 8;
#pragma unroll
            for (int j = 0; j < WN; ++j) sb[j] = s[BM + wn + 32 * j + (lane & 31)] >> shift;
#pragma unroll
            for (int i = 0; i < WM; ++i) sa[i] = s[wm + 32 * i + (lane & 31)] >> shift;
        }
    };
    // Fragments of part kk of step t.
    auto read_b = [&](int t, int kk, int j) __attribute__((always_inline)) {
        const char *here = lds + (t & 1) * kBuffer + kA;
        Fragment &f = fb[kk % kSets][j];
        if constexpr (EB == 2) f = fragment16<LB, BN>(here, wn + 32 * j, kk);
        else if constexpr (EXACT) f = fragment_exact<BN>(here, sb[j], wn + 32 * j, kk);
        else f = fragment64<BN>(here, wn + 32 * j, kk);
    };
    auto read_a = [&](int t, int kk, int i) __attribute__((always_inline)) {
        const char *here = lds + (t & 1) * kBuffer;
        Fragment &f = fa[kk % kSets][i];
        if constexpr (EB == 2) f = fragment16<LA, BM>(here, wm + 32 * i, kk);
        else if constexpr (EXACT) f = fragment_exact<BM>(here, sa[i], wm + 32 * i, kk);
        else f = fragment64<BM>(here, wm + 32 * i, kk);
    };
    // The products of part kk of step t, columns by columns.  Between them the next part's
    // fragments are read: into the other set, evenly, in the order of their use, or with one
    // set behind the last product that needs the fragment before.  piece(i), i <
    // kCopies, goes out between them too.
    auto multiply = [&](auto part, int t, auto piece) __attribute__((always_inline)) {
        constexpr int kk = decltype(part)::value, next = (kk + 1) % kParts;
        constexpr int kProducts = WM * WN, kReads = WM + WN;
        const int tn = kk + 1 == kParts ? t + 1 : t;
        if constexpr (EB == 1 && kk == 0) {
#pragma unroll
            for (int i = 0; i < WM; ++i) ua[i] = sa[i];
#pragma unroll
            for (int j = 0; j < WN; ++j) ub[j] = sb[j];
        }
        if constexpr (next == 0) read_scales(tn);
#pragma unroll
        for (int j = 0; j < WN; ++j) {
#pragma unroll
            for (int i = 0; i < WM; ++i) {
                const int m = j * WM + i;
                const Fragment &a = fa[kk % kSets][i], &b = fb[kk % kSets][j];
                if constexpr (EB == 1 && !EXACT)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                        b, a, acc[i][j], 0, 0, 2 * kk, (int)ub[j], 2 * kk, (int)ua[i]);
                else
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (kSets == 2) {
#pragma unroll
                    for (int r = m * kReads / kProducts; r < (m + 1) * kReads / kProducts; ++r) {
                        if (r == 0) read_b(tn, next, 0);
                        else if (r <= WM) read_a(tn, next, r - 1);
                        else read_b(tn, next, r - WM);
                    }
                } else {
                    if (j == WN - 1) read_a(tn, next, i);
                    if (i == WM - 1) read_b(tn, next, j);
                }
#pragma unroll
                for (int c = m * kCopies / kProducts; c < (m + 1) * kCopies / kProducts; ++c)
                    piece(c);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    auto nothing = [](int) __attribute__((always_inline)) {};

    if constexpr (EB == 1) sc.init(g, m0, n0, kbeg);
    if (steps > 1) copy(0);
    else copy_last(0);
    if (steps > 1) {
        if (steps > 2) copy(1);
        else copy_last(1);
        wait_copies<kCopies + (EB == 1 ? Scales<BM, BN, NT>::kCopies : 0)>();
    } else {
        wait_copies<0>();
    }
    __syncthreads();
    read_scales(0);
#pragma unroll
    for (int j = 0; j < WN; ++j) read_b(0, 0, j);
#pragma unroll
    for (int i = 0; i < WM; ++i) read_a(0, 0, i);
    // A step.  Before its last part, which reads the next step's first fragments: the next
    // step's copies, in flight since the step before, have landed, and this step's buffer,
    // which all waves have read, takes the copies after those (`more`).  The steps
    // are straight code: a branch would let the compiler move products behind it.
    auto step = [&](int t, auto before, auto piece) __attribute__((always_inline)) {
        static_for<kParts - 1>([&](auto part) __attribute__((always_inline)) { multiply(part, t, nothing); });
        wait_copies<0>();
        __syncthreads();
        before(t + 2);
        multiply(std::integral_constant<int, kParts - 1>{}, t, piece);
    };
    int t = 0;
    for (; t + 3 < steps; ++t)
        step(t, nothing, [&](int i) __attribute__((always_inline)) { copy_piece(t + 2, i); });
    if (t + 2 < steps) step(t++, copy_last, nothing);
    if (t + 1 < steps) step(t++, nothing, nothing);
    // (the reads behind the last products are of what an earlier step left in LDS, unused)
    static_for<kParts>([&](auto part) __attribute__((always_inline)) { multiply(part, t, nothing); });
    __syncthreads();
    float *out = (float *)lds + wave * kEpilogueFloats;
    finish_wave<T>(g, out, m0 + wm, n0 + wn, split, acc);
}

// ---- shapes of tiles and splits of k ----
struct TilePlan {
    int bm, bn;
    uint32_t tiles_m, tiles_n;
    int64_t k_per;
    int splits;
};

inline TilePlan plan_tiles(int64_t M, int64_t N, int64_t K, int step_k)
{
    TilePlan p{};
    auto tiles = [&](int bm, int bn) __attribute__((always_inline)) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
    // Few rows: the sums of rows that are not there would cost what the bytes of b leave (17 x
    // 4096 x 16384 bf16 26 us, 32 us in tiles of 128 x 128).  Past 32 rows with few columns
    // the parts' sums do (64 x 4096 x 16384 32 and 36 us, 64 x 4096 x 4096 18 and 16 us).
    if (M <= 32) p.bm = 32, p.bn = 256;
    else if (M <= 64 && tiles(64, 256) >= 64) p.bm = 64, p.bn = 256;
    // 256 x 256 where most of the device has a tile and padding costs less than a quarter
    // (262144 x 128 x 512 and its dx of 128 columns: 115 and 114 us in these tiles,
    // 139 and 77 us in tiles of 128 x 128; 8192 x 2048 x 8192: 229 and 280 us).
    else if (tiles(256, 256) >= 192 && 16 * tiles(256, 256) <= 5 * tiles(128, 128))
        p.bm = 256, p.bn = 256;
    else p.bm = 128, p.bn = 128;
    p.tiles_m = (uint32_t)((M + p.bm - 1) / p.bm);
    p.tiles_n = (uint32_t)((N + p.bn - 1) / p.bn);
    const int64_t t = (int64_t)p.tiles_m * p.tiles_n, steps = (K + step_k - 1) / step_k;
    // Fewer tiles than compute units: k is split, four steps or more a part, over one workgroup
    // a unit (512 x 4096 x 1024: 22 us, 28 us with two, whose partial sums cost more than they
    // hide), or two where their parts stay long (128 x 262144 x 512: 76 us, 84 us with one).
    int64_t s = t >= 256 ? 1 : 256 / t;
    if (t < 256 && p.bm < 256 && steps / (2 * s) >= 32) s *= 2;
    s = s < steps / 4 ? s : steps / 4;
    if (s < 1) s = 1;
    p.k_per = (steps + s - 1) / s * step_k;
    p.splits = (int)((K + p.k_per - 1) / p.k_per);
    return p;
}

inline uint64_t tile_part_bytes(int64_t M, int64_t N, int64_t K, int step_k)
{
    const TilePlan p = plan_tiles(M, N, K, step_k);
    return p.splits > 1 ? (uint64_t)p.splits * M * N * 4 : 0;
}

template <int EB, bool EXACT, typename T, Layout LA, Layout LB>
hipError_t run_tiles(GemmArgs g, float *part, hipStream_t stream)
{
    const TilePlan p = plan_tiles(g.M, g.N, g.K, kStepBytes / EB);
    g.k_per = p.k_per;
    g.part = p.splits > 1 ? part : nullptr;
    const dim3 grid(p.tiles_m * p.tiles_n * (uint32_t)p.splits);
    if (p.bm == 32)
        gemm_tile_kernel<EB, EXACT, T, LA, LB, 32, 256, 1, 4><<<grid, 256, 0, stream>>>(g, p.tiles_m, p.tiles_n);
    else if (p.bm == 64)
        gemm_tile_kernel<EB, EXACT, T, LA, LB, 64, 256, 1, 4><<<grid, 256, 0, stream>>>(g, p.tiles_m, p.tiles_n);
    else if (p.bm == 256)
        gemm_tile_kernel<EB, EXACT, T, LA, LB, 256, 256, 2, 4><<<grid, 512, 0, stream>>>(g, p.tiles_m, p.tiles_n);
    else
        gemm_tile_kernel<EB, EXACT, T, LA, LB, 128, 128, 2, 2><<<grid, 256, 0, stream>>>(g, p.tiles_m, p.tiles_n);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    return launch_split_sum<T>(g, p.splits, stream);
}

}  // namespace whtmix
