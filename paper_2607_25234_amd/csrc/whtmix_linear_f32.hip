// Products of float32 operands, each split into three bf16 terms (24 significant bits), six of
// the nine products formed on v_mfma_f32_32x32x16_bf16 with sums in float32.
//
// Two kernels.  Where the product is bound by memory, operands are split on their way to LDS
// (gemm_kernel).  Where it is bound by the matrix cores, that costs more vector
// instructions than the cores leave time for: a pass of its own splits each operand once
// (split_kernel) into the order in which the tile kernel (gemm_split_kernel) copies it.
#include "whtmix_gemm.h"

#include <algorithm>

namespace whtmix {
namespace {

constexpr int kStep = 32;
constexpr int kRowBytes = 64;      // of a plane: 32 bf16, of one row or of 32 rows of one k

// Where 16-byte chunk `chunk` of a row (or k) lies in a plane of ROWS rows: permuted so that
// the 16 lanes of an LDS cycle fall on all banks (rows of a fragment; 4 k x 2 groups of 16
// rows of a transposing read).
template <Layout L, int ROWS> __device__ __forceinline__ int place_chunk(int outer, int chunk)
{
    if constexpr (L == K_CONTIGUOUS) return outer * kRowBytes + (chunk ^ ((outer >> 2) & 3)) * 16;
    // (the gated form's halves; a single product's dw of 131072 x 64 x 256 63 us before and since)
    else if constexpr (ROWS == 64) return outer * (2 * ROWS) + (chunk ^ (2 * outer & 4)) * 16;
    else return outer * (2 * ROWS) + (chunk ^ ((4 * (outer & 3)) & (ROWS / 8 - 1))) * 16;
}

// Three bf16 terms hold a float32 below 2^128 - 2^119 (above, the first rounds to Inf) and from
// 2^-100 up (below, the last is subnormal).  Smaller values beside larger ones of their row of x
// or column of w are off by half of 2^-133 at most, bf16's least value.
constexpr float kSplitMax = 0x1.ffp127f, kSplitMin = 0x1p-95f;
constexpr int P = 3;               // bf16 terms of a float32

// A step of ROWS rows of an operand in the workgroup's registers, four elements along memory
// at a time: a row's chunks are neighbouring lanes'.
template <Layout L, int ROWS> struct Stage {
    static constexpr int kChunks = ROWS / 32, kPlane = ROWS * kRowBytes;
    static constexpr int kF32Row = ROWS + 4;        // float32 staging: floats of one k
    float v[kChunks][4];
    // Chunk i of the thread: (row, k) of its first element.
    static __device__ __forceinline__ void place(int i, int &row, int &k)
    {
        const int c = i * 256 + threadIdx.x;
        if (L == K_CONTIGUOUS) row = c >> 3, k = (c & 7) * 4;
        else k = c / (ROWS / 4), row = c % (ROWS / 4) * 4;
    }
    // The thread's first chunk at the current step; the others are a constant way apart.
    const float *at;
    int64_t apart, ahead;
    int rows, ks;           // left of the operand from there on
    __device__ __forceinline__ void init(const void *p, int64_t ld, int64_t R, int64_t K,
                                         int64_t r0, int64_t k0)
    {
        int row, k;
        place(0, row, k);
        at = (const float *)p + (L == K_CONTIGUOUS ? (r0 + row) * ld + k0 + k
                                                   : (k0 + k) * ld + r0 + row);
        apart = (L == K_CONTIGUOUS ? 32 : 1024 / ROWS) * ld;
        ahead = L == K_CONTIGUOUS ? kStep : kStep * ld;
        rows = (int)max(min(R - r0 - row, (int64_t)1 << 20), (int64_t)-(1 << 20));
        ks = (int)min(K - k0 - k, ((int64_t)1 << 31) - 1);
    }
    __device__ __forceinline__ void load()
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const bool in = L == K_CONTIGUOUS ? rows > 32 * i : ks > 1024 / ROWS * i;
            Chunk<float>::load(at + i * apart, in ? (L == K_CONTIGUOUS ? ks : rows) : 0, v[i]);
        }
        at += ahead;
        ks -= kStep;
    }
    // As float32, [k][row], for operands that do not split.
    __device__ __forceinline__ void store_f32(float *lds) const
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            int row, k;
            place(i, row, k);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                lds[(k + (L == K_CONTIGUOUS ? j : 0)) * kF32Row + row +
                    (L == K_CONTIGUOUS ? 0 : j)] = v[i][j];
        }
    }
    // The largest magnitudes staged so far of each row that the thread's chunks are of: one a
    // chunk (K_CONTIGUOUS), or the same four in all of them.  (A NaN is passed over: it
    // makes its row's sums NaN either way.)
    static constexpr int kTops = L == K_CONTIGUOUS ? kChunks : 4;
    __device__ __forceinline__ void largest(float (&top)[kTops]) const
    {
        if constexpr (L == K_CONTIGUOUS) {
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                top[i] = fmaxf(fmaxf(top[i], fabsf(v[i][0])), fabsf(v[i][1]));
                top[i] = fmaxf(fmaxf(top[i], fabsf(v[i][2])), fabsf(v[i][3]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < kChunks; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) top[j] = fmaxf(top[j], fabsf(v[i][j]));
        }
    }
    __device__ __forceinline__ void store(char *lds)
    {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            int row, k;
            place(i, row, k);
            const int inner = L == K_CONTIGUOUS ? k : row;
            char *p = lds + place_chunk<L, ROWS>(L == K_CONTIGUOUS ? row : k, inner >> 3) + (inner & 7) * 2;
#pragma unroll
            for (int s = 0; s < P; ++s) {
                const uint32_t w0 = pack_bf16(v[i][0], v[i][1]), w1 = pack_bf16(v[i][2], v[i][3]);
                *(u32x2 *)(p + s * kPlane) = (u32x2){w0, w1};
                if (s + 1 < P) {
                    v[i][0] -= bits_f32(w0 << 16);
                    v[i][1] -= bits_f32(w0 & 0xffff0000u);
                    v[i][2] -= bits_f32(w1 << 16);
                    v[i][3] -= bits_f32(w1 & 0xffff0000u);
                }
            }
        }
    }
};

// The operand of a 32x32x16 product: lane l holds row l % 32, k 8 (l / 32) + 0..7.
// K_STRIDED planes are read through the transposing LDS load: a group of 16
// lanes reads 4 k of 16 rows and each lane gets one row's 4 k.
template <Layout L, int ROWS>
__device__ __forceinline__ bf16x8 fragment(const char *plane, int row0, int k0)
{
    const int lane = threadIdx.x & 63;
    if constexpr (L == K_CONTIGUOUS) {
        return *(const bf16x8 *)(plane + place_chunk<L, ROWS>(row0 + (lane & 31),
                                                              (k0 >> 3) + (lane >> 5)));
    } else {
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s4 lds_s4;
        const int k = k0 + (lane >> 5) * 8 + ((lane >> 2) & 3);
        const int r = row0 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
        const char *p = plane + place_chunk<L, ROWS>(k, r >> 3) + (r & 7) * 2;    // k + 4: alike
        union {
            s4 h[2];
            bf16x8 f;
        } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)p);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(p + 4 * 2 * ROWS));
        return u.f;
    }
}

// The tile again with float32 products (v_mfma_f32_32x32x2_f32).
template <Layout LA, Layout LB, int BM, int BC, int NB, int WM>
__device__ __forceinline__ void float32_tile(const GemmArgs &g, Stage<LA, BM> &sa,
                                             Stage<LB, BC> (&sb)[NB], float *lds, int64_t m0,
                                             int64_t n0, int64_t kbeg, int64_t kend, int wm, int wn,
                                             f32x16 (&acc)[WM][2])
{
    constexpr int kA = Stage<LA, BM>::kF32Row, kB = Stage<LB, BC>::kF32Row;
    constexpr int kApart = NB == 1 ? 32 : kStep * kB;       // of a wave's columns, 32 by 32
    const int lane = threadIdx.x & 63;
    float *la = lds, *lb = lds + kStep * kA;
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    sa.init(g.a, g.lda, g.M, kend, m0, kbeg);
    sb[0].init(g.b, g.ldb, g.N, kend, n0, kbeg);
    if constexpr (NB == 2) sb[1].init(g.b2, g.ldb2, g.N, kend, n0, kbeg);
    for (int64_t k = kbeg; k < kend; k += kStep) {
        sa.load();
#pragma unroll
        for (int b = 0; b < NB; ++b) sb[b].load();
        __syncthreads();
        sa.store_f32(la);
#pragma unroll
        for (int b = 0; b < NB; ++b) sb[b].store_f32(lb + b * kStep * kB);
        __syncthreads();
        for (int kk = 0; kk < kStep; kk += 2) {
            const float *pa = la + (kk + (lane >> 5)) * kA + wm + (lane & 31);
            const float *pb = lb + (kk + (lane >> 5)) * kB + wn + (lane & 31);
#pragma unroll
            for (int i = 0; i < WM; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(pb[kApart * j], pa[32 * i],
                                                                     acc[i][j], 0, 0, 0);
        }
    }
}

// BM x BN sums by four waves of 64 columns.  The next step's loads are in flight during the
// products of this one; two or three workgroups fill in for each other at the barriers.
// Bound by the splits' vector instructions: 131072 x 64 x 256 with gelu 57-66 us (168 MB at
// 2.5-2.9 TB/s, two steps a tile), 3001 x 1000 x 2003's gradients 105 us each, 115 TFLOP/s.
template <Layout LA, Layout LB, int FORM, int BM, int BN>
__global__ void __launch_bounds__(256) gemm_kernel(GemmArgs g)
{
    constexpr int WAVES_N = BN / 64, WAVES_M = 4 / WAVES_N, WM = BM / WAVES_M / 32;
    // B's tile, or GATED both B's, one after the other, of as many columns each.
    constexpr int NB = FORM == GATED ? 2 : 1, BC = BN / NB;
    constexpr int kPlaneA = Stage<LA, BM>::kPlane, kPlaneB = Stage<LB, BC>::kPlane;
    constexpr int kPlanes = P * (kPlaneA + NB * kPlaneB), kEpilogue = 4 * kEpilogueFloats * 4;
    static_assert(kStep * (Stage<LA, BM>::kF32Row + NB * Stage<LB, BC>::kF32Row) * 4 <= kPlanes,
                  "float32 staging in the planes' place");
    __shared__ __attribute__((aligned(16))) char lds[kPlanes > kEpilogue ? kPlanes : kEpilogue];
    const int wave = threadIdx.x >> 6;
    const int64_t m0 = (int64_t)blockIdx.x * BM, n0 = (int64_t)blockIdx.y * BC;
    const int64_t kbeg = (int64_t)blockIdx.z * g.k_per, kend = min(g.K, kbeg + g.k_per);
    const int wm = wave % WAVES_M * (WM * 32), wn = wave / WAVES_M * (64 / NB);
    char *la = lds, *lb = lds + P * kPlaneA;
    f32x16 acc[WM][2];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    Stage<LA, BM> sa;
    Stage<LB, BC> sb[NB];
    float top_a[Stage<LA, BM>::kTops] = {}, top_b[NB][Stage<LB, BC>::kTops] = {};   // what the splits hold
    sa.init(g.a, g.lda, g.M, kend, m0, kbeg);
    sb[0].init(g.b, g.ldb, g.N, kend, n0, kbeg);
    if constexpr (NB == 2) sb[1].init(g.b2, g.ldb2, g.N, kend, n0, kbeg);
    sa.load();
#pragma unroll
    for (int b = 0; b < NB; ++b) sb[b].load();
    for (int64_t k = kbeg; k < kend; k += kStep) {
        __syncthreads();
        sa.largest(top_a);
#pragma unroll
        for (int b = 0; b < NB; ++b) sb[b].largest(top_b[b]);
        sa.store(la);
#pragma unroll
        for (int b = 0; b < NB; ++b) sb[b].store(lb + b * P * kPlaneB);
        if (k + kStep < kend) {
            sa.load();
#pragma unroll
            for (int b = 0; b < NB; ++b) sb[b].load();
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kStep; kk += 16) {
            bf16x8 fa[P][WM];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < WM; ++i)
                    fa[p][i] = fragment<LA, BM>(la + p * kPlaneA, wm + 32 * i, kk);
            // Of the nine products of three terms the six largest, small ones first: what is
            // left out is below 2^-24 of |x| |w|.
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                bf16x8 fb[P];
#pragma unroll
                for (int p = 0; p < P; ++p)
                    fb[p] = fragment<LB, BC>(lb + ((NB - 1) * j * P + p) * kPlaneB,
                                             wn + (NB == 1 ? 32 * j : 0), kk);
#pragma unroll
                for (int s = P - 1; s >= 0; --s)
#pragma unroll
                    for (int p = 0; p <= s; ++p)
#pragma unroll
                        for (int i = 0; i < WM; ++i)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[s - p], fa[p][i],
                                                                                acc[i][j], 0, 0, 0);
            }
        }
    }
    auto bad = [](float top) { return top >= kSplitMax || (top != 0.f && top < kSplitMin); };
    // A row's values (of this thread's k) that do not split send the whole tile through
    // float32 products.
    bool any = false;
#pragma unroll
    for (int i = 0; i < Stage<LA, BM>::kTops; ++i) any = any || bad(top_a[i]);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < Stage<LB, BC>::kTops; ++i) any = any || bad(top_b[b][i]);
    if (__syncthreads_or(any))
        float32_tile<LA, LB, BM, BC, NB, WM>(g, sa, sb, (float *)lds, m0, n0, kbeg, kend, wm, wn, acc);
    __syncthreads();
    float *out = (float *)lds + wave * kEpilogueFloats;
    if constexpr (FORM == GATED) finish_gated_wave<float>(g, out, m0 + wm, n0 + wn, blockIdx.z, acc);
    else finish_wave<float, FORM>(g, out, m0 + wm, n0 + wn, blockIdx.z, acc);
}

// Rows and columns of a tile: 128 x 128, or fewer rows where there are not more (1 x 2048 x
// 4096 14 us, 16 in tiles of 64 rows, 24 of 128; 64 x 2048 x 4096 26 us, 30 of 128).
int tile_rows(int64_t M) { return M <= 32 ? 32 : M <= 64 ? 64 : 128; }
int tile_columns(int64_t M) { return M <= 64 ? 256 : 128; }

// How many parts k is split into: two workgroups a unit where the output has few tiles (three
// fit), four steps of k or more each, or two where few rows make the sums cheap.  Fewer
// parts: 154 x 1491 x 16384 77 and 99 us with one workgroup a unit.  Shorter ones: 512 x 2048 x 512
// 22 and 25 us with two steps; 64 x 1000 x 1000 15 and 20 us with four.
int64_t splits_of(int64_t M, int64_t N, int64_t K)
{
    const int bm = tile_rows(M), bn = tile_columns(M);
    const int64_t tiles = ((M + bm - 1) / bm) * ((N + bn - 1) / bn);
    const int64_t steps = (K + kStep - 1) / kStep;
    return std::max<int64_t>(1, std::min<int64_t>(512 / tiles, steps / (M <= 64 ? 2 : 4)));
}

uint64_t gemm_bytes(int64_t M, int64_t N, int64_t K)
{
    const int64_t s = splits_of(M, N, K);
    return s > 1 ? (uint64_t)s * M * N * 4 : 0;
}

// Columns of the tiles' B's together.
int64_t columns(const GemmArgs &g, Form form) { return form == GATED ? 2 * g.N : g.N; }

template <Layout LA, Layout LB, Form FORM = PLAIN>
hipError_t run_gemm(GemmArgs g, float *ws, hipStream_t stream)
{
    const int64_t n = columns(g, FORM), s = splits_of(g.M, n, g.K);
    const int64_t steps = (g.K + kStep - 1) / kStep;
    g.k_per = (steps + s - 1) / s * kStep;
    const int64_t splits = (g.K + g.k_per - 1) / g.k_per;
    g.part = splits > 1 ? ws : nullptr;
    const int bm = tile_rows(g.M), bn = tile_columns(g.M);
    const dim3 grid((uint32_t)((g.M + bm - 1) / bm), (uint32_t)((n + bn - 1) / bn),
                    (uint32_t)splits);
    if (bm == 32) gemm_kernel<LA, LB, FORM, 32, 256><<<grid, dim3(256), 0, stream>>>(g);
    else if (bm == 64) gemm_kernel<LA, LB, FORM, 64, 256><<<grid, dim3(256), 0, stream>>>(g);
    else gemm_kernel<LA, LB, FORM, 128, 128><<<grid, dim3(256), 0, stream>>>(g);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    return launch_split_sum<float, FORM>(g, (int)splits, stream);
}

// ---- operands split in a pass of their own ----
// Terms in blocks of 16 k: [k / 16][term][row][16], rows padded to 256 and k to 16 with zeros.
// A row's two 16-byte halves are swapped in every second group of 8 rows: a cycle of an LDS
// read, 16 rows' halves 32 bytes apart, then falls on all banks.
constexpr int kSplitRows = 256, kBlockK = 16, kRowTermBytes = 32;

constexpr int64_t split_rows(int64_t rows) { return (rows + kSplitRows - 1) / kSplitRows * kSplitRows; }
constexpr int64_t split_blocks(int64_t k) { return (k + kBlockK - 1) / kBlockK; }
// Flags, one a workgroup of the pass (64 rows x 4 blocks of k): whether its values do not split.
constexpr int64_t split_groups(int64_t k) { return (split_blocks(k) + 3) / 4; }

uint64_t split_bytes(int64_t rows, int64_t k)
{
    return (uint64_t)split_blocks(k) * P * split_rows(rows) * kRowTermBytes +
           (uint64_t)split_groups(k) * (split_rows(rows) / 64) * 4;
}

struct SplitJob {
    const float *src;
    int64_t ld, rows;
    char *out;
    uint32_t *flags;
    uint32_t across, blocks;        // workgroups along the rows, and in all
    Layout layout;
};

// Workgroup `at` of an operand's.
template <Layout L>
__device__ __forceinline__ void split_block(const SplitJob &job, int64_t K, uint32_t at)
{
    const float *src = job.src;
    const int64_t ld = job.ld, rows = job.rows;
    const int t = threadIdx.x;
    // Sixteen k of a row a thread; neighbouring lanes take neighbouring rows.
    const int64_t row = (int64_t)(at % job.across) * 64 +
                        (L == K_CONTIGUOUS ? t % 16 + t / 64 * 16 : t % 64);
    const int64_t block = (int64_t)(at / job.across) * 4 + (L == K_CONTIGUOUS ? t / 16 % 4 : t / 64);
    const int64_t k0 = block * kBlockK;
    const int n = row < rows ? (int)max((int64_t)0, min((int64_t)kBlockK, K - k0)) : 0;
    float v[16];
    if constexpr (L == K_CONTIGUOUS) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            Chunk<float>::load(src + (n ? row * ld + k0 + 4 * i : 0), n - 4 * i,
                               *(float(*)[4])(v + 4 * i));
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = i < n ? src[(k0 + i) * ld + row] : 0.f;
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(v[i]));
    const int64_t padded = (int64_t)job.across * 64;
    if (block < split_blocks(K)) {
        char *to = job.out + (block * P * padded + row) * kRowTermBytes;
        const int swap = (int)(row >> 3 & 1) * 16;
#pragma unroll
        for (int s = 0; s < P; ++s) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
                if (s + 1 < P) {
                    v[2 * i] -= bits_f32(w[i] << 16);
                    v[2 * i + 1] -= bits_f32(w[i] & 0xffff0000u);
                }
            }
            *(u32x4 *)(to + s * padded * kRowTermBytes + swap) = (u32x4){w[0], w[1], w[2], w[3]};
            *(u32x4 *)(to + s * padded * kRowTermBytes + (swap ^ 16)) =
                (u32x4){w[4], w[5], w[6], w[7]};
        }
    }
    const int bad = __syncthreads_or(top >= kSplitMax || (top != 0.f && top < kSplitMin));
    if (t == 0) job.flags[at] = bad ? 1u : 0u;
}

// All operands of a product in one launch, the smaller under the larger's end (whole calls: 3001 x
// 1000 x 2 x 2003 gated 145 us, 152 in three launches, its gradients 390 and 398; 3001 x 1000 x
// 2003 86 and 91).
__global__ void __launch_bounds__(256) split_kernel(SplitJob a, SplitJob b, SplitJob b2, int64_t K)
{
    uint32_t at = blockIdx.x;
    SplitJob job = a;
    if (at >= a.blocks) {
        at -= a.blocks, job = b;
        if (at >= b.blocks) at -= b.blocks, job = b2;
    }
    if (job.layout == K_CONTIGUOUS) split_block<K_CONTIGUOUS>(job, K, at);
    else split_block<K_STRIDED>(job, K, at);
}

struct SplitOperand {
    const char *terms;
    const uint32_t *flags;
    int64_t rows;           // padded
    Layout layout;          // of the float32 operand
};

// Sums of a wave's tile from the float32 operands in memory, for values that do not split.
template <int FORM, int WM>
__device__ __forceinline__ void float32_wave(const GemmArgs &g, Layout la, Layout lb, int64_t m0,
                                             int64_t n0, int64_t kbeg, int64_t kend,
                                             f32x16 (&acc)[WM][2])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    auto at = [&](const void *p, Layout l, int64_t ld, int64_t row, int64_t rows, int64_t k) {
        if (row >= rows || k >= kend) return 0.f;
        return ((const float *)p)[l == K_CONTIGUOUS ? row * ld + k : k * ld + row];
    };
    for (int64_t k = kbeg + (lane >> 5); k - (lane >> 5) < kend; k += 2) {
        float a[WM], b[2];
#pragma unroll
        for (int i = 0; i < WM; ++i) a[i] = at(g.a, la, g.lda, m0 + 32 * i + (lane & 31), g.M, k);
#pragma unroll
        for (int j = 0; j < 2; ++j)
            b[j] = FORM == GATED && j == 1
                       ? at(g.b2, lb, g.ldb2, n0 + (lane & 31), g.N, k)
                       : at(g.b, lb, g.ldb, n0 + 32 * j + (lane & 31), g.N, k);
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(b[j], a[i], acc[i][j], 0, 0, 0);
    }
}

__device__ __forceinline__ int piece_of(int i, int pieces) { return i < pieces ? i : i - pieces; }

// Three buffers: a step's copies (16 k of three terms of both operands) have two steps to land.
// 16384 x 4096 x 4096 2500 us, 219 TFLOP/s of float32 or 1.3 PFLOP/s of bf16 products; 3001 x 1000
// x 2003 85 us, 141: 384 tiles of 128 x 128 leave the second of two places on half of the units
// empty.
template <int FORM, int BM, int BN, int WAVES_M, int WAVES_N>
__global__ void __launch_bounds__(64 * WAVES_M *WAVES_N)
    gemm_split_kernel(GemmArgs g, SplitOperand a, SplitOperand b, SplitOperand b2, uint32_t tiles_m,
                      uint32_t tiles_n)
{
    constexpr int NB = FORM == GATED ? 2 : 1, BC = BN / NB;    // as in gemm_kernel
    constexpr int NW = WAVES_M * WAVES_N, WM = BM / WAVES_M / 32;
    static_assert(BN / WAVES_N == 64, "a wave's epilogue takes 64 columns");
    constexpr int kA = P * BM * kRowTermBytes, kB = P * BN * kRowTermBytes, kBuffer = kA + kB;
    constexpr int kPieces = kBuffer / 1024, kPiecesA = kA / 1024, kCopies = (kPieces + NW - 1) / NW;
    static_assert(kBuffer % 1024 == 0 && kA % 1024 == 0, "whole pieces");
    constexpr int kEpilogue = NW * kEpilogueFloats * 4;
    __shared__ __attribute__((aligned(1024))) char lds[3 * kBuffer > kEpilogue ? 3 * kBuffer
                                                                               : kEpilogue];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    uint32_t tm, tn, split;
    place_tile(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn, split);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BC;
    const int64_t kbeg = (int64_t)split * g.k_per, kend = min(g.K, kbeg + g.k_per);
    const int steps = (int)((kend - kbeg + kBlockK - 1) / kBlockK);
    const int wm = (wave % WAVES_M) * (WM * 32), wn = (wave / WAVES_M) * (64 / NB);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

    // 1024 bytes a piece: 32 rows of a term, A's and then B's (those behind an operand's padding
    // repeat its last).  Where they do not come out even some are copied twice.
    const char *from[kCopies];
    int64_t ahead[kCopies];
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
        const int nth = piece_of(i * NW + wave, kPieces);
        const bool ofb = nth >= kPiecesA;
        int piece = ofb ? nth - kPiecesA : nth;
        const int per = (ofb ? BC : BM) / 32;
        const bool second = ofb && piece >= P * per;
        if (second) piece -= P * per;
        const SplitOperand &o = second ? b2 : ofb ? b : a;
        const int64_t row = min((ofb ? n0 : m0) + piece % per * 32, o.rows - 32);
        from[i] = o.terms + ((kbeg / kBlockK * P + piece / per) * o.rows + row) * kRowTermBytes;
        ahead[i] = P * o.rows * kRowTermBytes;
    }
    auto copy = [&](int t) __attribute__((always_inline)) {
        const uint32_t to = lds_base + (uint32_t)(t % 3) * kBuffer;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            copy16(from[i], lane * 16, to + piece_of(i * NW + wave, kPieces) * 1024);
            from[i] += ahead[i];
        }
    };

    f32x16 acc[WM][2];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    copy(0);
    if (steps > 1) copy(1);
    auto step = [&](int t, auto left, auto more) __attribute__((always_inline)) {
        wait_copies<decltype(left)::value>();
        __syncthreads();        // step t has landed for all; step t - 1 has been read by all
        more(t + 2);
        const char *here = lds + (t % 3) * kBuffer;
        const int half = ((lane >> 5) ^ (lane >> 3 & 1)) * 16, row = (lane & 31) * kRowTermBytes;
        bf16x8 fa[P][WM], fb[P][2];
#pragma unroll
        for (int p = P - 1; p >= 0; --p) {
#pragma unroll
            for (int i = 0; i < WM; ++i)
                fa[p][i] = *(const bf16x8 *)(here + (p * BM + wm + 32 * i) * kRowTermBytes + row + half);
#pragma unroll
            for (int j = 0; j < 2; ++j)
                fb[P - 1 - p][j] = *(const bf16x8 *)(
                    here + kA +
                    (((NB - 1) * j * P + P - 1 - p) * BC + wn + (NB == 1 ? 32 * j : 0)) *
                        kRowTermBytes +
                    row + half);
        }
        // The six largest of the nine products, small ones first: what is left out is below
        // 2^-24 of |x| |w|.
#pragma unroll
        for (int s = P - 1; s >= 0; --s)
#pragma unroll
            for (int p = s; p >= 0; --p)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < WM; ++i)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            fb[s - p][j], fa[p][i], acc[i][j], 0, 0, 0);
    };
    auto nothing = [](int) __attribute__((always_inline)) {};
    int t = 0;
    for (; t + 2 < steps; ++t) step(t, std::integral_constant<int, kCopies>{}, copy);
    if (t + 1 < steps) step(t++, std::integral_constant<int, kCopies>{}, nothing);
    step(t, std::integral_constant<int, 0>{}, nothing);

    // Values of this tile's operands that do not split: float32 products instead.
    bool bad = false;
    const int64_t g0 = kbeg / (4 * kBlockK), g1 = (kend + 4 * kBlockK - 1) / (4 * kBlockK);
    for (int64_t i = threadIdx.x; i < (g1 - g0) * (BM / 64 + BN / 64); i += 64 * NW) {
        const int64_t grp = g0 + i / (BM / 64 + BN / 64), r = i % (BM / 64 + BN / 64);
        const int64_t rb = r - BM / 64;
        const SplitOperand &o = NB == 2 && rb >= BC / 64 ? b2 : b;
        bad = bad || (r < BM / 64 ? a.flags[grp * (a.rows / 64) + min(m0 / 64 + r, a.rows / 64 - 1)]
                                  : o.flags[grp * (o.rows / 64) + n0 / 64 + rb % (BC / 64)]) != 0;
    }
    if (__syncthreads_or(bad))
        float32_wave<FORM, WM>(g, a.layout, b.layout, m0 + wm, n0 + wn, kbeg, kend, acc);
    __syncthreads();
    float *out = (float *)lds + wave * kEpilogueFloats;
    if constexpr (FORM == GATED) finish_gated_wave<float>(g, out, m0 + wm, n0 + wn, split, acc);
    else finish_wave<float, FORM>(g, out, m0 + wm, n0 + wn, split, acc);
}

// Whether the passes that split the operands (10 bytes an element at 4.5 TB/s, and a launch
// more) cost less than what the tile kernel saves: it reaches about 210 TFLOP/s of float32, the
// kernel that splits on the way about 150.  Measured, first against second: 16384 x 4096 x
// 4096 2567 and 3219 us, 3001 x 1000 x 2003 86 and 107 us, 512 x 2048 x 2048 56 and 43 us, 65536 x
// 128 x 512 90 and 76 us.
bool splits_first(int64_t M, int64_t N, int64_t K)
{
    if (M < 128 || N < 128 || K < 128 || split_groups(K) > 65535) return false;
    const double pass = 10.0 * ((double)M * K + (double)N * K) / 4.5e12 + 8e-6;
    const double saved = 2.0 * M * N * K * (1 / 150e12 - 1 / 210e12);
    return saved > pass && split_bytes(M, K) + split_bytes(N, K) <= uint64_t(1) << 32;
}

struct SplitPlan {
    int rows;               // of a tile: 128 (128 columns), 192 or 256 (256 columns)
    uint32_t tiles_m, tiles_n;
    int64_t k_per;
    int splits;
};

SplitPlan plan_split(int64_t M, int64_t N, int64_t K)
{
    SplitPlan p{};
    auto tiles = [&](int b) { return ((M + b - 1) / b) * ((N + b - 1) / b); };
    const bool large = tiles(256) >= 192 && 16 * tiles(256) <= 5 * tiles(128);
    const int b = large ? 256 : 128, at_once = large ? 256 : 512;
    p.rows = b;
    p.tiles_m = (uint32_t)((M + b - 1) / b);
    p.tiles_n = (uint32_t)((N + b - 1) / b);
    // Parts of k where that fills the device's last round better: each part costs a pass over
    // its sums, taken as 12 steps of k.
    const int64_t t = (int64_t)p.tiles_m * p.tiles_n, steps = (split_blocks(K) + 3) / 4;
    int64_t best = 1;
    double cost = 1e30;
    for (int64_t s = 1; s <= 32 && s <= std::max<int64_t>(1, steps / 4); ++s) {
        const double rounds = (double)((t * s + at_once - 1) / at_once);
        const double c = rounds * ((double)((steps + s - 1) / s) + 3) + (s > 1 ? 3.0 * s : 0.0);
        if (c < cost) cost = c, best = s;
    }
    p.k_per = (steps + best - 1) / best * 4 * kBlockK;
    p.splits = (int)((K + p.k_per - 1) / p.k_per);
    // Tiles of 192 rows where those leave fewer units idle in the last round.
    if (large && p.splits == 1) {
        const int64_t m = (M + 191) / 192, t192 = m * p.tiles_n;
        if ((t192 + 255) / 256 * 192 < (t + 255) / 256 * 256) p.rows = 192, p.tiles_m = (uint32_t)m;
    }
    return p;
}

SplitJob split_operand(const void *p, Layout l, int64_t ld, int64_t rows, int64_t K, char *&ws,
                       SplitOperand &o)
{
    o.rows = split_rows(rows);
    o.terms = ws;
    o.layout = l;
    char *flags = ws + (uint64_t)split_blocks(K) * P * o.rows * kRowTermBytes;
    o.flags = (const uint32_t *)flags;
    const uint32_t across = (uint32_t)(o.rows / 64);
    const SplitJob job{(const float *)p, ld, rows, ws, (uint32_t *)flags, across,
                       across * (uint32_t)split_groups(K), l};
    ws += (split_bytes(rows, K) + 1023) / 1024 * 1024;
    return job;
}

template <Form FORM>
hipError_t run_split(GemmArgs g, Layout la, Layout lb, void *ws, hipStream_t stream)
{
    char *w = (char *)ws;
    SplitOperand a{}, b{}, b2{};
    const SplitJob ja = split_operand(g.a, la, g.lda, g.M, g.K, w, a);
    const SplitJob jb = split_operand(g.b, lb, g.ldb, g.N, g.K, w, b);
    SplitJob jb2{};
    if (FORM == GATED) jb2 = split_operand(g.b2, lb, g.ldb2, g.N, g.K, w, b2);
    split_kernel<<<dim3(ja.blocks + jb.blocks + jb2.blocks), dim3(256), 0, stream>>>(ja, jb, jb2, g.K);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const SplitPlan p = plan_split(g.M, columns(g, FORM), g.K);
    g.k_per = p.k_per;
    g.part = p.splits > 1 ? (float *)w : nullptr;
    const dim3 grid(p.tiles_m * p.tiles_n * (uint32_t)p.splits);
    if (p.rows == 256)
        gemm_split_kernel<FORM, 256, 256, 2, 4>
            <<<grid, dim3(512), 0, stream>>>(g, a, b, b2, p.tiles_m, p.tiles_n);
    else if (p.rows == 192)
        gemm_split_kernel<FORM, 192, 256, 2, 4>
            <<<grid, dim3(512), 0, stream>>>(g, a, b, b2, p.tiles_m, p.tiles_n);
    else
        gemm_split_kernel<FORM, 128, 128, 2, 2>
            <<<grid, dim3(256), 0, stream>>>(g, a, b, b2, p.tiles_m, p.tiles_n);
    e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    return launch_split_sum<float, FORM>(g, p.splits, stream);
}

uint64_t bytes_of(const GemmArgs &g, Form form)
{
    const int64_t n = columns(g, form);
    if (!splits_first(g.M, n, g.K)) return gemm_bytes(g.M, n, g.K);
    const SplitPlan p = plan_split(g.M, n, g.K);
    auto up = [](uint64_t v) { return (v + 1023) / 1024 * 1024; };
    return up(split_bytes(g.M, g.K)) + (form == GATED ? 2 : 1) * up(split_bytes(g.N, g.K)) +
           (p.splits > 1 ? (uint64_t)p.splits * g.M * n * 4 : 0);
}

}  // namespace

uint64_t gemm_f32_bytes(const GemmArgs &g) { return bytes_of(g, PLAIN); }

hipError_t gemm_f32(const GemmArgs &g, Layout la, Layout lb, void *ws, hipStream_t stream)
{
    if (splits_first(g.M, g.N, g.K)) return run_split<PLAIN>(g, la, lb, ws, stream);
    float *w = (float *)ws;
    if (la == K_CONTIGUOUS && lb == K_STRIDED)
        return run_gemm<K_CONTIGUOUS, K_STRIDED>(g, w, stream);
    if (la == K_CONTIGUOUS) return run_gemm<K_CONTIGUOUS, K_CONTIGUOUS>(g, w, stream);
    return run_gemm<K_STRIDED, K_STRIDED>(g, w, stream);
}

uint64_t gemm_f32_bytes(const GemmArgs &g, Form form) { return bytes_of(g, form); }

hipError_t gemm_f32(const GemmArgs &g, Form form, void *ws, hipStream_t stream)
{
    const bool first = splits_first(g.M, columns(g, form), g.K);
    if (form == GATED)
        return first ? run_split<GATED>(g, K_CONTIGUOUS, K_STRIDED, ws, stream)
                     : run_gemm<K_CONTIGUOUS, K_STRIDED, GATED>(g, (float *)ws, stream);
    return first ? run_split<HALVES>(g, K_STRIDED, K_STRIDED, ws, stream)
                 : run_gemm<K_STRIDED, K_STRIDED, HALVES>(g, (float *)ws, stream);
}

}  // namespace whtmix
