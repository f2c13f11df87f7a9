// Rows of a table by token ids, and the table's gradient by sorted tokens.
//
//   y[n] = scale table[id_n]                       (id < 0: zeros; id >= vocab: NaN)
//   dtable[v] = scale sum over n with id_n = v of dy[n]
//
// The gradient sorts (id, n) pairs, stable, by radix: equal ids then lie together in ascending n.
// Each run of them is summed in float32 in that order, stretch by stretch, without atomics on
// values, so results do not change from run to run.  Runs may be of one token or of all of them, so
// the sorted list is cut into ranges of equal length: a workgroup adds what its range holds,
// writes the runs that lie in it, and leaves the sums of the others to be joined in order by a
// kernel of its own.
//
// Bound by memory where tokens are many: 65536 x 1024 bf16 of a table of 50000 rows 37 us forward (268 MB,
// table rows that come often out of the caches), and backward 61 us of sums, 25 of sorting in
// two passes and 6 of joining.  17 rows 2.6 us: the latency of an id and then a row.
#include "whtmix_row.h"

#include <algorithm>

namespace whtmix {
namespace {

// ---- forward ----
struct EmbeddingKernelArgs {
    const void *ids, *table;
    void *y;
    int64_t rows, vocab, C;
    float scale;
    int lanes_log2;         // lanes a row
};

// U rows a group of lanes at a time, whose ids and then rows are in flight together; workgroups
// of the grid's second dimension take the columns past the lanes'.
template <typename T, typename Id, int U>
__global__ void __launch_bounds__(256) embedding_kernel(EmbeddingKernelArgs a)
{
    constexpr int N = Chunk<T>::N;
    const int groups = 256 >> a.lanes_log2;
    const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1), grp = threadIdx.x >> a.lanes_log2;
    const int64_t c = (((int64_t)blockIdx.y << a.lanes_log2) + lane) * N;
    const int n = (int)min((int64_t)N, a.C - c);
    if (n <= 0) return;
    for (int64_t base = (int64_t)blockIdx.x * (groups * U) + grp; base < a.rows;
         base += (int64_t)gridDim.x * (groups * U)) {
        int64_t id[U];
        float v[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = base + u * groups;
            id[u] = row < a.rows ? (int64_t)((const Id *)a.ids)[row] : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool real = (uint64_t)id[u] < (uint64_t)a.vocab;
            load_row<T>((const T *)a.table + (real ? id[u] * a.C + c : 0), real ? n : 0, v[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = base + u * groups;
            if (row >= a.rows) break;
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[u][i] = id[u] < a.vocab ? v[u][i] * a.scale : bits_f32(0x7fc00000u);
            if (id[u] < 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) v[u][i] = 0.f;
            }
            store_row<T>((T *)a.y + row * a.C + c, n, v[u]);
        }
    }
}

int log2_up(int64_t v, int most)
{
    int l = 0;
    while (l < most && (int64_t(1) << l) < v) ++l;
    return l;
}

template <typename T, typename Id> hipError_t forward(const EmbeddingArgs &a)
{
    const int64_t chunks = (a.C + Chunk<T>::N - 1) / Chunk<T>::N;
    const int l = log2_up(chunks, 8), groups = 256 >> l;
    const EmbeddingKernelArgs k{a.ids, a.table, a.y, a.rows, a.vocab, a.C, a.scale, l};
    const uint32_t across = (uint32_t)((chunks + (1 << l) - 1) >> l);
    auto blocks = [&](int U) {
        return (uint32_t)std::min<int64_t>((a.rows + groups * U - 1) / (groups * U),
                                           kMaxBlocks / across);
    };
    if (blocks(4) * across >= 1024)
        embedding_kernel<T, Id, 4><<<dim3(blocks(4), across), dim3(256), 0, a.stream>>>(k);
    else
        embedding_kernel<T, Id, 1><<<dim3(blocks(1), across), dim3(256), 0, a.stream>>>(k);
    return hipGetLastError();
}

// ---- the sort ----
// Pairs of (key, n), the key an id of the table or `vocab` for tokens that have no gradient, which
// come last.  Digits of up to 9 bits: byte tokens and their padding are sorted in one pass.
constexpr int kBins = 512, kDigitBits = 9;
constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64, kItems = 4;
constexpr int kTile = kSortThreads * kItems;

struct SortArgs {
    const void *ids;        // of the first pass
    const uint32_t *keys, *at;      // of the others
    uint32_t *keys_out, *at_out;
    uint32_t *counts;       // [tiles][kBins], then [kBins] totals where a scan made them
    int64_t rows, vocab;
    uint32_t tiles;
    int shift, bits;
    bool scanned;           // counts hold the sums over the tiles before
};

template <typename Id> __device__ __forceinline__ uint32_t key_of(const SortArgs &a, int64_t i)
{
    const uint64_t id = (uint64_t)(int64_t)((const Id *)a.ids)[i];
    return id < (uint64_t)a.vocab ? (uint32_t)id : (uint32_t)a.vocab;
}

// Item j of the thread: tiles in order, a tile's waves in order, 64 neighbours at a time.
__device__ __forceinline__ int64_t item(int64_t tile, int j)
{
    return tile * kTile + (threadIdx.x >> 6) * (64 * kItems) + j * 64 + (threadIdx.x & 63);
}

__device__ __forceinline__ void wave_fence()     // orders a wave's own LDS accesses
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// How often each digit comes in a tile (a count: the order of the additions does not matter).
template <typename Id, bool FIRST>
__global__ void __launch_bounds__(kSortThreads) count_kernel(SortArgs a)
{
    __shared__ uint32_t count[kBins];
    count[threadIdx.x] = 0;
    __syncthreads();
    uint32_t key[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const int64_t i = item(blockIdx.x, j);
        key[j] = i < a.rows ? (FIRST ? key_of<Id>(a, i) : a.keys[i]) : 0;
    }
#pragma unroll
    for (int j = 0; j < kItems; ++j)
        if (item(blockIdx.x, j) < a.rows)
            atomicAdd(&count[(key[j] >> a.shift) & ((1u << a.bits) - 1)], 1u);
    __syncthreads();
    a.counts[(int64_t)blockIdx.x * kBins + threadIdx.x] = count[threadIdx.x];
}

// Counts -> sums over the tiles before, and the totals: 32 digits a workgroup, its threads in 32
// parts of the tiles.
__global__ void __launch_bounds__(1024) scan_kernel(uint32_t *counts, uint32_t tiles)
{
    __shared__ uint32_t sums[32][33];
    const int d = threadIdx.x & 31, part = threadIdx.x >> 5;
    uint32_t *mine = counts + blockIdx.x * 32 + d;
    const uint32_t per = (tiles + 31) / 32, from = min(tiles, part * per),
                   to = min(tiles, from + per);
    uint32_t s = 0;
    for (uint32_t t = from; t < to; t += 8) {
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) s += t + u < to ? mine[(uint64_t)(t + u) * kBins] : 0;
    }
    sums[part][d] = s;
    __syncthreads();
    uint32_t before = 0;
    for (int p = 0; p < part; ++p) before += sums[p][d];
    if (part == 31) mine[(uint64_t)tiles * kBins] = before + s;
    for (uint32_t t = from; t < to; t += 8) {
        uint32_t v[8];
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) v[u] = t + u < to ? mine[(uint64_t)(t + u) * kBins] : 0;
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) {
            if (t + u < to) mine[(uint64_t)(t + u) * kBins] = before;
            before += v[u];
        }
    }
}

// LDS of a workgroup that puts a tile's items in order.
struct SortLds {
    uint32_t count[kSortWaves][kBins];
    uint32_t waves[kSortWaves];
};

// The items' ranks among those of their digit in the wave, and in lds.count how many there are.
template <int ITEMS>
__device__ __forceinline__ void rank_items(SortLds &lds, const uint32_t (&key)[ITEMS],
                                           const bool (&in)[ITEMS], int shift, int bits,
                                           uint32_t (&digit)[ITEMS], uint32_t (&rank)[ITEMS])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t *count = lds.count[wave];
#pragma unroll
    for (int i = 0; i < kBins / 64; ++i) count[i * 64 + lane] = 0;
    wave_fence();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        digit[j] = (key[j] >> shift) & ((1u << bits) - 1);
        // The lanes with the same digit.
        uint64_t same = __ballot(in[j]);
        for (int b = 0; b < bits; ++b) {
            const bool set = digit[j] >> b & 1;
            const uint64_t with = __ballot(set);
            same &= set ? with : ~with;
        }
        const uint32_t before = (uint32_t)__popcll(same & ((uint64_t(1) << lane) - 1));
        const uint32_t had = in[j] ? count[digit[j]] : 0;
        rank[j] = had + before;
        wave_fence();
        if (in[j] && before == 0) count[digit[j]] = had + (uint32_t)__popcll(same);
        wave_fence();
    }
}

// The sum of v over the threads before this one (kBins of them).
__device__ __forceinline__ uint32_t sum_before(SortLds &lds, uint32_t v)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)s, d);
        if (lane >= d) s += o;
    }
    if (lane == 63) lds.waves[wave] = s;
    __syncthreads();
    uint32_t before = s - v;
    for (int w = 0; w < wave; ++w) before += lds.waves[w];
    __syncthreads();
    return before;
}

static_assert(kBins == kSortThreads, "a thread takes a digit");

// Where the tile's items of each wave and digit start: `start` is where the tile's of digit
// threadIdx.x do.
__device__ __forceinline__ void wave_starts(SortLds &lds, uint32_t start)
{
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t n = lds.count[w][threadIdx.x];
        lds.count[w][threadIdx.x] = start;
        start += n;
    }
    __syncthreads();
}

template <typename Id, bool FIRST>
__global__ void __launch_bounds__(kSortThreads) scatter_kernel(SortArgs a)
{
    __shared__ SortLds lds;
    uint32_t key[kItems], at[kItems], digit[kItems], rank[kItems];
    bool in[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const int64_t i = item(blockIdx.x, j);
        in[j] = i < a.rows;
        key[j] = in[j] ? (FIRST ? key_of<Id>(a, i) : a.keys[i]) : 0;
        at[j] = FIRST ? (uint32_t)i : in[j] ? a.at[i] : 0;
    }
    // The digit's items in the tiles before, and in all.
    uint32_t before = 0, all = 0;
    if (a.scanned) {
        before = a.counts[(int64_t)blockIdx.x * kBins + threadIdx.x];
        all = a.counts[(int64_t)a.tiles * kBins + threadIdx.x];
    } else {
        for (uint32_t t = 0; t < a.tiles; t += 32) {
            uint32_t v[32];
#pragma unroll
            for (uint32_t u = 0; u < 32; ++u)
                v[u] = t + u < a.tiles ? a.counts[(int64_t)(t + u) * kBins + threadIdx.x] : 0;
#pragma unroll
            for (uint32_t u = 0; u < 32; ++u) {
                before += t + u < blockIdx.x ? v[u] : 0;
                all += v[u];
            }
        }
    }
    rank_items(lds, key, in, a.shift, a.bits, digit, rank);
    const uint32_t start = sum_before(lds, all) + before;
    wave_starts(lds, start);
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        if (!in[j]) continue;
        const uint32_t to = lds.count[threadIdx.x >> 6][digit[j]] + rank[j];
        a.keys_out[to] = key[j];
        a.at_out[to] = at[j];
    }
}

// All passes of up to kTile tokens in one workgroup.
template <typename Id>
__global__ void __launch_bounds__(kSortThreads) sort_tile_kernel(SortArgs a, int passes)
{
    __shared__ SortLds lds;
    __shared__ uint32_t keys[kTile], ats[kTile];
    uint32_t key[kItems], at[kItems], digit[kItems], rank[kItems];
    bool in[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const int64_t i = item(0, j);
        in[j] = i < a.rows;
        key[j] = in[j] ? key_of<Id>(a, i) : 0;
        at[j] = (uint32_t)i;
    }
    for (int p = 0; p < passes; ++p) {
        rank_items(lds, key, in, p * a.bits, a.bits, digit, rank);
        __syncthreads();
        uint32_t all = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) all += lds.count[w][threadIdx.x];
        const uint32_t start = sum_before(lds, all);
        wave_starts(lds, start);
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            if (!in[j]) continue;
            const uint32_t to = lds.count[threadIdx.x >> 6][digit[j]] + rank[j];
            keys[to] = key[j];
            ats[to] = at[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            const int i = (int)item(0, j);
            key[j] = in[j] ? keys[i] : 0;
            at[j] = in[j] ? ats[i] : 0;
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        if (!in[j]) continue;
        a.keys_out[item(0, j)] = key[j];
        a.at_out[item(0, j)] = at[j];
    }
}

// ---- the sums ----
struct SumArgs {
    const uint32_t *keys, *at;      // sorted
    const void *dy;
    void *dtable;
    float *part;            // [ranges][2][C]: of the run a range goes on with, of the one it leaves
    int64_t rows, vocab, C, ranges;
    int stretch, range;     // tokens of a group of lanes, of a workgroup's groups together
    int lanes_log2;
    uint32_t slices;        // groups of columns
    uint32_t sum_blocks;    // workgroups that sum; the others write the zeros
    float scale;
};

constexpr int kZeroRows = 16;       // rows of the table a wave looks after

// Zeros to the rows of the table that no token names: a lane looks for one in the sorted keys.
template <typename T> __device__ __forceinline__ void zero_rows(const SumArgs &a, int64_t first)
{
    const int lane = threadIdx.x & 63;
    const int64_t v = first + (lane & (kZeroRows - 1));
    int64_t lo = 0, hi = a.rows;        // the first key of v or above
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if ((int64_t)a.keys[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    const bool none = v < a.vocab && (lo == a.rows || (int64_t)a.keys[lo] != v);
    const uint32_t rows = (uint32_t)__ballot(none) & ((1u << kZeroRows) - 1);
    if (rows == 0) return;
    constexpr int N = Chunk<T>::N;
    const int64_t chunks = (a.C + N - 1) / N;
    const float zero[N] = {};
    T *to = (T *)a.dtable + first * a.C;
    for (int r = 0; r < kZeroRows; ++r) {
        if (!(rows >> r & 1)) continue;
        for (int64_t k = lane; k < chunks; k += 64)
            store_row<T>(to + r * a.C + k * N, (int)min((int64_t)N, a.C - k * N), zero);
    }
}

// LDS of a workgroup whose groups of lanes take neighbouring stretches of a sorted list.
template <int N, int THREADS> struct StretchLds {
    float first[THREADS * N], last[THREADS * N];    // sums of a stretch's first, last run
    uint8_t state[THREADS];
};

// Sums the runs of equal keys in the list's entries [begin, end), of `size` in all; entry i has
// key_of(i) and the row row_of(i), whose chunk of columns load() brings.  A run that lies in the
// range goes to write(key, s); the sums of one that comes from before it or goes on behind it to
// left(which, key, s), which = 0 or 1.  Each group of lanes takes `stretch` entries; what goes on
// from one to the next is joined in order through LDS.
template <typename T, int THREADS, typename Key, typename Row, typename Load, typename Write,
          typename Left>
__device__ __forceinline__ void sum_runs(StretchLds<Chunk<T>::N, THREADS> &lds, int64_t begin,
                                         int64_t end, int64_t size, int stretch, int lanes_log2,
                                         Key key_of, Row row_of, Load load, Write write, Left left)
{
    constexpr int N = Chunk<T>::N, U = 8;
    enum { BEFORE = 1, AFTER = 2, WHOLE = 4 };      // of the runs that are left there
    const int groups = THREADS >> lanes_log2;
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1), grp = threadIdx.x >> lanes_log2;
    const int64_t i0 = begin + (int64_t)grp * stretch, i1 = min(end, i0 + stretch);
    auto keep = [&](float *to, const float (&s)[N]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < N; ++k) to[threadIdx.x * N + k] = s[k];
    };
    int mine = 0;
    uint32_t key = 0, key0 = 0;
    float s[N];
    if (i0 < end) {
        key = key0 = key_of(i0);
        bool before = i0 > 0 && key_of(i0 - 1) == key;
        const bool after = i1 < size && key_of(i1) == key_of(i1 - 1);
        if (before) mine = BEFORE;
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] = 0.f;
        for (int64_t i = i0; i < i1; i += U) {
            uint32_t ku[U], row[U];
            RawChunk<T> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                ku[u] = key_of(min(i + u, i1 - 1));
                row[u] = row_of(min(i + u, i1 - 1));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) load(row[u], i + u < i1, ku[u], v[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (ku[u] != key) {
                    if (before) keep(lds.first, s);
                    else write(key, s);
                    before = false;
                    key = ku[u];
#pragma unroll
                    for (int k = 0; k < N; ++k) s[k] = 0.f;
                }
#pragma unroll
                for (int k = 0; k < N; ++k) s[k] += v[u][k];
            }
        }
        if (before) {
            keep(lds.first, s);
            if (after) mine |= WHOLE;
        } else if (after) {
            keep(lds.last, s);
            mine |= AFTER;
        } else {
            write(key, s);
        }
    }
    lds.state[threadIdx.x] = (uint8_t)mine;
    __syncthreads();
    // A run from `s` on through the stretches that follow: whether it goes on past the range.
    auto join = [&](bool on) __attribute__((always_inline)) {
        for (int q = grp + 1; on && q < groups; ++q) {
            const int t = (q << lanes_log2) + lane;
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] += lds.first[t * N + k];
            on = lds.state[t] & WHOLE;
        }
        return on;
    };
    if (grp == 0 && (mine & BEFORE)) {
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] = lds.first[threadIdx.x * N + k];
        join(mine & WHOLE);
        left(0, key0, s);
    }
    if (mine & AFTER) {
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] = lds.last[threadIdx.x * N + k];
        if (join(true)) left(1, key, s);
        else write(key, s);
    }
}

template <typename T> __global__ void __launch_bounds__(256) sum_kernel(SumArgs a)
{
    constexpr int N = Chunk<T>::N;
    __shared__ StretchLds<N, 256> lds;
    if (blockIdx.x >= a.sum_blocks) {
        const int64_t step = (int64_t)(gridDim.x - a.sum_blocks) * 4 * kZeroRows;
        for (int64_t v = ((int64_t)(blockIdx.x - a.sum_blocks) * 4 + (threadIdx.x >> 6)) * kZeroRows;
             v < a.vocab; v += step)
            zero_rows<T>(a, v);
        return;
    }
    const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1);
    const int64_t r = blockIdx.x / a.slices;
    const int64_t c = (((int64_t)(blockIdx.x % a.slices) << a.lanes_log2) + lane) * N;
    const int n = (int)max((int64_t)0, min((int64_t)N, a.C - c));
    const T *dy = (const T *)a.dy + (n ? c : 0);
    float *part = a.part + 2 * r * a.C + c;
    sum_runs<T, 256>(
        lds, r * a.range, min(a.rows, (r + 1) * a.range), a.rows, a.stretch, a.lanes_log2,
        [&](int64_t i) __attribute__((always_inline)) { return a.keys[i]; },
        [&](int64_t i) __attribute__((always_inline)) { return a.at[i]; },
        [&](uint32_t row, bool in, uint32_t key, RawChunk<T> &v) __attribute__((always_inline)) {
            v.load(dy + (int64_t)row * a.C, in && key < (uint64_t)a.vocab ? n : 0);
        },
        [&](uint32_t key, float (&s)[N]) __attribute__((always_inline)) {
            if (key >= (uint64_t)a.vocab || n == 0) return;
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] *= a.scale;
            store_row<T>((T *)a.dtable + (int64_t)key * a.C + c, n, s);
        },
        [&](int which, uint32_t key, float (&s)[N]) __attribute__((always_inline)) {
            if (key < (uint64_t)a.vocab) store_floats(part + which * a.C, n, s);
        });
}

// The runs that go over several ranges: the workgroup of the range in which one starts adds its
// parts, each group of lanes a stretch of them, then the stretches in order.
template <typename T> __global__ void __launch_bounds__(256) join_kernel(SumArgs a)
{
    constexpr int N = Chunk<T>::N, U = 8;
    __shared__ float sums[256 * N];
    const int64_t r = blockIdx.x / a.slices;
    const int64_t i0 = r * a.range, i1 = i0 + a.range;
    if (i1 >= a.rows) return;
    const uint32_t key = a.keys[i1];
    if (key >= (uint64_t)a.vocab || a.keys[i1 - 1] != key) return;
    if (i0 > 0 && a.keys[i0 - 1] == key) return;
    // Ranges after this one that go on with the run.
    int64_t more = 0;
    for (;;) {
        const int64_t q = r + 1 + more + threadIdx.x;
        const int count = __syncthreads_count(q < a.ranges && a.keys[min(q, a.ranges - 1) * a.range] == key);
        more += count;
        if (count < 256) break;
    }
    const int groups = 256 >> a.lanes_log2;
    const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1), grp = threadIdx.x >> a.lanes_log2;
    const int64_t c = (((int64_t)(blockIdx.x % a.slices) << a.lanes_log2) + lane) * N;
    const int n = (int)max((int64_t)0, min((int64_t)N, a.C - c));
    const int64_t per = (more + groups) / groups;          // of more + 1 parts
    const int64_t from = grp * per, to = min(more + 1, from + per);
    float s[N];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = 0.f;
    for (int64_t i = from; i < to; i += U) {
        float v[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t j = min(i + u, to - 1);
            load_floats(a.part + ((r + j) * 2 + (j == 0 ? 1 : 0)) * a.C + (n ? c : 0),
                        i + u < to ? n : 0, v[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] += v[u][k];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) sums[threadIdx.x * N + k] = s[k];
    __syncthreads();
    if (grp > 0 || n == 0) return;
    for (int g = 1; g < groups; ++g)
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] += sums[((g << a.lanes_log2) + lane) * N + k];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] *= a.scale;
    store_row<T>((T *)a.dtable + (int64_t)key * a.C + c, n, s);
}

// ---- few ids ----
// A vocabulary of a digit's size (byte tokens): a workgroup sorts its own tokens in LDS and writes
// the sums of each id's to memory, one row of C floats an id; a second kernel adds those of an
// id in order.  Two launches in place of four (131072 x 64 float32 of 256 ids: 15 + 4 us).
struct FewArgs {
    const void *ids, *dy;
    void *dtable;
    float *part;            // [tiles][vocab][C]
    uint32_t *counts;       // [tiles][vocab]: how many tokens of the tile have the id
    int64_t rows, C;
    int vocab, bits, stretch, lanes_log2;
    uint32_t tiles;
    float scale;
};

constexpr int kFewItems = 2, kFewTile = kSortThreads * kFewItems;

template <typename T, typename Id>
__global__ void __launch_bounds__(kSortThreads) few_ids_kernel(FewArgs a)
{
    constexpr int N = Chunk<T>::N;
    __shared__ SortLds lds;
    __shared__ StretchLds<N, kSortThreads> runs;
    __shared__ uint16_t keys[kFewTile], ats[kFewTile];
    const int64_t base = (int64_t)blockIdx.x * kFewTile;
    const int size = (int)min((int64_t)kFewTile, a.rows - base);
    uint32_t key[kFewItems], digit[kFewItems], rank[kFewItems];
    int at[kFewItems];
    bool in[kFewItems];
#pragma unroll
    for (int j = 0; j < kFewItems; ++j) {
        at[j] = (int)(threadIdx.x >> 6) * (64 * kFewItems) + j * 64 + (int)(threadIdx.x & 63);
        in[j] = at[j] < size;
        const uint64_t id = in[j] ? (uint64_t)(int64_t)((const Id *)a.ids)[base + at[j]] : 0;
        key[j] = id < (uint64_t)a.vocab ? (uint32_t)id : (uint32_t)a.vocab;
    }
    rank_items(lds, key, in, 0, a.bits, digit, rank);
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) all += lds.count[w][threadIdx.x];
    if ((int)threadIdx.x < a.vocab) a.counts[(int64_t)blockIdx.x * a.vocab + threadIdx.x] = all;
    wave_starts(lds, sum_before(lds, all));
#pragma unroll
    for (int j = 0; j < kFewItems; ++j) {
        if (!in[j]) continue;
        const uint32_t to = lds.count[threadIdx.x >> 6][digit[j]] + rank[j];
        keys[to] = (uint16_t)key[j];
        ats[to] = (uint16_t)at[j];
    }
    __syncthreads();
    const int64_t c = (threadIdx.x & ((1 << a.lanes_log2) - 1)) * N;
    const int n = (int)max((int64_t)0, min((int64_t)N, a.C - c));
    const T *dy = (const T *)a.dy + base * a.C + (n ? c : 0);
    float *part = a.part + (int64_t)blockIdx.x * a.vocab * a.C + c;
    sum_runs<T, kSortThreads>(
        runs, 0, size, size, a.stretch, a.lanes_log2,
        [&](int64_t i) __attribute__((always_inline)) { return (uint32_t)keys[i]; },
        [&](int64_t i) __attribute__((always_inline)) { return (uint32_t)ats[i]; },
        [&](uint32_t row, bool in, uint32_t key, RawChunk<T> &v) __attribute__((always_inline)) {
            v.load(dy + (int64_t)row * a.C, in && (int)key < a.vocab ? n : 0);
        },
        [&](uint32_t key, float (&s)[N]) __attribute__((always_inline)) {
            if ((int)key < a.vocab) store_floats(part + (int64_t)key * a.C, n, s);
        },
        [](int, uint32_t, float (&)[N]) __attribute__((always_inline)) {});    // no run leaves a tile
}

// A chunk's sums over the tiles: the workgroup's groups of lanes take stretches of them.
template <typename T> __global__ void __launch_bounds__(256) few_ids_join_kernel(FewArgs a)
{
    constexpr int N = Chunk<T>::N, U = 8;
    __shared__ float sums[256 * N];
    const int groups = 256 >> a.lanes_log2;
    const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1), grp = threadIdx.x >> a.lanes_log2;
    const int64_t v = blockIdx.x, c = (int64_t)lane * N;
    const int n = (int)max((int64_t)0, min((int64_t)N, a.C - c));
    const uint32_t per = (a.tiles + groups - 1) / groups;
    const uint32_t from = min(a.tiles, grp * per), to = min(a.tiles, from + per);
    float s[N];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = 0.f;
    for (uint32_t t = from; t < to; t += U) {
        uint32_t some[U];
        float p[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t q = min(t + u, to - 1);
            some[u] = a.counts[(int64_t)q * a.vocab + v];
            load_floats(a.part + ((int64_t)q * a.vocab + v) * a.C + (n ? c : 0),
                        t + u < to ? n : 0, p[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] += some[u] ? p[u][k] : 0.f;    // else never written
    }
#pragma unroll
    for (int k = 0; k < N; ++k) sums[threadIdx.x * N + k] = s[k];
    __syncthreads();
    if (grp > 0 || n == 0) return;
    for (int g = 1; g < groups; ++g)
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] += sums[((g << a.lanes_log2) + lane) * N + k];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] *= a.scale;
    store_row<T>((T *)a.dtable + v * a.C + c, n, s);
}

struct Plan {
    bool few;
    int bits, passes;       // of a digit; of the sort
    int64_t tiles;
    int stretch, range, lanes_log2;
    int64_t ranges, slices;
    uint64_t pairs, counts, part;   // bytes: one of four arrays; counts; partial sums
    bool scan;
};

uint64_t up256(uint64_t v) { return (v + 255) / 256 * 256; }

Plan make_plan(int64_t rows, int64_t vocab, int64_t C, int dtype)
{
    Plan p{};
    const int bits = std::max(1, log2_up(vocab + 1, 31));       // of the keys 0 .. vocab
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tiles = (rows + kTile - 1) / kTile;
    p.scan = p.tiles > 128;
    const int per = dtype == DTYPE_BF16 ? 8 : 4;
    const int64_t chunks = (C + per - 1) / per;
    p.lanes_log2 = log2_up(chunks, 6);
    // Ids of one digit, where the tiles' sums are few: a tile's time goes by C and by the ids (us so
    // and by the whole sort, 16384 tokens: C = 64, 256 ids, float32 15.5 and 19.7; C = 128, 256 ids,
    // bf16 20.0 and 21.2; C = 128, 500 ids 24.0 and 20.6; C = 256, 256 ids 26.6 and 20.6; 262144
    // tokens, C = 64, 256 ids, float32 24 and 38).  24 MiB of sums are the most a caller is told of.
    // Lists that one workgroup sorts are quick (1000 tokens, bf16: C = 128, 256 ids 20.3 and 15.4, C =
    // 8 21.0 and 9.9, C = 32 14.2 and 17.1; 300 tokens, C = 64 12.5 and 15.4).
    const int64_t few_tiles = (rows + kFewTile - 1) / kFewTile;
    const uint64_t few_part = (uint64_t)few_tiles * vocab * C * 4;
    if (vocab < kBins && C <= 128 && vocab * C <= 1 << 15 && few_part <= uint64_t(24) << 20 &&
        (rows > kTile || (C >= 32 && C <= 64))) {
        p.few = true;
        p.tiles = few_tiles;
        const int64_t groups = kSortThreads >> p.lanes_log2;
        p.stretch = (int)((std::min<int64_t>(rows, kFewTile) + groups - 1) / groups);
        p.counts = up256((uint64_t)few_tiles * vocab * 4);
        p.part = few_part;
        return p;
    }
    p.slices = (chunks + (1 << p.lanes_log2) - 1) >> p.lanes_log2;
    // Stretches for 2^18 lanes, of 8 to 256 tokens (194910 x 240 bf16: 64 us, 74 for half as many lanes
    // and 70 for twice as many; 65536 x 1024: 62, 66 and 65).
    p.stretch = 1 << (3 + log2_up(rows * chunks >> 21, 5));
    p.range = p.stretch * (256 >> p.lanes_log2);
    p.ranges = (rows + p.range - 1) / p.range;
    p.pairs = up256((uint64_t)rows * 4);
    p.counts = up256((uint64_t)(p.tiles + 1) * kBins * 4);
    p.part = (uint64_t)p.ranges * 2 * C * 4;
    return p;
}

template <typename Id>
hipError_t sort(const EmbeddingBackwardArgs &a, const Plan &p, char *ws, const uint32_t *&keys,
                const uint32_t *&at)
{
    uint32_t *k[2] = {(uint32_t *)ws, (uint32_t *)(ws + 2 * p.pairs)};
    uint32_t *n[2] = {(uint32_t *)(ws + p.pairs), (uint32_t *)(ws + 3 * p.pairs)};
    SortArgs s{};
    s.ids = a.ids, s.rows = a.rows, s.vocab = a.vocab;
    s.counts = (uint32_t *)(ws + 4 * p.pairs);
    s.tiles = (uint32_t)p.tiles, s.bits = p.bits, s.scanned = p.scan;
    keys = k[0], at = n[0];
    if (p.tiles == 1) {
        s.keys_out = k[0], s.at_out = n[0];
        sort_tile_kernel<Id><<<dim3(1), dim3(kSortThreads), 0, a.stream>>>(s, p.passes);
        return hipGetLastError();
    }
    for (int i = 0; i < p.passes; ++i) {
        s.shift = i * p.bits;
        s.keys_out = k[i & 1], s.at_out = n[i & 1];
        s.keys = k[(i & 1) ^ 1], s.at = n[(i & 1) ^ 1];
        const dim3 grid((uint32_t)p.tiles), block(kSortThreads);
        if (i == 0) count_kernel<Id, true><<<grid, block, 0, a.stream>>>(s);
        else count_kernel<Id, false><<<grid, block, 0, a.stream>>>(s);
        if (p.scan)
            scan_kernel<<<dim3(kBins / 32), dim3(1024), 0, a.stream>>>(s.counts, s.tiles);
        if (i == 0) scatter_kernel<Id, true><<<grid, block, 0, a.stream>>>(s);
        else scatter_kernel<Id, false><<<grid, block, 0, a.stream>>>(s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        keys = s.keys_out, at = s.at_out;
    }
    return hipSuccess;
}

template <typename T> hipError_t backward_few(const EmbeddingBackwardArgs &a, const Plan &p)
{
    FewArgs f{};
    f.ids = a.ids, f.dy = a.dy, f.dtable = a.dtable;
    f.counts = (uint32_t *)a.ws, f.part = (float *)((char *)a.ws + p.counts);
    f.rows = a.rows, f.C = a.C, f.vocab = (int)a.vocab, f.bits = p.bits, f.stretch = p.stretch;
    f.lanes_log2 = p.lanes_log2, f.tiles = (uint32_t)p.tiles, f.scale = a.scale;
    const dim3 grid((uint32_t)p.tiles), block(kSortThreads);
    if (a.wide_ids) few_ids_kernel<T, int64_t><<<grid, block, 0, a.stream>>>(f);
    else few_ids_kernel<T, int32_t><<<grid, block, 0, a.stream>>>(f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    few_ids_join_kernel<T><<<dim3((uint32_t)a.vocab), dim3(256), 0, a.stream>>>(f);
    return hipGetLastError();
}

template <typename T> hipError_t backward(const EmbeddingBackwardArgs &a)
{
    const Plan p = make_plan(a.rows, a.vocab, a.C, a.dtype);
    if (p.few) return backward_few<T>(a, p);
    char *ws = (char *)a.ws;
    SumArgs s{};
    hipError_t e = a.wide_ids ? sort<int64_t>(a, p, ws, s.keys, s.at)
                              : sort<int32_t>(a, p, ws, s.keys, s.at);
    if (e != hipSuccess) return e;
    s.dy = a.dy, s.dtable = a.dtable, s.part = (float *)(ws + 4 * p.pairs + p.counts);
    s.rows = a.rows, s.vocab = a.vocab, s.C = a.C;
    s.ranges = p.ranges, s.range = p.range, s.stretch = p.stretch;
    s.lanes_log2 = p.lanes_log2, s.slices = (uint32_t)p.slices, s.scale = a.scale;
    s.sum_blocks = (uint32_t)(p.ranges * p.slices);
    const int64_t zeros = std::min<int64_t>((a.vocab + 4 * kZeroRows - 1) / (4 * kZeroRows), 1 << 20);
    sum_kernel<T><<<dim3(s.sum_blocks + (uint32_t)zeros), dim3(256), 0, a.stream>>>(s);
    if ((e = hipGetLastError()) != hipSuccess || p.ranges < 2) return e;
    join_kernel<T><<<dim3((uint32_t)((p.ranges - 1) * p.slices)), dim3(256), 0, a.stream>>>(s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(const EmbeddingArgs &a)
{
    if (a.dtype == DTYPE_BF16)
        return a.wide_ids ? forward<__bf16, int64_t>(a) : forward<__bf16, int32_t>(a);
    return a.wide_ids ? forward<float, int64_t>(a) : forward<float, int32_t>(a);
}

uint64_t embedding_backward_bytes(int64_t rows, int64_t vocab, int64_t C, int dtype)
{
    const Plan p = make_plan(rows, vocab, C, dtype);
    return 4 * p.pairs + p.counts + p.part;
}

hipError_t launch_embedding_backward(const EmbeddingBackwardArgs &a)
{
    return a.dtype == DTYPE_BF16 ? backward<__bf16>(a) : backward<float>(a);
}

}  // namespace whtmix
