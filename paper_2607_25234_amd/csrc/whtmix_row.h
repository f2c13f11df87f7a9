// Device helpers of the kernels that hold a row in the registers of G lanes: sums over them, and
// the row's chunks in block-scaled 8 bits.
#pragma once

#include "whtmix_vec.h"

namespace whtmix {

// The value of the lane `CTRL` (a DPP control) names.
template <int CTRL> __device__ __forceinline__ float lane_move(float v)
{
    return bits_f32((uint32_t)__builtin_amdgcn_update_dpp(0, (int)f32_bits(v), CTRL, 0xf, 0xf, true));
}

// Sum over groups of G neighbouring lanes of a wave (G a power of two), in every lane, by vector
// instructions alone: neighbours in a quad, then mirrored halves of 8 and of 16 (whose lanes hold
// equal sums by then), then the rows of 16 and the halves of the wave trade places.
template <int G> __device__ __forceinline__ float lane_sum(float v)
{
    static_assert(G >= 2 && G <= 64 && (G & (G - 1)) == 0, "a power of two of lanes");
    v += lane_move<0xB1>(v);
    if constexpr (G >= 4) v += lane_move<0x4E>(v);
    if constexpr (G >= 8) v += lane_move<0x141>(v);
    if constexpr (G >= 16) v += lane_move<0x140>(v);
    if constexpr (G >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(f32_bits(v), f32_bits(v), false, false);
        v = bits_f32((uint32_t)r[0]) + bits_f32((uint32_t)r[1]);
    }
    if constexpr (G >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
        v = bits_f32((uint32_t)r[0]) + bits_f32((uint32_t)r[1]);
    }
    return v;
}

// What two or three values' sums over a wave have in common: the halves (and rows of 16) of
// different values trade places, so that one register goes on with all of them.  fold_sums leaves in
// lane l one of 16 parts of the sum of value folded(l), unfold_sums gives all lanes each finished one.
// 5003 x 1111 float32, whose rows are four values a lane, forward and backward 33.9 us, 38.4 with
// each sum by itself.
template <int K> __device__ __forceinline__ float fold_sums(const float (&v)[K])
{
    static_assert(K == 2 || K == 3, "values");
    auto add32 = [](float a, float b) {     // a's sum in the lower half, b's in the upper
        const auto r = __builtin_amdgcn_permlane32_swap(f32_bits(a), f32_bits(b), false, false);
        return bits_f32((uint32_t)r[0]) + bits_f32((uint32_t)r[1]);
    };
    auto add16 = [](float a, float b) {     // of each half: a's in its lower row, b's in its upper
        const auto r = __builtin_amdgcn_permlane16_swap(f32_bits(a), f32_bits(b), false, false);
        return bits_f32((uint32_t)r[0]) + bits_f32((uint32_t)r[1]);
    };
    const float a = add32(v[0], v[1]);
    if constexpr (K == 2) return add16(a, a);
    else return add16(a, add32(v[2], v[2]));
}
template <int K> __device__ __forceinline__ int folded(int lane)
{
    return K == 3 && (lane & 16) ? 2 : lane >> 5;
}
template <int K> __device__ __forceinline__ void unfold_sums(float u, float (&v)[K])
{
    if constexpr (K == 3) {
        const auto r = __builtin_amdgcn_permlane16_swap(f32_bits(u), f32_bits(u), false, false);
        u = bits_f32((uint32_t)r[0]);
        v[2] = bits_f32((uint32_t)r[1]);
    }
    const auto r = __builtin_amdgcn_permlane32_swap(f32_bits(u), f32_bits(u), false, false);
    v[0] = bits_f32((uint32_t)r[0]);
    v[1] = bits_f32((uint32_t)r[1]);
}

// K sums over the G lanes that hold a row.  For rows wider than a wave `part` (LDS, K floats for
// each wave of the workgroup) is another one than in the call before, whose reads may
// still be under way.
template <int G, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float *part)
{
    if constexpr (G < 64) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = lane_sum<G>(v[k]);
    } else {
        float u = lane_sum<16>(fold_sums<K>(v));
        if constexpr (G > 64) {
            constexpr int W = G / 64, L = W <= 2 ? 2 : W <= 4 ? 4 : W <= 8 ? 8 : 16;
            const int lane = threadIdx.x & 63, i = lane & (L - 1);
            part += threadIdx.x / G * (W * K) + folded<K>(lane);
            if ((lane & 15) == 0) part[(threadIdx.x % G >> 6) * K] = u;
            __syncthreads();
            u = lane_sum<L>(i < W ? part[i * K] : 0.f);
        }
        unfold_sums<K>(u, v);
    }
}

// A chunk in 8 bits with its block's scale.  A block of 32 is 32 / N
// neighbouring lanes, all of which call this (chunks past C hold zeros).
template <typename T>
__device__ __forceinline__ void store_mx(const float (&v)[Chunk<T>::N], uint8_t *q,
                                         uint8_t *scales, int64_t c)
{
    constexpr int N = Chunk<T>::N;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, mx_magnitude(v[i]));
#pragma unroll
    for (int d = 1; d < kMxBlock / N; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    const uint32_t byte = mx_scale_byte(top);
    const float inv = mx_inverse(byte);
    uint32_t w[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
        w[i] = mx_pack(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], inv);
    __builtin_memcpy(__builtin_assume_aligned(q + c, N), w, N);
    if (c % kMxBlock == 0) scales[c / kMxBlock] = (uint8_t)byte;
}

// A chunk as it lies in memory: half the registers of bf16's floats, and bf16's last one of a row, of
// fewer elements, moved in at most three parts (of four elements, two and one) where element by
// element every wave of a ragged row would wait for seven (98779 x 91: 17 us, 22).
template <typename T> struct RawChunk {
    static constexpr int N = Chunk<T>::N;
    uint32_t u[4];
    // From memory; those past n are zeros.
    __device__ __forceinline__ void load(const T *p, int n)
    {
        if (n >= N) {
            __builtin_memcpy(u, p, 16);
        } else if constexpr (N == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = i < n ? f32_bits(p[i]) : 0u;
        } else {
            uint32_t four[2] = {0, 0}, two = 0;
            uint16_t one = 0;
            if (n & 4) __builtin_memcpy(four, p, 8);
            if (n & 2) __builtin_memcpy(&two, p + (n & 4), 4);
            if (n & 1) __builtin_memcpy(&one, p + (n & 6), 2);
            // the parts behind the first four elements, in order
            const uint32_t a = n & 2 ? two : (uint32_t)one, b = n & 2 ? (uint32_t)one : 0u;
            u[0] = n & 4 ? four[0] : a;
            u[1] = n & 4 ? four[1] : b;
            u[2] = n & 4 ? a : 0u;
            u[3] = n & 4 ? b : 0u;
        }
    }
    // The first n elements to memory.
    __device__ __forceinline__ void store(T *p, int n) const
    {
        if (n >= N) {
            __builtin_memcpy(p, u, 16);
        } else if constexpr (N == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) p[i] = bits_f32(u[i]);
        } else {
            if (n & 4) __builtin_memcpy(p, u, 8);
            const uint32_t a = n & 4 ? u[2] : u[0], b = n & 4 ? u[3] : u[1];
            if (n & 2) __builtin_memcpy(p + (n & 4), &a, 4);
            const uint16_t one = (uint16_t)(n & 2 ? b : a);
            if (n & 1) __builtin_memcpy(p + (n & 6), &one, 2);
        }
    }
    // Floats rounded to the type.
    __device__ __forceinline__ void pack(const float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (N == 4) u[i] = f32_bits(v[i]);
            else u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        }
    }
    // Element i (a constant after unrolling).
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (N == 4) return bits_f32(u[i]);
        else return bits_f32(i & 1 ? u[i >> 1] & 0xffff0000u : u[i >> 1] << 16);
    }
};

template <typename T>
__device__ __forceinline__ void load_row(const T *p, int n, float (&v)[Chunk<T>::N])
{
    RawChunk<T> r;
    r.load(p, n);
#pragma unroll
    for (int i = 0; i < Chunk<T>::N; ++i) v[i] = r[i];
}

template <typename T>
__device__ __forceinline__ void store_row(T *p, int n, const float (&v)[Chunk<T>::N])
{
    RawChunk<T> r;
    r.pack(v);
    r.store(p, n);
}

// A chunk's floats of a vector of C, those past its end as zeros.
template <int N> __device__ __forceinline__ void load_floats(const float *p, int n, float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4)
        load_row<float>(p + i, max(0, n - i), *(float(*)[4])(v + i));
}

template <int N>
__device__ __forceinline__ void store_floats(float *p, int n, const float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4)
        store_row<float>(p + i, max(0, n - i), *(const float(*)[4])(v + i));
}

// Workgroups of a launch, at most: rows beyond go round the grid (a launch holds fewer
// than 2^32 threads).
constexpr int64_t kMaxBlocks = int64_t(1) << 21;

}  // namespace whtmix
