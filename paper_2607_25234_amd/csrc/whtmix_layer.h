// Internal interface of the feed-forward sublayer's operators: the norm, the
// block-scaled 8-bit (MX) form and the matrix products.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "whtmix_launch.h"

namespace whtmix {

// Block-scaled 8 bits: e4m3 values in blocks of kMxBlock along the row, one
// power of two 2^(byte - 127) a block; rows are stored with mx_width(C)
// values, those past C zero.
constexpr int kMxBlock = 32;
constexpr int64_t mx_width(int64_t C) { return (C + kMxBlock - 1) / kMxBlock * kMxBlock; }

enum Activation { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4 };

// ---- norm: t = x + residual, y = t * rsqrt(mean(t^2) + eps) * weight ----
struct NormArgs {
    const void *x;          // [rows] rows of C elements, ldx apart
    const void *residual;   // [rows][C] or null
    const float *weight;    // [C]
    void *y;                // [rows][C], or null with q
    void *h;                // [rows][C]: t rounded, or null
    void *q;                // [rows][mx_width(C)] e4m3, or null
    uint8_t *scales;        // [rows][mx_width(C) / 32]
    int64_t rows, C, ldx;
    float eps;
    int dtype;
    hipStream_t stream;
};
// weight null: y = x as it is (the quantiser); then rows are not normalised.
hipError_t launch_norm(const NormArgs &a);

struct NormBackwardArgs {
    const void *h;          // [rows][C]
    const float *weight;    // [C]
    const void *dy;         // [rows][C]
    const void *dh;         // [rows][C] or null
    void *dx;               // [rows][C]
    float *dweight;         // [C] or null
    float *ws;              // norm_backward_floats(...) floats
    int64_t rows, C;
    float eps;
    int dtype;
    hipStream_t stream;
};
uint64_t norm_backward_floats(int64_t rows, int64_t C, int dtype, bool dweight);
hipError_t launch_norm_backward(const NormBackwardArgs &a);

hipError_t launch_dequantize(const void *q, const uint8_t *scales, void *y, int64_t rows,
                             int64_t C, int dtype, hipStream_t stream);

// out[c] = sum over the n rows of part [n][C], in order: partial column sums.
hipError_t launch_column_sum(const float *part, int64_t n, int64_t C, float *out,
                             hipStream_t stream);

// Zeros, by a kernel (a fill that a captured graph replays); an even count of bytes.
hipError_t launch_zero(void *p, uint64_t bytes, hipStream_t stream);

// ---- matrix products ----
// y = act(x w + bias) + residual; z = x w + bias where asked for.
struct LinearArgs {
    const void *x;          // [M] rows of K elements, ldx apart
    const void *w;          // [K][N]
    const float *bias;      // [N] or null
    const void *residual;   // [M][N] or null
    void *y;                // [M][N]
    void *z;                // [M][N] or null
    int64_t M, K, N, ldx;
    int act;
    int dtype;
    float *ws;              // linear_bytes(...) bytes
    hipStream_t stream;
};
uint64_t linear_bytes(const LinearArgs &a);
hipError_t launch_linear(const LinearArgs &a);

// dz = dy * act'(z); dx = dz w^T; dw = x^T dz; dbias = column sums of dz.
struct LinearBackwardArgs {
    const void *x, *w, *dy;
    const void *z;          // [M][N], null with ACT_NONE
    void *dx;               // [M][K] or null
    void *dw;               // [K][N] or null
    float *dbias;           // [N] or null
    int64_t M, K, N, ldx;
    int act;
    int dtype;
    float *ws;              // linear_backward_bytes(...) bytes
    hipStream_t stream;
};
uint64_t linear_backward_bytes(const LinearBackwardArgs &a);
hipError_t launch_linear_backward(const LinearBackwardArgs &a);

// The product of 8-bit rows: y (dtype) or yq, ys (8 bits).
struct LinearMxArgs {
    const void *xq;         // [M][mx_width(K)]
    const uint8_t *xs;      // [M][mx_width(K) / 32]
    const void *wq;         // [N][mx_width(K)]: the weights' columns as rows
    const uint8_t *ws8;     // [N][mx_width(K) / 32]
    const float *bias;      // [N] or null
    const void *residual;   // [M][N] of dtype or null
    void *y;                // [M][N] of dtype, or null with yq
    void *yq;               // [M][mx_width(N)]
    uint8_t *ys;            // [M][mx_width(N) / 32]
    int64_t M, K, N;
    int act;
    int dtype;
    float *ws;              // linear_mx_bytes(...) bytes
    hipStream_t stream;
};
uint64_t linear_mx_bytes(const LinearMxArgs &a);
hipError_t launch_linear_mx(const LinearMxArgs &a);

// ---- from whtmix_api.cpp: the per-(device, stream) workspace and errors ----
// Holds the workspaces' lock from the lookup until the kernels that use one
// are enqueued.
class WorkspaceLock {
public:
    WorkspaceLock();
    ~WorkspaceLock();
    WorkspaceLock(const WorkspaceLock &) = delete;
    WorkspaceLock &operator=(const WorkspaceLock &) = delete;
};
// A whtmix_status; the caller holds a WorkspaceLock.
int stream_workspace(void *stream, int64_t bytes, float **out);
// Keeps the error's text for whtmix_last_error; a whtmix_status.
int report_hip(hipError_t e, const char *what);

}  // namespace whtmix
