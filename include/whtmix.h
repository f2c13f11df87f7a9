/*
 * whtmix.h -- C ABI of the MI355X (gfx950) WHTMix token mixer.
 *
 * The mixer is the Walsh-Hadamard token mixer of "WHTMix: Efficient Stereo
 * Depth Estimation via Walsh-Hadamard Token Mixing", section III-B, eqs.
 * (2)-(3), in its joint per-frequency-gain form:
 *
 *     Y[b] = H_N (G o (H_N X[b] H_C)) H_C,      b = 0 .. B-1
 *
 *   X[b], Y[b]  N x C (tokens x channels), row-major, channels fastest;
 *   H_n         the orthonormal Sylvester-ordered Walsh-Hadamard matrix,
 *               entry (i, j) = (-1)^popcount(i & j) / sqrt(n), n = 2^k;
 *               H_n is symmetric and orthogonal, so H_n^{-1} = H_n;
 *   G           N_pad x C float32 per-frequency gain shared by every slice b
 *               ("o" is the element-wise product).
 *
 * C must be a power of two.  N may be any count >= 1: rows N .. N_pad-1 of
 * X, N_pad = 2^ceil(log2 N), are taken as zeros so that H_N acts on a
 * power-of-two length (section III-B), the mixer runs on the N_pad x C slice,
 * and Y keeps its first N rows.  For a power-of-two N, N_pad = N.
 *
 * The paper's own gains are log-domain vectors g_c (length C) and g_t
 * (length N_pad) applied by eq. (2) then eq. (3); that is this operation with
 * G[n][c] = exp(g_t[n]) * exp(g_c[c]), and whtmix_forward_separable() computes
 * it from the log gains directly.
 *
 * All computation runs in hand-written HIP kernels on the GPU.  Arithmetic is
 * float32 (bf16 inputs are widened exactly, bf16 outputs are rounded to
 * nearest even once at the end); the four orthonormal 1/sqrt factors are
 * applied together as the exact power of two 1/(N*C) at the gain multiply.
 *
 * Threading and streams: every entry point is safe to call from several host
 * threads.  Work is enqueued on the caller's stream and the call returns
 * without waiting for it.  The library keeps one float32 workspace of
 * B*N_pad*C*4 bytes per (device, stream) for shapes that need more than one
 * pass; it is allocated (or grown) on the first call that needs it, which
 * therefore synchronises that stream and is not safe inside HIP graph
 * capture.  A captured graph keeps the address of the workspace that its calls
 * took: size it by such calls on the capturing stream beforehand, and let no
 * larger call on that stream grow it, and nothing release it, while the graph
 * is in use.
 */
#ifndef WHTMIX_H
#define WHTMIX_H

#include <stdint.h>

#if defined(__GNUC__)
#define WHTMIX_API __attribute__((visibility("default")))
#else
#define WHTMIX_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of x and y (the gain is always float32). */
typedef enum whtmix_dtype {
    WHTMIX_DTYPE_F32 = 0,
    WHTMIX_DTYPE_BF16 = 1
} whtmix_dtype;

/* Return codes.  Every argument check runs on the host before any HIP call;
 * a rejected call enqueues nothing and writes nothing. */
typedef enum whtmix_status {
    WHTMIX_SUCCESS = 0,
    WHTMIX_ERROR_INVALID_VALUE = 1,    /* null pointer, B < 0, N < 1, partial
                                          x/y overlap, a gain overlapping y,
                                          bad option values */
    WHTMIX_ERROR_NOT_POWER_OF_TWO = 2, /* C not a power of two >= 1 */
    WHTMIX_ERROR_UNSUPPORTED_DTYPE = 3,
    WHTMIX_ERROR_MISALIGNED = 4,       /* x, y or gain not 16-byte aligned */
    WHTMIX_ERROR_OUT_OF_MEMORY = 5,    /* workspace allocation failed */
    WHTMIX_ERROR_HIP = 6,              /* HIP runtime / launch error; text in
                                          whtmix_last_error() */
    WHTMIX_ERROR_TOO_LARGE = 7,        /* N_pad*C > 2^30, sizes overflow, or
                                          module C > 4096 */
    WHTMIX_ERROR_DEVICE_TIMEOUT = 8    /* whtmix_stream_status only: a
                                          ONE_LAUNCH call on the stream gave
                                          up waiting for one of its passes
                                          (its output is not valid) */
} whtmix_status;

/* Execution plans.  AUTO picks by the padded slice size L = N_pad*C:
 *   L <= 2^10          one small workgroup per slice, all stages in LDS;
 *   2^11 <= L <= 2^15  FUSED: one workgroup per slice, a single pass; for
 *                      L = 2^15 up to 48 slices TWO_PASS instead;
 *   L = 2^16           WAVE_TILES up to 3 slices, TWO_PASS from 4 to 16,
 *                      FUSED (two register sets) from 48 slices, THREE_PASS
 *                      between;
 *   L >= 2^17          THREE_PASS: forward over the low bits of the flat
 *                      index, then forward over the high bits + gain +
 *                      inverse over the high bits, then inverse over the low
 *                      bits, exchanging through the workspace.
 * WAVE_TILES runs the same three passes on one-wave tiles of 2^9 elements
 * whose butterflies stay inside the wave (DPP and lane-swap exchanges, no
 * LDS): three launches of 2^(K-9) workgroups per slice; 2^12 <= L <= 2^16
 * and N*C a multiple of 8 (AUTO falls back to the plans above otherwise);
 * forced, B*L < 2^35 besides (WHTMIX_ERROR_TOO_LARGE beyond).
 * TWO_PASS (L = 2^15 or 2^16, N*C a multiple of 8) replaces WAVE_TILES's
 * first two launches by one: each of a slice's 2^(K-12) workgroups reads the
 * whole slice and forms its share of the low-bit transform as a signed sum
 * of the slice's blocks, then runs the high bits, the gain and their
 * inverse; WAVE_TILES's last launch follows.  B rounded up to a multiple of
 * 8, times L, must stay below 2^35.
 * ONE_LAUNCH (never chosen by AUTO) runs WAVE_TILES's three passes in a
 * single cooperative launch, ordered by per-slice counters in a small
 * per-stream block; B <= 2046 besides.  On MI355X it is slower than the plans
 * AUTO picks: a cooperative launch alone costs about 20 us, and a hand-off
 * between workgroups through memory costs more than a kernel boundary.
 * THREE_PASS may also be forced for 2^12 <= L <= 2^16 (tests compare it with
 * FUSED on the same shapes).  The backward pass and the block take FUSED
 * for slices up to 2^15 and THREE_PASS from 2^16 whatever the forward plan. */
typedef enum whtmix_plan {
    WHTMIX_PLAN_AUTO = 0,
    WHTMIX_PLAN_SMALL = 1,
    WHTMIX_PLAN_FUSED = 2,
    WHTMIX_PLAN_THREE_PASS = 3,
    WHTMIX_PLAN_ONE_LAUNCH = 4,
    WHTMIX_PLAN_WAVE_TILES = 5,
    WHTMIX_PLAN_TWO_PASS = 6
} whtmix_plan;

typedef struct whtmix_options {
    int plan;          /* whtmix_plan; WHTMIX_PLAN_AUTO = 0 */
    /* Optional hipEvent_t handles (NULL to skip).  events[0] is recorded on
     * the stream before the first kernel and events[i] after the i-th kernel
     * of the plan (at most 3 kernels).  Used for per-kernel timing. */
    void *events[4];
    /* ONE_LAUNCH: polls of the kernel's counter waits before the call gives
     * up (0 = the default, about a second or two).  A call that gives up
     * exits normally with an invalid output and raises the stream's error
     * word (whtmix_stream_status).  Tests force that path with a tiny
     * limit. */
    uint32_t spin_limit;
} whtmix_options;

/* Describes how a shape would run (no GPU work, no allocation).  plan,
 * kernels and workspace_bytes are whtmix_forward's; the backward pass and the
 * block run 2^16-element slices, whose forward is FUSED, with the three-pass
 * plan (and its workspace). */
typedef struct whtmix_plan_info {
    int plan;             /* resolved whtmix_plan (never AUTO) */
    int kernels;          /* kernels launched per call (1 or 3) */
    int log2_slice;       /* K = log2(N*C) */
    int outer_bits;       /* THREE_PASS, WAVE_TILES, ONE_LAUNCH: flat-index bits of the
                             outer passes */
    int run_bits;         /* THREE_PASS, WAVE_TILES, ONE_LAUNCH: log2 of the contiguous run carried
                             by the middle pass */
    int64_t workspace_bytes; /* float32 workspace this call needs */
    int64_t padded_tokens;   /* N_pad */
    /* How whtmix_module_forward runs this shape: 0 SMALL (projections on the
     * vector ALUs), 1 projections fused into the mixer's kernels on the
     * matrix cores, 2 projection kernels around the float32 mixer; -1 when C
     * exceeds the block's limit. */
    int module_path;
    int module_outer_bits;   /* THREE_PASS: the block's outer-pass bits */
    /* 1 when whtmix_module_backward runs its projections inside the mixer
     * backward's passes (given B > 0 and a requested gain gradient); its
     * events then bracket [transforms of Z and dZ', gain gradient], [Z',
     * dW_out], [dX, dW_in] instead of [Z, Z', dZ', dW_out], [the mixer's
     * gradients], [dX, dW_in]. */
    int module_backward_fused;
} whtmix_plan_info;

/*
 * whtmix_forward -- y[b] = H_N (G o (H_N x[b] H_C)) H_C for b in [0, B)
 * (section III-B, eqs. (2)-(3), joint gain).
 *
 *   x      device pointer, [B][N][C] contiguous elements of `dtype`
 *          (read only).  May equal y exactly (in place); any other overlap
 *          with y is rejected.
 *   gain   device pointer, [N_pad][C] contiguous float32 (linear gains),
 *          shared by all b; must not overlap y.
 *   y      device pointer, [B][N][C] contiguous elements of `dtype` (written).
 *   B      number of independent slices; B == 0 is a no-op (pointers are not
 *          inspected).
 *   N, C   tokens (>= 1) and channels (a power of two >= 1), N_pad*C <= 2^30.
 *   dtype  whtmix_dtype of x and y.
 *   stream hipStream_t to enqueue on (NULL = the null stream).
 *
 * The caller owns x, gain and y and keeps them alive until the stream work
 * is done.  Pointers must be 16-byte aligned.  Returns a whtmix_status.
 * Kernel faults surface asynchronously through the stream like any HIP op.
 */
WHTMIX_API int whtmix_forward(const void *x, const float *gain, void *y,
                   int64_t B, int64_t N, int64_t C, int dtype, void *stream);

/*
 * whtmix_forward_noalloc -- whtmix_forward for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc).  Same arguments, result, plan (AUTO) and checks as
 * whtmix_forward, but the workspace of the three-pass, two-pass and wave-tile
 * plans is a fixed 32 MiB device array inside the library (one per device, held until the process ends) instead
 * of the per-stream workspace, and the call allocates nothing: no hipMalloc,
 * no hipFree, no stream synchronisation.  Limit: shapes whose plan needs a
 * workspace must have B * N_pad * C <= 2^23; larger ones return
 * WHTMIX_ERROR_TOO_LARGE (text in whtmix_last_error()) with nothing
 * enqueued.  Every call on a device shares that device's array, so calls
 * that overlap on one device (on different streams or host threads) race;
 * serialise them.
 */
WHTMIX_API int whtmix_forward_noalloc(const void *x, const float *gain, void *y,
                           int64_t B, int64_t N, int64_t C, int dtype, void *stream);

/* As whtmix_forward, with options (NULL = defaults). */
WHTMIX_API int whtmix_forward_ex(const void *x, const float *gain, void *y,
                      int64_t B, int64_t N, int64_t C, int dtype, void *stream,
                      const whtmix_options *options);

/*
 * whtmix_forward_separable -- the paper's parametrisation, eq. (2) then
 * eq. (3):  Z <- H_C^{-1}(exp(g_c) o H_C Z) along channels, then
 *           Z <- H_N^{-1}(exp(g_t) o H_N Z) along tokens,
 * i.e. whtmix_forward with G[n][c] = exp(g_t[n]) * exp(g_c[c]).  The gain of
 * each frequency is formed on the device as exp(g_t[n] + g_c[c]), so the
 * only gain traffic is the two small vectors.
 *
 *   log_gain_tokens    device pointer, [N_pad] float32 log gains g_t
 *   log_gain_channels  device pointer, [C] float32 log gains g_c
 * Both are 16-byte aligned and must not overlap y (zero log gains, the
 * paper's initialisation, give Y = X).  Other arguments, options and return
 * codes as whtmix_forward_ex (options may be NULL).
 */
WHTMIX_API int whtmix_forward_separable(const void *x, const float *log_gain_tokens,
                             const float *log_gain_channels, void *y,
                             int64_t B, int64_t N, int64_t C, int dtype,
                             void *stream, const whtmix_options *options);

/*
 * whtmix_backward -- gradients through whtmix_forward for an upstream
 * gradient dy = dL/dy (the paper trains the gains, section IV-A).  With the
 * orthonormal transforms T(v) = H_Npad vpad H_C of zero-padded slices:
 *     dx[b] = H_N (G o T(dy[b])) H_C, first N rows (the mixer is
 *             self-adjoint, so this is whtmix_forward applied to dy);
 *     dgain = sum over b of T(x[b]) o T(dy[b])        ([N_pad][C] float32).
 *
 *   x, dy  device pointers, [B][N][C] elements of `dtype` (x is not read when
 *          dgain is NULL).
 *   gain   [N_pad][C] float32, as passed to the forward call.
 *   dx     [B][N][C] of `dtype`, or NULL to skip; may be dy itself.
 *   dgain  [N_pad][C] float32, overwritten (not accumulated), or NULL to skip.
 * At least one of dx, dgain must be non-NULL.  No output may overlap an
 * input or another output (except dx == dy).  With B == 0 dgain is filled
 * with zeros.  The gain gradient is summed over the batch in a fixed order,
 * so results are bitwise reproducible.  The call uses a float32 workspace of
 * up to 2*B*N_pad*C (+ partial sums) floats; other conventions and options as
 * whtmix_forward_ex (events: [0] before, [1] after the gain gradient, [2]
 * after dx).  With the three-pass plan and both outputs requested, the two
 * gradients share dy's transform: the gain gradient is complete at [1] and
 * only dx's last pass runs between [1] and [2].
 */
WHTMIX_API int whtmix_backward(const void *x, const void *dy, const float *gain,
                    void *dx, float *dgain, int64_t B, int64_t N, int64_t C,
                    int dtype, void *stream, const whtmix_options *options);

/*
 * whtmix_backward_separable -- gradients through whtmix_forward_separable:
 *     dx                as whtmix_backward with G[n][c] = exp(g_t[n] + g_c[c]),
 *     d_log_gain_tokens[n]   = sum over c of dG[n][c] G[n][c]   ([N_pad]),
 *     d_log_gain_channels[c] = sum over n of dG[n][c] G[n][c]   ([C]),
 * (the chain rule through exp).  The two log-gain gradients are both NULL or
 * both non-NULL; everything else as whtmix_backward.
 */
WHTMIX_API int whtmix_backward_separable(const void *x, const void *dy,
                              const float *log_gain_tokens,
                              const float *log_gain_channels, void *dx,
                              float *d_log_gain_tokens,
                              float *d_log_gain_channels, int64_t B,
                              int64_t N, int64_t C, int dtype, void *stream,
                              const whtmix_options *options);

/*
 * whtmix_module_forward -- the whole block of section III-B, eqs. (1)-(4),
 * with the joint gain:
 *     Z = X[b] W_in;   Z <- H_N (G o (H_N Z H_C)) H_C;   Y[b] = Z W_out
 * (Z zero-padded to N_pad rows before H_N, Y cropped to the first N rows),
 * the drop-in replacement of the self-attention block with its projections.
 *
 *   x      [B][N][C] elements of `dtype`; may equal y exactly (in place).
 *   w_in   [C][C] elements of `dtype`, row-major: Z[n][j] = sum_i X[n][i]
 *          W_in[i][j].
 *   gain   [N_pad][C] float32 linear gains (as whtmix_forward).
 *   w_out  [C][C] elements of `dtype`: Y[n][j] = sum_i Z[n][i] W_out[i][j].
 *   y      [B][N][C] elements of `dtype` (written).
 * C is a power of two <= 4096 (WHTMIX_ERROR_TOO_LARGE above).  Inputs must
 * not overlap y except x == y.  Arithmetic is float32: for bf16 the products
 * X W_in are exact, Z' W_out uses a two-term bf16 split of Z' (relative
 * residual below 2^-17), and y is rounded to nearest even once.  For
 * 16 <= C <= 128, and for bf16 C = 256 from N_pad*C = 2^17, the projections
 * run on the matrix cores inside the mixer's first and last kernels (three
 * kernels for N_pad*C > 2^15, plus a small weight-repacking kernel for C = 256 and
 * for bf16 C = 128 on many slices of 2^16 or 2^17 elements;
 * whtmix_plan_describe's module_path says which); other shapes run separate
 * projection kernels around the float32 mixer.  Workspace: the mixer's, plus
 * 2*C*C elements of packed weights (where they are repacked, and the separate kernels) and
 * B*N*C floats of Z (the separate kernels).  Other conventions, plans and options as
 * whtmix_forward_ex (events: for the three-pass plan around each of its
 * three passes, otherwise [0] before and [1] after the call's kernels).
 */
WHTMIX_API int whtmix_module_forward(const void *x, const void *w_in,
                          const float *gain, const void *w_out, void *y,
                          int64_t B, int64_t N, int64_t C, int dtype,
                          void *stream, const whtmix_options *options);

/*
 * whtmix_module_forward_separable -- whtmix_module_forward with the paper's
 * log-domain gains (eqs. (2)-(3)): log_gain_tokens [N_pad] and
 * log_gain_channels [C] float32, as whtmix_forward_separable.
 */
WHTMIX_API int whtmix_module_forward_separable(const void *x, const void *w_in,
                                    const float *log_gain_tokens,
                                    const float *log_gain_channels,
                                    const void *w_out, void *y, int64_t B,
                                    int64_t N, int64_t C, int dtype,
                                    void *stream,
                                    const whtmix_options *options);

/*
 * whtmix_module_backward -- gradients through whtmix_module_forward for an
 * upstream gradient dy = dL/dY (the paper trains the block, section IV-A):
 *     dZ' = dY W_out^T,            dW_out = sum over b of Z'^T dY,
 *     dZ, dgain = the mixer's gradients (whtmix_backward) at (Z, dZ'),
 *     dX = dZ W_in^T,              dW_in  = sum over b of X^T dZ,
 * with Z = X W_in and Z' = mixer(Z) recomputed in float32.  For 16 <= C <=
 * 128 on three-pass slices up to 2^25 elements, and bf16 C = 256 on
 * 2^26..2^28 (with a requested gain gradient), the projections run inside
 * the mixer backward's passes and Z and dZ' are never stored
 * (whtmix_plan_describe's module_backward_fused).
 *
 *   x, dy         [B][N][C] elements of `dtype`.
 *   w_in, w_out   [C][C] elements of `dtype`, as passed to the forward call.
 *   gain          [N_pad][C] float32.
 *   dx            [B][N][C] of `dtype` (written); may be dy itself.
 *   dw_in, dw_out [C][C] float32, overwritten.
 *   dgain         [N_pad][C] float32, overwritten, or NULL to skip.
 * No output may overlap an input or another output (except dx == dy); B*N <
 * 2^31.  Weight gradients are summed over row chunks in a fixed order, so
 * results are bitwise reproducible.  Workspace: the mixer's backward
 * workspace and the weight-gradient partial sums; where the projections or the weight gradients run apart from the
 * mixer's passes (any other shape, C = 16 on 2^24 and 2^25 elements, C = 128 on
 * 2^16 and 2^17, and C = 256) 3*B*N*C floats and the forward workspace besides,
 * and 3*C*C packed weight elements.  Other conventions as
 * whtmix_module_forward (events: [0] before, then after each phase: [1]
 * dW_out, [2] the mixer's gradients, [3] dX and dW_in; with the projections
 * inside the mixer's passes [1] the gain gradient, [2] dW_out (and dW_in
 * where the two are formed together), [3] dX and dW_in).
 */
WHTMIX_API int whtmix_module_backward(const void *x, const void *w_in,
                           const float *gain, const void *w_out,
                           const void *dy, void *dx, float *dw_in,
                           float *dw_out, float *dgain, int64_t B, int64_t N,
                           int64_t C, int dtype, void *stream,
                           const whtmix_options *options);

/*
 * whtmix_module_backward_separable -- as whtmix_module_backward for the
 * block with log-domain gains: d_log_gain_tokens [N_pad] and
 * d_log_gain_channels [C] float32 (both NULL or both non-NULL), as
 * whtmix_backward_separable.
 */
WHTMIX_API int whtmix_module_backward_separable(const void *x, const void *w_in,
                                     const float *log_gain_tokens,
                                     const float *log_gain_channels,
                                     const void *w_out, const void *dy,
                                     void *dx, float *dw_in, float *dw_out,
                                     float *d_log_gain_tokens,
                                     float *d_log_gain_channels, int64_t B,
                                     int64_t N, int64_t C, int dtype,
                                     void *stream,
                                     const whtmix_options *options);

/*
 * ---- The feed-forward sublayer ----
 *
 * The mixer is linear; what follows it in a layer is the residual's addition
 * with a norm, and two matrix products with an activation between them (the
 * feed-forward part of the transformer stack, section III-A).  Rules that these
 * entry points share:
 *   - rows are contiguous, channels fastest; rows of x are ldx elements apart
 *     (ldx >= its width, so that x may be columns of a wider array);
 *   - any width >= 1 and any count of rows >= 0, at most 2^30 rows and
 *     2^22 columns (WHTMIX_ERROR_TOO_LARGE); with no rows the gradients of
 *     weights are zeros and the rest is a no-op;
 *   - pointers need the alignment of their elements (8-bit values: 16 bytes);
 *   - matrices have the dtype of x, vectors (bias, norm weight) and their
 *     gradients are float32;
 *   - arithmetic is float32 and each output is rounded once, to nearest even;
 *   - no output overlaps an input or another output, but for those named;
 *   - the checks, the workspace, streams and errors are those of the mixer.
 *
 * Block-scaled 8 bits ("MX"): a row of C values is stored as C rounded up to a
 * multiple of 32 float8 e4m3 values (those past C are zero) and one byte s per
 * 32 of them; a value is q * 2^(s - 127).  The scale is the least power of two
 * in 2^-126 .. 2^120 with which the block's largest finite magnitude stays
 * within e4m3's 448; Inf and NaN are stored as NaN.
 */
typedef enum whtmix_activation {
    WHTMIX_ACT_NONE = 0,
    WHTMIX_ACT_RELU = 1,      /* max(z, 0); its derivative at 0 is 0 */
    WHTMIX_ACT_GELU = 2,      /* z (1 + erf(z / sqrt 2)) / 2 */
    WHTMIX_ACT_GELU_TANH = 3, /* z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2 */
    WHTMIX_ACT_SILU = 4       /* z / (1 + exp(-z)) */
} whtmix_activation;

/*
 * whtmix_norm_forward -- root-mean-square norm with the residual's addition:
 *     t = x + residual,   h = t,   y = t / sqrt(mean(t^2) + eps) * weight.
 *   x         [rows] rows of C elements of `dtype`, ldx apart.
 *   residual  [rows][C] or NULL (t = x).      weight  [C] float32.
 *   y         [rows][C] of `dtype`; may be x (with ldx = C).
 *   h         [rows][C] of `dtype`, t rounded, or NULL; may be x (with ldx =
 *             C) or the residual, but not y.
 * y is formed from t before its rounding.  eps >= 0 and finite.
 */
WHTMIX_API int whtmix_norm_forward(const void *x, const void *residual,
                        const float *weight, void *y, void *h, int64_t rows,
                        int64_t C, int64_t ldx, double eps, int dtype,
                        void *stream);

/*
 * whtmix_norm_mx_forward -- whtmix_norm_forward with y in block-scaled 8 bits:
 *   q [rows][C up to 32] e4m3, scales [rows][C up to 32 / 32].
 */
WHTMIX_API int whtmix_norm_mx_forward(const void *x, const void *residual,
                           const float *weight, void *q, uint8_t *scales,
                           void *h, int64_t rows, int64_t C, int64_t ldx,
                           double eps, int dtype, void *stream);

/*
 * whtmix_norm_backward -- gradients of whtmix_norm_forward from the kept
 * stream h: with r = 1 / sqrt(mean(h^2) + eps), n = h r, g = dy weight,
 *     dx = dh + r (g - n mean(g n)),   dweight = sum over rows of dy n.
 *   h, dy     [rows][C] of `dtype`.
 *   dh        [rows][C] of `dtype`, the gradient of h, or NULL (zeros).
 *   dx        [rows][C] of `dtype`: the gradient of x and of the residual;
 *             may be dy or dh.
 *   dweight   [C] float32, or NULL to skip.
 * dweight is summed in a fixed order.  Workspace: for dweight, up to 1536 rows
 * of C floats; for rows of more than 16384 elements, two floats a row besides.
 */
WHTMIX_API int whtmix_norm_backward(const void *h, const float *weight,
                         const void *dy, const void *dh, void *dx,
                         float *dweight, int64_t rows, int64_t C, double eps,
                         int dtype, void *stream);

/* whtmix_quantize_mx -- rows in block-scaled 8 bits: x [rows] rows of C
 * elements of `dtype`, ldx apart; q and scales as whtmix_norm_mx_forward. */
WHTMIX_API int whtmix_quantize_mx(const void *x, void *q, uint8_t *scales,
                       int64_t rows, int64_t C, int64_t ldx, int dtype,
                       void *stream);

/* whtmix_dequantize_mx -- the values that q and scales stand for, rounded to
 * `dtype`: y [rows][C]. */
WHTMIX_API int whtmix_dequantize_mx(const void *q, const uint8_t *scales, void *y,
                         int64_t rows, int64_t C, int dtype, void *stream);

/*
 * whtmix_linear_forward -- matrix product with bias, activation and residual:
 *     z = x w + bias,   y = act(z) + residual.
 *   x         [M] rows of K elements of `dtype`, ldx apart.
 *   w         [K][N] of `dtype` (z[m][n] = sum_k x[m][k] w[k][n]).
 *   bias      [N] float32, or NULL.
 *   residual  [M][N] of `dtype`, or NULL.
 *   y         [M][N] of `dtype`; may be the residual.
 *   z         [M][N] of `dtype`, what the backward pass keeps, or NULL.
 * Sums are float32; with float32 elements the products are six bf16 products
 * of three-term splits (what they leave out is below 2^-24 |x| |w|), or float32
 * ones in tiles where a value is 2^128 - 2^119 or more, or where a row of x or a
 * column of w is nonzero and below 2^-95 throughout.  (A value below 2^-109
 * beside larger ones of its row or column is off by 2^-134 at most.)
 * Workspace: partial sums where k is split over workgroups; large float32
 * operands' terms (six bytes an element); bf16 operands whose rows do not start
 * at 16 bytes, packed.
 */
WHTMIX_API int whtmix_linear_forward(const void *x, const void *w,
                          const float *bias, const void *residual, void *y,
                          void *z, int64_t M, int64_t K, int64_t N,
                          int64_t ldx, int activation, int dtype,
                          void *stream);

/*
 * whtmix_linear_backward -- gradients of whtmix_linear_forward:
 *     dz = dy act'(z),   dx = dz w^T,   dw = x^T dz,   dbias = sum_m dz.
 *   x, w      as passed forward;  dy [M][N] of `dtype`.
 *   z         [M][N] as kept (may be NULL with WHTMIX_ACT_NONE).
 *   dx        [M][K] of `dtype`, or NULL to skip.
 *   dw        [K][N] of `dtype`, or NULL to skip.
 *   dbias     [N] float32, or NULL to skip.
 * The residual's gradient is dy itself.  dz enters the products rounded to
 * `dtype` (bf16: what the matrix cores read; for a float32 dz pass float32
 * copies) and dbias unrounded.  Sums over rows are made in a fixed order, which
 * sizes and the outputs asked for choose: dbias may differ in its last bits with
 * and without dx.  Workspace: dz where a product reads it from memory, partial sums, and what the
 * forward product takes.
 */
WHTMIX_API int whtmix_linear_backward(const void *x, const void *w,
                           const void *dy, const void *z, void *dx, void *dw,
                           float *dbias, int64_t M, int64_t K, int64_t N,
                           int64_t ldx, int activation, int dtype,
                           void *stream);

/*
 * whtmix_linear_mx_forward -- whtmix_linear_forward on block-scaled 8 bits:
 *   xq, xs    the activations, [M] rows of K values.
 *   wq, ws    the weights' columns as rows: [N] rows of K values.
 *   bias, residual  as whtmix_linear_forward, the residual of `dtype`.
 *   y         [M][N] of `dtype` (may be the residual), or NULL with
 *   yq, ys    the output in block-scaled 8 bits, [M] rows of N values.
 * Either y or both yq and ys.  Products of K > 512 with a bfloat16 or 8-bit
 * output run on the scaled matrix instructions, which keep about 15 bits below
 * the largest of 64 products before they add to a float32 sum: off by 1e-6 of
 * the sum of magnitudes, root mean square, for normal values, by 1e-5 for
 * values spread over 2^6.  The others' sums are float32 throughout, of bf16
 * values (what lies below 2^-125 is taken to the nearest 2^-133); a caller that
 * wants such sums of more k takes y in float32 and rounds it, or quantises it
 * with whtmix_quantize_mx.
 */
WHTMIX_API int whtmix_linear_mx_forward(const void *xq, const uint8_t *xs,
                             const void *wq, const uint8_t *ws,
                             const float *bias, const void *residual, void *y,
                             void *yq, uint8_t *ys, int64_t M, int64_t K,
                             int64_t N, int activation, int dtype,
                             void *stream);

/*
 * ---- What a text model has besides: layer norm, gated products, embedding ----
 *
 * The rules of the feed-forward sublayer hold for these too.
 */

/*
 * whtmix_layer_norm_forward -- layer norm with the residual's addition:
 *     t = x + residual,   h = t,
 *     y = (t - mean(t)) / sqrt(mean((t - mean(t))^2) + eps) * weight + bias.
 *   x         [rows] rows of C elements of `dtype`, ldx apart.
 *   residual  [rows][C] or NULL (t = x).
 *   weight    [C] float32.      bias  [C] float32, or NULL (zeros).
 *   y         [rows][C] of `dtype`; may be x (with ldx = C).
 *   h         [rows][C] of `dtype`, t rounded, or NULL; may be x (with ldx =
 *             C) or the residual, but not y.
 * y is formed from t before its rounding.  eps >= 0 and finite.  A row's sums, of
 * its values and of their squared distances from the mean, are float32, in the
 * backward pass too: both below 2^128, which distances up to 2^64 / sqrt(C) keep.
 */
WHTMIX_API int whtmix_layer_norm_forward(const void *x, const void *residual,
                              const float *weight, const float *bias, void *y,
                              void *h, int64_t rows, int64_t C, int64_t ldx,
                              double eps, int dtype, void *stream);

/*
 * whtmix_layer_norm_mx_forward -- whtmix_layer_norm_forward with y in
 * block-scaled 8 bits: q [rows][C up to 32] e4m3, scales [rows][C up to 32 / 32].
 */
WHTMIX_API int whtmix_layer_norm_mx_forward(const void *x, const void *residual,
                                 const float *weight, const float *bias,
                                 void *q, uint8_t *scales, void *h,
                                 int64_t rows, int64_t C, int64_t ldx,
                                 double eps, int dtype, void *stream);

/*
 * whtmix_layer_norm_backward -- gradients of whtmix_layer_norm_forward from the
 * kept stream h: with r = 1 / sqrt(mean((h - mean(h))^2) + eps), n = (h -
 * mean(h)) r, g = dy weight,
 *     dx = dh + r (g - mean(g) - n mean(g n)),
 *     dweight = sum over rows of dy n,   dbias = sum over rows of dy.
 *   h, dy     [rows][C] of `dtype`.
 *   dh        [rows][C] of `dtype`, the gradient of h, or NULL (zeros).
 *   dx        [rows][C] of `dtype`: the gradient of x and of the residual;
 *             may be dy or dh.
 *   dweight, dbias  [C] float32, or NULL to skip.
 * Both are summed in a fixed order.  Workspace: for them, none for a few rows and
 * up to 1536 rows of 2 C floats; for rows of more than 16384 elements, five floats a row besides.
 */
WHTMIX_API int whtmix_layer_norm_backward(const void *h, const float *weight,
                               const void *dy, const void *dh, void *dx,
                               float *dweight, float *dbias, int64_t rows,
                               int64_t C, double eps, int dtype, void *stream);

/*
 * whtmix_gated_forward -- gated product, both projections in one kernel:
 *     zg = x wg + bg,   zu = x wu + bu,   y = act(zg) zu  (element by element).
 *   x         [M] rows of K elements of `dtype`, ldx apart.
 *   wg, wu    [K][N] of `dtype`, N <= 2^21.
 *   bg, bu    [N] float32, each or NULL.
 *   y         [M][N] of `dtype`.
 *   zg, zu    [M][N] of `dtype`, what the backward pass keeps, each or NULL.
 * y is formed from zg and zu before their rounding.  Sums as
 * whtmix_linear_forward's.  Workspace: as whtmix_linear_forward's, for both
 * products.
 */
WHTMIX_API int whtmix_gated_forward(const void *x, const void *wg, const void *wu,
                         const float *bg, const float *bu, void *y, void *zg,
                         void *zu, int64_t M, int64_t K, int64_t N, int64_t ldx,
                         int activation, int dtype, void *stream);

/*
 * whtmix_gated_backward -- gradients of whtmix_gated_forward:
 *     dzg = dy zu act'(zg),   dzu = dy act(zg),
 *     dx = dzg wg^T + dzu wu^T,   dwg = x^T dzg,   dwu = x^T dzu,
 *     dbg = sum_m dzg,   dbu = sum_m dzu.
 *   x, wg, wu  as passed forward;  dy [M][N] of `dtype`.
 *   zg, zu    [M][N] as kept (needed with WHTMIX_ACT_NONE too).
 *   dx        [M][K] of `dtype`, or NULL to skip.
 *   dwg, dwu  [K][N] of `dtype`, or both NULL to skip.
 *   dbg, dbu  [N] float32, or both NULL to skip.
 * dzg and dzu enter the products rounded to `dtype` (as whtmix_linear_backward's
 * dz) and the biases' sums unrounded.  Sums over rows are made in a fixed
 * order, which sizes and the outputs asked for choose: dbg and dbu may differ in
 * their last bits with and without dx.  Workspace: dzg and dzu where a product reads them from memory, partial
 * sums, the weights side by side where N is not a multiple of 64 (or `dtype`
 * float32), and what the products take.
 */
WHTMIX_API int whtmix_gated_backward(const void *x, const void *wg, const void *wu,
                          const void *dy, const void *zg, const void *zu,
                          void *dx, void *dwg, void *dwu, float *dbg,
                          float *dbu, int64_t M, int64_t K, int64_t N,
                          int64_t ldx, int activation, int dtype, void *stream);

/*
 * whtmix_gated_mx_forward -- whtmix_gated_forward on block-scaled 8 bits:
 *   xq, xs    the activations, [M] rows of K values.
 *   wgq, wgs, wuq, wus  the weights' columns as rows: [N] rows of K values.
 *   bg, bu    [N] float32, each or NULL.
 *   y         [M][N] of `dtype`, or NULL with
 *   yq, ys    the output in block-scaled 8 bits, [M] rows of N values.
 * Either y or both yq and ys.  Sums as whtmix_linear_mx_forward's.
 */
WHTMIX_API int whtmix_gated_mx_forward(const void *xq, const uint8_t *xs,
                            const void *wgq, const uint8_t *wgs,
                            const void *wuq, const uint8_t *wus,
                            const float *bg, const float *bu, void *y, void *yq,
                            uint8_t *ys, int64_t M, int64_t K, int64_t N,
                            int activation, int dtype, void *stream);

/* Element type of token ids. */
typedef enum whtmix_index {
    WHTMIX_INDEX_I32 = 0,
    WHTMIX_INDEX_I64 = 1
} whtmix_index;

/*
 * whtmix_embedding_forward -- rows of a table by token ids:
 *     y[n] = scale table[ids[n]].
 *   ids       [rows] of the type `index`.
 *   table     [vocab][C] of `dtype`, vocab <= 2^30.
 *   y         [rows][C] of `dtype`.
 * A negative id is padding: its row is zeros.  An id of vocab or more names no
 * row: its row is NaN.  scale is finite.
 */
WHTMIX_API int whtmix_embedding_forward(const void *ids, const void *table, void *y,
                             int64_t rows, int64_t vocab, int64_t C,
                             double scale, int index, int dtype, void *stream);

/*
 * whtmix_embedding_backward -- the table's gradient:
 *     dtable[v] = scale (sum of dy[n] over the n with ids[n] = v).
 *   ids       [rows] of the type `index`, as passed forward.
 *   dy        [rows][C] of `dtype`.
 *   dtable    [vocab][C] of `dtype`: every row is written, zeros where no id
 *             names it.  Padding and ids of vocab or more have no gradient.
 * Sums are float32, in an order that ids, rows, vocab and C fix.  Workspace: 16
 * bytes a token, 2048 bytes for every 2048 tokens, and C floats for every 16
 * tokens at most; or, for vocabularies below 512 of rows of up to 128, up to 24
 * MiB of partial sums and 4 vocab bytes for every 1024 tokens.
 */
WHTMIX_API int whtmix_embedding_backward(const void *ids, const void *dy, void *dtable,
                              int64_t rows, int64_t vocab, int64_t C,
                              double scale, int index, int dtype, void *stream);

/* Fills *info with the plan whtmix_forward_ex would use.  Validates the
 * shape, dtype and options exactly as the forward call does (pointers are
 * not needed).  Returns a whtmix_status. */
WHTMIX_API int whtmix_plan_describe(int64_t B, int64_t N, int64_t C, int dtype,
                         const whtmix_options *options,
                         whtmix_plan_info *info);

/* Static description of a status code (never NULL). */
WHTMIX_API const char *whtmix_status_string(int status);

/* Text of the last WHTMIX_ERROR_HIP / OUT_OF_MEMORY on the calling thread
 * ("" if none). */
WHTMIX_API const char *whtmix_last_error(void);

/* Synchronises every stream that owns a workspace and frees all workspaces.
 * Returns a whtmix_status. */
WHTMIX_API int whtmix_release_workspaces(void);

/* Synchronises `stream` (hipStream_t) on the current device, then reports
 * and clears the error word its ONE_LAUNCH calls raise: WHTMIX_SUCCESS when
 * every ONE_LAUNCH call since the last check completed, or
 * WHTMIX_ERROR_DEVICE_TIMEOUT when one gave up waiting for a pass (its
 * output is invalid; later calls are unaffected).  Other plans never raise
 * it.  Returns WHTMIX_ERROR_HIP if the synchronisation fails. */
WHTMIX_API int whtmix_stream_status(void *stream);

/* Library version as major*10000 + minor*100 + patch. */
WHTMIX_API int whtmix_version(void);

#ifdef __cplusplus
}
#endif

#endif /* WHTMIX_H */
