/*
 * nnconv.h -- C ABI of libnnconv: mixed-precision 2-D convolution in the
 * three training passes (forward, backward-data, backward-weight) on one
 * AMD Instinct MI355X (gfx950); and, after it, the operators of gated sequence blocks on
 * channel-last tokens (norm, recurrence) and the solver they are trained with.
 *
 * The operation is the paper's convolution call (Sec. 3.2, Listings 4-5:
 * convolution(x, base_axis=1, outmaps, kernel, ...)), trained by
 * back-propagation (Sec. 2.1) in mixed precision: half-precision storage of
 * weights, activations and gradients, products accumulated in fp32, and a
 * loss scale S that multiplies the incoming gradient and is divided out of
 * the weight gradient before the fp32 update (Sec. 3.3, Listing 6).
 *
 * Definitions (cross-correlation, symmetric zero padding):
 *   P = floor((H + 2*pad_h - dil_h*(R-1) - 1) / stride_h) + 1   (same for Q)
 *   Cg = C/groups, Kg = K/groups; output channel k reads input channels
 *   [ (k/Kg)*Cg, (k/Kg)*Cg + Cg ).
 *   forward   y[n,k,p,q]  = alpha * sum_{c<Cg,r<R,s<S} xz[n,(k/Kg)*Cg+c, p*sh-ph+r*dh, q*sw-pw+s*dw] * w[k,c,r,s]
 *   dgrad     dx = alpha * (adjoint of the forward map in x) applied to dy
 *   wgrad     dw = beta * dw + inv_loss_scale * (adjoint of the forward map in w)(x, dy)
 *   where xz is x extended by zeros.  dy is expected to carry the loss scale
 *   already (the caller scaled the loss); dgrad keeps it, wgrad removes it.
 *
 * Layouts (dense, contiguous):
 *   NNCONV_NCHW  x[N][C][H][W], y/dy[N][K][P][Q], w/dw[K][Cg][R][S]
 *   NNCONV_NHWC  x[N][H][W][C], y/dy[N][P][Q][K], w/dw[K][R][S][Cg]
 *
 * Ownership and execution:
 *   - Every buffer is a device pointer owned by the caller; the library
 *     allocates no memory (scratch comes from the caller's workspace, sized
 *     by nnconv_workspace_size) and never synchronises.
 *   - Work is queued on the caller's HIP stream (hipStream_t passed as
 *     void*; NULL means the default stream).  Calls return once queued.
 *     They queue kernel launches only (no memset, copy or event), so a
 *     sequence of calls may be captured into a HIP graph and replayed.
 *   - The library keeps no mutable global state (the one exception is the
 *     scratch array of nnconv_wgrad_noalloc, see there): calls are
 *     reentrant, and calls on different streams with disjoint buffers may
 *     run concurrently.
 *   - Fast (matrix-core) paths need 16-byte aligned pointers and Cg, Kg that
 *     are multiples of 8, or one group: other channel counts are then padded
 *     with zero channels in the workspace (operands that are copied for it
 *     may have any alignment) where that is the faster way.  Other valid
 *     shapes, and layers of a few channels that padding would slow down, run
 *     on direct kernels with identical semantics.
 *   - Depthwise convolution (groups == c == k, one channel per group, the
 *     MobileNet / EfficientNet layers trained with the paper's framework)
 *     with c a multiple of 8, a square 3x3, 5x5 or 7x7 filter and 16-byte
 *     aligned activations runs on dedicated kernels: stride 1 without
 *     dilation on the matrix cores, with diagonal weight matrices, where an
 *     estimate of both kernels' times says so (large enough grids and well
 *     filled tiles; forward and backward-data of 3x3 filters only in bf16 with
 *     outputs 9 to 16 wide; backward-weight of 3x3 filters up to 16 wide and
 *     of 5x5 ones, from 96 workgroups up), the rest on the vector ALUs.  w and
 *     dw are [K][R][S] in both layouts (one channel per filter).
 *   - Grouped convolution with m = C/groups = K/groups channels per group,
 *     m < 64 dividing 64 and c a multiple of 64 (e.g. 32 groups of 4-32
 *     channels) runs as groups of 64 channels with block-diagonal weights on
 *     the matrix-core kernels.  Results for finite inputs are those of the
 *     grouped convolution; a non-finite input value also makes the outputs
 *     of the other groups sharing its 64-channel block NaN.
 *   - Non-finite inputs: forward and backward-weight multiply the zeros of
 *     the zero-extended input at taps outside the image, as the definition
 *     reads, so an inf or NaN weight (forward) or dy (backward-weight) makes
 *     every sum it meets non-finite, padding included.  Backward-data has
 *     only the terms the adjoint definition has: where the matrix-core and
 *     depthwise kernels read dy zero-extended, a weight scan queued with
 *     the call has the border pixels recomputed from the definition when
 *     any weight is inf or NaN (small-group convolution excepted, above).
 *
 * Errors: every argument check happens on the host before anything is
 * queued.  On a non-OK status nothing is launched and no output or
 * workspace byte is touched.  No exception crosses the ABI and nothing is
 * printed.
 */
#ifndef NNCONV_H
#define NNCONV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define NNCONV_VERSION 1

typedef enum {
    NNCONV_OK = 0,
    NNCONV_ERR_INVALID_ARG = 1,   /* bad shape, null pointer, bad enum */
    NNCONV_ERR_UNSUPPORTED = 2,   /* valid but not provided (e.g. dtype combination) */
    NNCONV_ERR_WORKSPACE = 3,     /* ws_bytes smaller than nnconv_workspace_size() */
    NNCONV_ERR_MISALIGNED = 4,    /* pointer alignment below the element size */
    NNCONV_ERR_HIP = 5            /* the HIP runtime refused a launch */
} nnconv_status;

typedef enum { NNCONV_NCHW = 0, NNCONV_NHWC = 1 } nnconv_layout;
/* NNCONV_F8: the 8-bit moments of nnconv_adamw_update only. */
typedef enum { NNCONV_F16 = 0, NNCONV_BF16 = 1, NNCONV_F32 = 2, NNCONV_F8 = 3 } nnconv_dtype;
typedef enum { NNCONV_FWD = 0, NNCONV_DGRAD = 1, NNCONV_WGRAD = 2 } nnconv_pass;

/* Convolution geometry (the parameters of the paper's convolution call plus
 * stride, padding, dilation, groups, layout and operand type). */
typedef struct {
    int32_t n, c, h, w;          /* batch, input channels, input height, width */
    int32_t k, r, s;             /* output channels, filter height, width */
    int32_t stride_h, stride_w;  /* >= 1 */
    int32_t pad_h, pad_w;        /* >= 0, zero padding on both sides */
    int32_t dil_h, dil_w;        /* >= 1 */
    int32_t groups;              /* >= 1, divides c and k */
    int32_t layout;              /* nnconv_layout */
    int32_t dtype;               /* nnconv_dtype of x, w, y, dy, dx: F16 or BF16 */
} nnconv_desc;

/* Library version (NNCONV_VERSION). */
int32_t nnconv_version(void);

/* The hipError_t code behind the most recent NNCONV_ERR_HIP returned on the
 * calling thread (0 if there was none). */
int32_t nnconv_last_hip_error(void);

/* Static, human-readable name of a status code. */
const char *nnconv_status_string(nnconv_status status);

/* Output size (P, Q) from the floor formula above.
 * INVALID_ARG for a null argument, non-positive sizes, negative padding,
 * groups not dividing c and k, or an empty output. */
nnconv_status nnconv_output_dims(const nnconv_desc *desc, int32_t *p, int32_t *q);

/* Bytes of device workspace that nnconv_fwd / nnconv_dgrad / nnconv_wgrad
 * need for this geometry (0 is a valid answer).  Depends only on desc and
 * pass.  Workspace contents need not be initialised and are garbage after
 * the call.  With one group and a channel count that is not a multiple of 8
 * the answer covers channel-last copies with padded channels for the
 * matrix-core kernels; such a call also accepts less, down to nothing
 * (forward, backward-data) or the direct kernel's fp32 partials
 * (backward-weight: up to 64 of dw), and then runs on the slow direct
 * kernels (backward-weight without the copies' room but with the partials':
 * on the same kernels, slower, with the same results). */
nnconv_status nnconv_workspace_size(const nnconv_desc *desc, nnconv_pass pass, size_t *bytes);

/* Forward pass (definition above): y = alpha * conv(x, w).
 * x, w, y: device pointers in desc->layout, element type desc->dtype.
 * Accumulation in fp32; y is rounded to nearest-even once, overflow gives
 * +-inf.  y must not overlap x, w or ws. */
nnconv_status nnconv_fwd(const nnconv_desc *desc, const void *x, const void *w, void *y,
                         float alpha, void *ws, size_t ws_bytes, void *hip_stream);

/* Backward-data pass: dx = alpha * (adjoint in x)(dy).  dy carries the
 * loss scale and dx keeps it.  Input positions that no output reads get an
 * exact 0.  dx must not overlap dy, w or ws. */
nnconv_status nnconv_dgrad(const nnconv_desc *desc, const void *dy, const void *w, void *dx,
                           float alpha, void *ws, size_t ws_bytes, void *hip_stream);

/* Tiles of the matrix-core implicit GEMM that runs the forward pass and the
 * backward-data pass when the reduction channels per filter tap (Cg for the
 * forward pass, Kg for backward-data) are a multiple of 64.  nnconv_fwd and
 * nnconv_dgrad pick one per shape; the _tile variants below force one, for
 * tests that must reach every tile on small shapes and for tuning.  Every
 * tile computes the same sums (the fp32 summation order may differ). */
typedef enum {
    NNCONV_TILE_256x256_8W = 0,   /* 8 waves of 128x64, 2 stages of 64-element slices */
    NNCONV_TILE_128x128_2S = 1,   /* 4 waves of 64x64, 2 stages */
    NNCONV_TILE_128x128 = 2,      /* 4 waves of 64x64, single stage */
    NNCONV_TILE_128x64 = 3,       /* 4 waves of 64x32, single stage */
    NNCONV_TILE_256x256_16W = 4,  /* 16 waves of 64x64, 2 stages */
    NNCONV_TILE_256x256_RING = 6, /* 4 waves of 128x128, ring of 4 32-element slices */
    NNCONV_TILE_256x128_RING = 7, /* 4 waves of 128x64, ring of 3 */
    NNCONV_TILE_256x64_RING = 8,  /* 4 waves of 64x64, ring of 4 */
    /* Halo staging, for stride-1 geometries whose input image has the
     * output's size and whose taps shift a pixel by at most 64 raster
     * positions (3x3 filters with padding 1 on images up to 63 pixels
     * wide; backward-data of the same at stride 1): 256-pixel tiles, each
     * 64-channel slice of the input staged once per tile for all taps. */
    NNCONV_TILE_HALO_256x64 = 9,    /* 4 waves of 64x64 */
    NNCONV_TILE_HALO_256x128 = 10,  /* 4 waves of 128x64 */
    NNCONV_TILE_HALO_256x64_2T = 11, /* 256x64, B tiles of two taps per barrier */
    /* Halo staging with the weight fragments loaded from L2 straight into
     * registers several taps ahead and the next channel slice's halo loading
     * during the current one (one workgroup per CU unless stated). */
    NNCONV_TILE_HALO_R256x128 = 12, /* 4 waves of 128x64; taps within 64 raster
                                       positions (3x3 on images up to 31 wide) */
    NNCONV_TILE_HALO_R128x256 = 13, /* 4 waves of 128x64 side by side */
    NNCONV_TILE_HALO_R224x256 = 14, /* 4 waves of 224x64 side by side; taps within
                                       32 raster positions (3x3 up to 15 wide) */
    NNCONV_TILE_HALO_R256x64S = 15  /* 4 waves of 64x64, a single 64-channel
                                       reduction slice (Cg = 64 forward, Kg = 64
                                       backward-data), two workgroups per CU */
} nnconv_tile;

/* nnconv_fwd / nnconv_dgrad with the tile forced (an nnconv_tile value).
 * Same arguments, semantics and errors, plus: INVALID_ARG for a negative
 * tile; UNSUPPORTED when the tile is not one of nnconv_tile, or when the
 * call would not run on the implicit-GEMM kernel (reduction channels per tap
 * not a multiple of 64, depthwise or small-group convolution, the stem's
 * 8- and 4-channel shapes, operands not 16-byte aligned or past 2 GiB, backward-data
 * with more than 4 stride phases), and for a halo tile on any other geometry
 * than the one it states or on grouped convolution. */
nnconv_status nnconv_fwd_tile(const nnconv_desc *desc, const void *x, const void *w, void *y,
                              float alpha, void *ws, size_t ws_bytes, void *hip_stream,
                              int32_t tile);
nnconv_status nnconv_dgrad_tile(const nnconv_desc *desc, const void *dy, const void *w, void *dx,
                                float alpha, void *ws, size_t ws_bytes, void *hip_stream,
                                int32_t tile);

/* Backward-weight pass with the loss-scale step of Sec. 3.3 / Listing 6:
 *   dw = (accumulate ? dw : 0) + inv_loss_scale * sum_{n,p,q} dy * xz
 * The batch-pixel reduction is split over the workspace in fp32 and summed
 * in a fixed order, so results are bitwise reproducible.
 * dw_dtype: NNCONV_F32 (for fp32 master weights) or desc->dtype.
 * accumulate: 0 overwrites dw (its old contents are not read), 1 adds.
 * overflow_flag: NULL or a device int32 that the caller zeroed; the call
 *   stores 1 into it when any final dw element is inf or NaN and never
 *   clears it (one flag can cover every layer of a step, as
 *   check_inf_or_nan_grad does in Listing 6). */
nnconv_status nnconv_wgrad(const nnconv_desc *desc, const void *x, const void *dy, void *dw,
                           int32_t dw_dtype, float inv_loss_scale, int32_t accumulate,
                           int32_t *overflow_flag, void *ws, size_t ws_bytes, void *hip_stream);

/* For callers that cannot allocate device memory or size a workspace --
 * code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc: nnconv_wgrad with the workspace taken from a library-owned
 * scratch array of NNCONV_NOALLOC_WS_BYTES (64 MiB) instead of an argument.
 * Same arguments (minus ws, ws_bytes), semantics, results (bitwise equal to
 * nnconv_wgrad's with the workspace that nnconv_workspace_size asks for) and
 * errors, plus NNCONV_ERR_WORKSPACE, returned before anything is queued, when
 * the geometry needs more workspace than the scratch holds
 * (nnconv_workspace_size(desc, NNCONV_WGRAD) > NNCONV_NOALLOC_WS_BYTES;
 * channel counts that are not multiples of 8, with one group, need no room for
 * copies there; every channel-last ResNet-50 layer at batch 256 fits).
 *   - The scratch is a device array of the library: every GPU the library
 *     runs on holds one copy from the first call on it (made with that GPU
 *     current, outside graph capture) until the process ends.  The call
 *     itself allocates nothing.
 *   - Every call on one GPU shares that GPU's copy, which keeps the last
 *     call's contents; nothing in it needs to start at zero.  Calls that
 *     overlap on one GPU (several streams or threads without ordering)
 *     race on it: order them on one stream. */
#define NNCONV_NOALLOC_WS_BYTES (64 * 1024 * 1024)
nnconv_status nnconv_wgrad_noalloc(const nnconv_desc *desc, const void *x, const void *dy,
                                   void *dw, int32_t dw_dtype, float inv_loss_scale,
                                   int32_t accumulate, int32_t *overflow_flag,
                                   void *hip_stream);

/* Layout transforms (pure data movement of 16-bit elements, bit exact).
 *
 * The paper's convolution call takes its channels on axis 1 (base_axis = 1
 * in Sec. 3.2, Listing 5), i.e. [N][C][H][W] activations with [K][Cg][R][S]
 * weights, stored in half precision (Sec. 3.3).  The matrix-core kernels
 * read channel-last tensors, where one 16-byte load is 8 consecutive
 * channels of a pixel; these calls move data between the two forms (the
 * NCHW entry points above use them internally through the workspace) and
 * pad the channel count of the 3-channel input image to 4 (or 8) for the
 * stem.
 * All pointers are caller-owned device memory; src and dst must not
 * overlap.  INVALID_ARG for null pointers or non-positive sizes (or a pad
 * below the channel count); MISALIGNED for pointers not 2-byte aligned.
 *
 * Activations: src[N][C][H][W] -> dst[N][H][W][c_pad], c_pad >= C; channels
 * C..c_pad-1 of dst are zero (the stem's 3 channels padded to 4). */
nnconv_status nnconv_nchw_to_nhwc(const void *src, void *dst, int32_t n, int32_t c, int32_t h,
                                  int32_t w, int32_t c_pad, void *hip_stream);

/* Activations: src[N][H][W][C] -> dst[N][C][H][W]. */
nnconv_status nnconv_nhwc_to_nchw(const void *src, void *dst, int32_t n, int32_t c, int32_t h,
                                  int32_t w, void *hip_stream);

/* Channel padding in channel-last form: src[rows][c] -> dst[rows][c_pad],
 * extra channels zero (rows = N*H*W). */
nnconv_status nnconv_pad_channels(const void *src, void *dst, int64_t rows, int32_t c,
                                  int32_t c_pad, void *hip_stream);

/* Weights: src[K][Cg][R][S] -> dst[K][R][S][cg_pad], cg_pad >= Cg, padding
 * zero. */
nnconv_status nnconv_weight_kcrs_to_krsc(const void *src, void *dst, int32_t k, int32_t cg,
                                         int32_t r, int32_t s, int32_t cg_pad, void *hip_stream);

/* Weights: src[K][R][S][Cg] -> dst[K][Cg][R][S]. */
nnconv_status nnconv_weight_krsc_to_kcrs(const void *src, void *dst, int32_t k, int32_t cg,
                                         int32_t r, int32_t s, void *hip_stream);

/* Training-step pieces after the backward passes (Sec. 3.3, Listing 6).
 *
 * A step with dynamic loss scaling, all on one stream and with no host
 * synchronisation:
 *   1. the caller seeds dy of the loss with the current scale S (it can read
 *      S from the device state below, e.g. as a 0-d tensor view);
 *   2. nnconv_wgrad for every layer with inv_loss_scale = 1, dw_dtype F32
 *      and one shared overflow flag (zeroed once, at set-up);
 *   3. nnconv_sgd_update for every parameter array, passing the state and
 *      the flag: it divides the gradient by S and does nothing at all when
 *      the flag is set;
 *   4. nnconv_loss_scaler_update once: it advances the scaler by the flag
 *      and clears the flag for the next step.
 * The order 3-before-4 matters: the update uses the scale the gradients
 * were computed with, and the scale only grows afterwards, as in the
 * listing. */

/* Device-resident dynamic loss-scaler state (24 bytes, caller-owned device
 * memory, 4-byte aligned).  Readable by the caller at any time; written
 * only by the two calls below. */
typedef struct {
    float scale;      /* current loss scale S */
    float factor;     /* growth / shrink factor (2 in the paper) */
    int32_t interval; /* clean steps between growths (2000 in the paper) */
    int32_t counter;  /* clean steps since the last growth or overflow */
    int32_t skipped;  /* steps skipped because of an inf or NaN gradient */
    int32_t reserved; /* zero */
} nnconv_loss_scaler;

/* Queues the initialisation of *state: scale = initial_scale, factor,
 * interval, counter = skipped = 0.
 * INVALID_ARG: null state, initial_scale or factor not finite and > 0,
 * interval < 0.  MISALIGNED: state not 4-byte aligned. */
nnconv_status nnconv_loss_scaler_init(nnconv_loss_scaler *state, float initial_scale,
                                      float factor, int32_t interval, void *hip_stream);

/* One step of the dynamic scaler of Listing 6, driven by *overflow_flag (a
 * device int32, nonzero = this step's gradients held an inf or a NaN):
 *   flag set:   scale /= factor; counter = 0; skipped += 1
 *   flag clear: if counter > interval { scale *= factor; counter = 0 }
 *               counter += 1
 * and then *overflow_flag = 0.  The test runs before the increment, so with
 * interval 2000 the first growth comes on the 2002nd consecutive clean step
 * and later ones every 2001 clean steps.  One thread; queue it after every
 * nnconv_sgd_update of the step.
 * INVALID_ARG: null pointer.  MISALIGNED: either pointer not 4-byte
 * aligned. */
nnconv_status nnconv_loss_scaler_update(nnconv_loss_scaler *state, int32_t *overflow_flag,
                                        void *hip_stream);

/* fp32 master-weight update (Sec. 3.3: 16-bit working weights, fp32 master
 * copy updated in fp32).  The paper names no solver; this is momentum SGD
 * with L2 weight decay, element-wise over count entries:
 *   g = grad / S + weight_decay * master      (S = state->scale, 1 if NULL)
 *   momentum = momentum_coef * momentum + g
 *   master  -= lr * momentum
 *   w16      = round-to-nearest-even(master)  (when w16 is not NULL)
 * computed in fp32 (1/S taken once, so a power-of-two S is exact).
 * master, momentum, grad: device fp32 arrays of count elements, in any
 * common element order (the nnconv_wgrad dw order of the layer's layout
 * matches the weights).  w16: NULL or device array of count elements of
 * w16_dtype (F16 or BF16), e.g. the layer's weights for the next forward.
 * overflow_flag: NULL or the step's device flag; when it is nonzero the
 * call changes nothing (the step is skipped).  The flag is only read.
 * In-place; master, momentum, grad and w16 must not overlap.  count = 0 is
 * a no-op.  16-byte aligned arrays and count % 4 == 0 take a vectorised
 * path.
 * INVALID_ARG: count < 0, null master/momentum/grad, w16_dtype not F16 or
 * BF16 when w16 is given.  MISALIGNED: fp32 arrays or state/flag not 4-byte
 * aligned, w16 not 2-byte aligned. */
nnconv_status nnconv_sgd_update(int64_t count, float *master, float *momentum, void *w16,
                                int32_t w16_dtype, const float *grad,
                                const nnconv_loss_scaler *state, const int32_t *overflow_flag,
                                float lr, float momentum_coef, float weight_decay,
                                void *hip_stream);

/* Operators of a gated sequence block on channel-last tokens.
 *
 * A sequence of t tokens with c channels is an NHWC image of height 1 and
 * width t, and a projection of its channels is a 1x1 convolution, so that
 * nnconv_fwd, nnconv_dgrad and nnconv_wgrad are the block's matrix products.
 * The calls below are what stands between them, and the solver that such
 * blocks are trained with.  They follow the conventions above: caller-owned
 * buffers, kernel launches only, gradients that carry the loss scale, and
 * parameter gradients in fp32 with inv_loss_scale, accumulate and
 * overflow_flag as nnconv_wgrad has them.  Sums, statistics and states are
 * fp32; every 16-bit output is rounded once, to nearest even.  Results are
 * bitwise reproducible for given sizes and inputs. */

/* Root-mean-square norm over the channels of each row, with the residual's
 * addition in front:
 *   r     = x + residual, rounded to dtype  (x itself without a residual)
 *   rstd  = 1 / sqrt(mean over c of r^2 + eps)
 *   y     = gain * r * rstd
 * The norm reads r as it is stored, so that the backward pass, which reads
 * the stored r, is the gradient of what was computed.  Rows are dense: [rows][c]. */
typedef struct {
    int64_t rows;   /* >= 0: N*H*W of a channel-last activation, or tokens; 0 is a no-op */
    int32_t c;      /* channels, 1 to 2^28 */
    int32_t dtype;  /* F16 or BF16: x, residual, sum, y, dy, dsum, dx */
    int32_t group;  /* nnconv_rmsnorm_fwd_q8: channels with one scale, 32, 64 or 128;
                       0: one scale per row.  Others ignore it. */
    float eps;      /* finite, >= 0 */
} nnconv_rmsnorm_desc;

/* Forward: y and, where the pointers are not NULL, sum (= r) and rstd
 * (fp32, [rows], for the backward pass).  A row whose mean square passes fp32's
 * range has rstd 0, one below it with eps = 0 an infinite rstd.
 * residual: NULL or [rows][c].
 * gain: fp32, [c].  sum may be x or residual itself (updated in place);
 * nothing else may overlap an output.  A row of zeros with eps = 0 gives NaN,
 * as the formula does.  Any alignment of at least one element; 16-byte aligned
 * rows are the fast ones.
 * INVALID_ARG: rows < 0, c < 1, bad dtype, eps negative or not finite, null x,
 * gain or y.  UNSUPPORTED: dtype F32.  MISALIGNED: pointers below their
 * element size. */
nnconv_status nnconv_rmsnorm_fwd(const nnconv_rmsnorm_desc *desc, const void *x,
                                 const void *residual, const float *gain, void *sum, void *y,
                                 float *rstd, void *hip_stream);

/* Forward with y in 8 bits (e4m3: 4 exponent bits, 3 mantissa bits, largest
 * value 448, no infinities) and fp32 scales:
 *   scale = max |y| / 448 over the row, or over each group of `group` channels
 *           (the last group of a row may be short); 0 where that is below 2^-126
 *   q     = e4m3(y / scale), to nearest even, y unrounded; 0 where scale is 0
 * so that q * scale stands for y; y is in fp32, and both quotients are rounded to
 * fp32 as a division is.  q: [rows][c] bytes; scales:
 * [rows][ceil(c / group)], or [rows].  The maximum passes over NaN; a NaN y has
 * a NaN code, and an infinite y an infinite scale and a NaN code.  Otherwise as
 * nnconv_rmsnorm_fwd; INVALID_ARG too for another group and null scales. */
nnconv_status nnconv_rmsnorm_fwd_q8(const nnconv_rmsnorm_desc *desc, const void *x,
                                    const void *residual, const float *gain, void *sum, void *q,
                                    float *scales, float *rstd, void *hip_stream);

/* Bytes of workspace of nnconv_rmsnorm_bwd. */
nnconv_status nnconv_rmsnorm_workspace_size(const nnconv_rmsnorm_desc *desc, size_t *bytes);

/* Backward, with xh = r * rstd:
 *   dx    = dsum + rstd * (dy * gain - xh * mean over c of (dy * gain * xh))
 *   dgain = (accumulate ? dgain : 0) + inv_loss_scale * sum over rows of dy * xh
 * sum and rstd are the forward's (sum is x without a residual).  dsum: NULL
 * (taken as 0) or the gradient that reaches r along the residual stream.
 * dx is the gradient of r, hence of x and of residual alike; it may be dy or
 * dsum itself.  dgain (fp32, [c]) may be NULL: then it is left out.  ws needs
 * 4-byte alignment.
 * Errors as nnconv_rmsnorm_fwd's, and as nnconv_wgrad's for accumulate and ws. */
nnconv_status nnconv_rmsnorm_bwd(const nnconv_rmsnorm_desc *desc, const void *sum, const void *dy,
                                 const void *dsum, const float *gain, const float *rstd, void *dx,
                                 float *dgain, float inv_loss_scale, int32_t accumulate,
                                 int32_t *overflow_flag, void *ws, size_t ws_bytes,
                                 void *hip_stream);

/* Gated linear recurrence over the tokens of each sequence, channel by channel:
 *   z_t = f_t + bias, limited to [-80, 80];  a_t = 1 / (1 + exp(-z_t))
 *   h_t = a_t * h_(t-1) + (1 - a_t) * x_t,   h_0 = h0
 *   y_t = h_t * g_t / (1 + exp(-g_t))        (y_t = h_t without g)
 * The limit keeps both a and 1 - a above 0, so that a gate never makes a NaN
 * of an infinite state; a NaN passes through.  One channel (c = 1) is walked
 * token by token, a sequence a lane. */
typedef struct {
    int32_t n;      /* sequences, >= 0 */
    int32_t t;      /* tokens of each, >= 0 */
    int32_t c;      /* channels, 1 to 2^28 */
    int32_t dtype;  /* F16 or BF16: x, f, g, y and their gradients */
    int64_t ld;     /* elements from a token to the next in x, f, g, dx, df, dg, >= c:
                       3 * c where they are thirds of one projection's output */
    int64_t ldy;    /* the same in y and dy, >= c */
} nnconv_recurrence_desc;

/* Tokens between two states that the forward pass saves for the backward. */
#define NNCONV_RECURRENCE_SAVE 64

/* Bytes of `saved`: fp32 [n][ceil(t / NNCONV_RECURRENCE_SAVE)][c]. */
nnconv_status nnconv_recurrence_saved_size(const nnconv_recurrence_desc *desc, size_t *bytes);

/* Bytes of workspace of nnconv_recurrence_fwd (NNCONV_FWD) or
 * nnconv_recurrence_bwd (NNCONV_DGRAD). */
nnconv_status nnconv_recurrence_workspace_size(const nnconv_recurrence_desc *desc,
                                               nnconv_pass pass, size_t *bytes);

/* Forward.  x, f, g (may be NULL): token j of sequence i starts at element
 * (i * t + j) * ld; y with ldy.  bias: fp32, [c], or NULL.  lengths: NULL or
 * device int32 [n], taken into 0..t: tokens from the length on leave the
 * state as it is and have y = 0 (their x, f and g may hold anything).
 * h0: fp32 [n][c], NULL for zeros.  ht: NULL or fp32 [n][c], the state after
 * the last token; it may be h0 itself: with t = 1 a call is one step of
 * serving.  saved: NULL or what nnconv_recurrence_bwd needs.  No other output
 * may overlap anything.  ws: 8-byte aligned; calls that may overlap in time
 * need workspaces of their own.
 * INVALID_ARG: sizes below the limits above, bad dtype, null x, f or y;
 * UNSUPPORTED: dtype F32, more channels, a sequence of more than 2^36 elements or
 * 2^29 tokens; WORKSPACE; MISALIGNED: pointers below their element
 * size (ws: below 8). */
nnconv_status nnconv_recurrence_fwd(const nnconv_recurrence_desc *desc, const void *x,
                                    const void *f, const float *bias, const void *g,
                                    const int32_t *lengths, const float *h0, void *y, float *ht,
                                    float *saved, void *ws, size_t ws_bytes, void *hip_stream);

/* Backward.  saved is the forward's.  dy: the gradient of y; dht: NULL or that
 * of the last state.  With dh_t the gradient of h_t (its own y's and the next
 * state's):
 *   dx_t = (1 - a_t) dh_t,  df_t = a_t (1 - a_t) (h_(t-1) - x_t) dh_t,
 *   dg_t = dy_t h_t d(g sigma(g))/dg,  dh0 = a_1 dh_1,
 *   dbias = (accumulate ? dbias : 0) + inv_loss_scale * sum over tokens of df
 * (df unrounded in the sum; the limit of z counts as the identity).  Tokens
 * from the length on have zero gradients.  dx, df and, where g is given, dg
 * are written; dh0 (fp32 [n][c], may be dht itself) and dbias (fp32 [c]) may be
 * NULL.  Errors as the forward's and as nnconv_wgrad's for accumulate; null
 * saved, dy, dx, df, or dg where g is given: INVALID_ARG. */
nnconv_status nnconv_recurrence_bwd(const nnconv_recurrence_desc *desc, const void *x,
                                    const void *f, const float *bias, const void *g,
                                    const int32_t *lengths, const float *saved, const void *dy,
                                    const float *dht, void *dx, void *df, void *dg, float *dh0,
                                    float *dbias, float inv_loss_scale, int32_t accumulate,
                                    int32_t *overflow_flag, void *ws, size_t ws_bytes,
                                    void *hip_stream);

/* AdamW over many tensors in one launch, in place of nnconv_sgd_update in the
 * step above (and like it before nnconv_loss_scaler_update): with t the
 * number of steps taken including this one and S the loss scale,
 *   g = grad / S,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   master -= lr (m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps)
 *                 + weight_decay * master)
 *   w16 = round-to-nearest-even(master)
 * in fp32, with m and v unrounded in the master's update (0 / 0, with eps = 0
 * and a v of 0, is NaN).
 *
 * state_dtype F32: m and v are fp32 arrays.  F8: m is e4m3 (largest 448) and
 * v e5m2 (largest 57344) codes, with one power of two for every
 * NNCONV_ADAMW_BLOCK elements (m_scale, v_scale: bytes e that stand for
 * 2^(e - 127), ceil(count / NNCONV_ADAMW_BLOCK) of them): the smallest one
 * that brings the block's largest finite magnitude within range (0 for a block of
 * zeros).  A change of v by 0.1 % is far below a code's spacing, and rounding to nearest
 * would lose it in every step; codes are therefore rounded up or down at
 * random, up with the probability of the part lost, so that they are right on
 * average.  The random numbers are a hash of (seed, t, index of the tensor in the list,
 * element), so a step can be repeated.  A v above 0 keeps a code above 0.
 * A power of two as the scale keeps the codes' grid in place from step to
 * step.  A value that is not finite has a NaN code. */
#define NNCONV_ADAMW_BLOCK 64
typedef struct {
    float *master;        /* fp32, [count] */
    const void *grad;     /* [count] of grad_dtype, loss-scaled */
    void *w16;            /* NULL or [count] of w16_dtype: the working copy */
    void *m, *v;          /* [count] of state_dtype */
    uint8_t *m_scale, *v_scale; /* state_dtype F8 only */
    int64_t count;        /* >= 0 */
    float weight_decay;   /* finite */
    int32_t grad_dtype;   /* F32, F16 or BF16 */
    int32_t w16_dtype;    /* F16 or BF16 (ignored without w16) */
    int32_t state_dtype;  /* F32 or F8 */
} nnconv_adamw_tensor;

/* A list of tensors laid out for nnconv_adamw_update.  Filled by
 * nnconv_adamw_plan_init; holds no memory of its own. */
typedef struct {
    void *table;       /* the caller's device buffer */
    int64_t chunks;
    int32_t tensors;
    int32_t reserved;
} nnconv_adamw_plan;

/* Bytes of device memory for the plan of `n` tensors. */
nnconv_status nnconv_adamw_plan_size(const nnconv_adamw_tensor *tensors, int32_t n, size_t *bytes);

/* Checks the list (a host array, not needed after the call), fills *plan and
 * queues kernels that write the list to `table`, which has to
 * live as long as the plan is used.  Once per set of tensors.
 * INVALID_ARG: n < 0, null or negative members, bad dtypes, weight decay not
 * finite; MISALIGNED: members below their element size, table below 16;
 * WORKSPACE: table_bytes too small. */
nnconv_status nnconv_adamw_plan_init(const nnconv_adamw_tensor *tensors, int32_t n, void *table,
                                     size_t table_bytes, nnconv_adamw_plan *plan,
                                     void *hip_stream);

/* One step.  step: device int32, the number of steps taken so far (0 at
 * first); the call adds 1.  state: the loss scaler's, or NULL (S = 1).
 * overflow_flag: NULL or the step's device flag; where it is set the call
 * changes nothing, step included.  Calls that may overlap in time need plans
 * of their own.
 * INVALID_ARG: null plan or step, lr or eps negative or not finite, betas outside
 * [0, 1). */
nnconv_status nnconv_adamw_update(const nnconv_adamw_plan *plan, int32_t *step, float lr,
                                  float beta1, float beta2, float eps, uint32_t seed,
                                  const nnconv_loss_scaler *state, const int32_t *overflow_flag,
                                  void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* NNCONV_H */
