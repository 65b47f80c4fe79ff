/*
 * snip.h -- C ABI of the MI355X (gfx950) library for the quantized linear-layer hot path
 * of SNIP (arXiv 2602.01410).
 *
 * The library implements what runs on every GPU in every training step of a mixed-precision
 * linear layer (paper Sec. 2.2, Fig. "mixed precision training"): the inputs, weights and
 * output gradients are quantized to FP8 or FP4 before each of the three GEMMs
 *     forward      Y [M,N] = X [M,K] * W[N,K]^T
 *     data grad    dX[M,K] = dY[M,N] * W[N,K]
 *     weight grad  dW[N,K] = dY[M,N]^T * X[M,K]
 * (shapes as in Sec. 4.1 / 4.3.1), the GEMM output stays in BF16, and the Frobenius norms of
 * the tensors and of their quantization error are collected (Sec. 3.1, Step 1) as input to
 * the loss- and weight-divergence estimates of Sec. 4.  Which format each operand uses is the
 * per-layer decision of the paper's ILP (Sec. 4.2); here it arrives as a snip_layer_plan.
 *
 * Quantization (Sec. 2.3): every group of 32 consecutive elements along the contraction
 * dimension of the consuming GEMM shares one power-of-two scale 2^e stored as an E8M0 byte
 * (value 2^(byte-127)); elements are FP8 E4M3 (no infinities, max 448) or FP4 E2M1 (max 6),
 * rounded to nearest with ties to the even mantissa.  This is the paper's
 * "scale = FPX_MAX / max|x|" with the scale restricted to a power of two.
 *
 * General conventions
 *  - Every pointer argument marked "device" is GPU memory owned by the caller; the library
 *    never allocates, frees or keeps a pointer, and holds no global state.
 *  - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All work is
 *    enqueued on it; no call synchronizes.  Outputs are valid once the stream has reached
 *    the end of the call.
 *  - Arguments are validated on the host before anything is launched: a call that returns
 *    an error has had no effect.  Errors are reported by return code only.
 *  - Calls are re-entrant; calls on different streams may overlap if their outputs and
 *    workspaces do not.
 *  - Blocks that contain an infinity or a NaN get scale byte 0xFF and all-zero codes; no
 *    error is raised for them.
 */
#ifndef SNIP_H
#define SNIP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SNIP_OK = 0,
    SNIP_ERR_NULL = 1,       /* a required pointer is NULL */
    SNIP_ERR_SHAPE = 2,      /* negative extent, blocked extent not a multiple of 32, ld too small */
    SNIP_ERR_FORMAT = 3,     /* unknown enum value, or an operand's format differs from the plan */
    SNIP_ERR_LAYOUT = 4,     /* misaligned pointer / leading dimension, operands' contraction extents differ */
    SNIP_ERR_WORKSPACE = 5,  /* workspace missing or too small */
    SNIP_ERR_HIP = 6         /* a kernel launch failed */
} snip_status;

typedef enum { SNIP_FP8_E4M3 = 0, SNIP_FP4_E2M1 = 1 } snip_fmt;

/* Direction of the 32-element blocks in the SOURCE matrix. */
typedef enum {
    SNIP_AXIS_ROW = 0,       /* along a row (contiguous elements); stored matrix = source */
    SNIP_AXIS_COL = 1        /* down a column; stored matrix = transpose of the source */
} snip_axis;

/* How the power-of-two scale 2^e is derived from the block maximum amax = m * 2^n, 1 <= m < 2. */
typedef enum {
    SNIP_SCALE_NO_OVERFLOW = 0, /* smallest 2^e with amax / 2^e <= FPX_MAX (the paper's scale,
                                   rounded so that the block maximum stays representable) */
    SNIP_SCALE_OCP_FLOOR = 1    /* e = n - emax(FPX); elements above FPX_MAX saturate */
} snip_scale_rule;

typedef enum { SNIP_OUT_BF16 = 0, SNIP_OUT_FP32 = 1 } snip_out_dtype;

/* Scaling groups of the paper's own recipe, in the stored orientation. */
typedef enum {
    SNIP_GROUP_TILE_1x128 = 1,      /* 128 consecutive elements of a stored row (activations, gradients) */
    SNIP_GROUP_BLOCK_128x128 = 128  /* 128 stored rows x 128 elements (weights) */
} snip_group;

/* A quantized matrix in its stored orientation: `cols` is the blocked (contraction) extent.
 *   codes : device. FP8: rows*cols bytes, row-major. FP4: rows*cols/2 bytes, row-major, element
 *           2i in the low nibble and 2i+1 in the high nibble of byte i. 16-byte aligned.
 *   scales: device. E8M0 bytes, [rows][cols/32] row-major. 4-byte aligned.
 *   scales_g4: device or NULL.  A second copy of the same scale bytes, grouped for the GEMMs:
 *           [ceil(cols/128)][rows_pad][4], i.e. the four scales of 128 consecutive contraction
 *           elements of a row in one dword, rows contiguous; rows_pad = rows rounded up to a
 *           multiple of 256 (dwords of rows >= `rows`, and bytes of blocks >= cols/32, are
 *           unspecified).  16-byte aligned (the quantize kernels write it with 16-byte stores;
 *           SNIP_ERR_LAYOUT otherwise).  snip_quantize fills it when it is not NULL; when both
 *           operands of a GEMM carry one the GEMM copies its scales from it with fully coalesced loads,
 *           otherwise it falls back to a slower kernel that gathers from `scales`.  Size: snip_qtensor_scale_g4_bytes.
 *   rows, cols: extents of the stored matrix; cols must be a multiple of 32. */
typedef struct {
    void*    codes;
    uint8_t* scales;
    uint8_t* scales_g4;
    int64_t  rows, cols;
    int32_t  fmt;            /* snip_fmt */
} snip_qtensor;

/* Element format of each operand of each GEMM of one linear layer.  The paper's option set
 * (Sec. 4.2: one format each for inputs, weights, gradients) is the special case
 * fwd_x == wgrad_x, fwd_w == dgrad_w, dgrad_dy == wgrad_dy. */
typedef struct {
    int32_t fwd_x, fwd_w, dgrad_dy, dgrad_w, wgrad_dy, wgrad_x;   /* snip_fmt each */
} snip_layer_plan;

/* Squared Frobenius norms (Sec. 3.1 Step 1): of the tensor, and of q(x) - x for both candidate
 * formats.  A fused quantize call fills sum_sq and the chosen format's field and writes NaN
 * into the other.
 * Range: differences are exact and squares are formed and added per lane in fp32 (wave sums in
 * fp32, everything above in double), so the stated 1e-5 relative accuracy
 * holds for tensors whose nonzero magnitudes lie within [2^-56, 2^48]: below, the squares of
 * the errors (about 2^-5 |x| for FP8) leave the fp32 normal range and count as less than they
 * are; above, sums of squares overflow to infinity.  A lane adds at most rows / 64 (column
 * blocks) or cols / 8 (row blocks) groups of 8 elements before its sum moves to the next level
 * (squared differences one by one, the elements' own squares in pairs, or 32 of a column's block
 * first where columns are only summed and not quantized),
 * which keeps the rounding of a sum of n equal terms below 1e-5 up to about 2^22 rows. */
typedef struct { double sum_sq, err_sq_fp4, err_sq_fp8; } snip_stats;

/* ---- sizes (host, pure) ------------------------------------------------------------- */

/* Bytes of codes / scales for a stored matrix of rows x cols; 0 on a bad argument. */
size_t snip_qtensor_code_bytes(int64_t rows, int64_t cols, snip_fmt fmt);
size_t snip_qtensor_scale_bytes(int64_t rows, int64_t cols);
size_t snip_qtensor_scale_g4_bytes(int64_t rows, int64_t cols);

/* Workspace (device bytes) sufficient for any call below on a source matrix of at most
 * rows x cols, including per-line statistics. */
size_t snip_workspace_bytes(int64_t rows, int64_t cols);

/* ---- quantize (Sec. 2.3; which tensors: Sec. 2.2) ------------------------------------ */

/* Quantize a bf16 matrix.
 *   x     : device, bf16 [rows][ld], 16-byte aligned; ld >= cols, ld a multiple of 8.
 *   axis  : SNIP_AXIS_ROW: blocks along rows; cols % 32 == 0; out is rows x cols.
 *           SNIP_AXIS_COL: blocks down columns; rows % 32 == 0, cols even; out is stored
 *           transposed, cols x rows, so that it equals quantize(transpose(x), ROW).
 *   out   : host struct whose codes/scales point to device buffers of at least
 *           snip_qtensor_code_bytes / snip_qtensor_scale_bytes; out->rows, out->cols and
 *           out->fmt must already describe the stored matrix and `fmt`.
 *   stats : device or NULL.  If given, the squared norms of x and of the quantization error
 *           of `fmt` are produced by the same pass (then `workspace` is required).
 *   workspace: device, >= snip_workspace_bytes(rows, cols) bytes, 16-byte aligned; may be
 *           NULL when stats is NULL.
 * Column-block calls are worked on by one workgroup per 128-column unit; the environment variable
 * SNIP_QUANT_COL_UNIT=wave|workgroup, read at every call, fixes the work distribution for tests and
 * measurements (codes and scales do not depend on it; fused statistics are summed in another
 * fixed order). */
snip_status snip_quantize(const void* x, int64_t rows, int64_t cols, int64_t ld,
                          snip_fmt fmt, snip_axis axis, snip_scale_rule rule,
                          const snip_qtensor* out, snip_stats* stats,
                          void* workspace, size_t workspace_bytes, void* stream);

/* Which error sums the fused statistics of snip_quantize_both deliver. */
typedef enum { SNIP_STATS_CHOSEN_FORMAT = 0, SNIP_STATS_BOTH_FORMATS = 1 } snip_stats_scope;

/* Both orientations of one tensor from one pass over it (Sec. 2.2: every GEMM input is quantized
 * for two GEMMs that contract different axes, e.g. X along its rows for Y = X W^T and down its
 * columns for dW = dY^T X).  Produces exactly what
 *     snip_quantize(x, ..., out_row->fmt, SNIP_AXIS_ROW, rule, out_row, stats_row, ...) and
 *     snip_quantize(x, ..., out_col->fmt, SNIP_AXIS_COL, rule, out_col, stats_col, ...)
 * produce (codes, scales and grouped scale copies bit for bit; the statistics summed in another
 * fixed order), reading x from HBM once.  The two formats may differ.
 *   rows, cols: both multiples of 32; other arguments as for snip_quantize.
 *   out_row : stored rows x cols;  out_col : stored cols x rows.
 *   stats_row, stats_col: device, both or neither (SNIP_ERR_NULL for just one).
 *   scope   : SNIP_STATS_CHOSEN_FORMAT: as the fused statistics of snip_quantize (the field of the
 *             format not written is NaN).  SNIP_STATS_BOTH_FORMATS: all three fields, i.e. what
 *             snip_quant_error_stats_both delivers, out of the same pass: the complete Step-1
 *             record of a tensor (Sec. 3.1; the ILP needs the error of the option not in use,
 *             Sec. 4.2) together with its two quantized orientations from one read.  Ignored
 *             without statistics outputs.
 * A 128-column unit is worked on by one workgroup or, in calls with statistics on large tensors, by
 * one wave; the environment variable SNIP_QUANT_BOTH_UNIT=4x4|lds|4x8|wave (waves of a workgroup x
 * 32-row tiles of the unit they share; lds: 4x4 with the tiles copied into LDS first; a wave per unit),
 * read at every call, fixes the form where it exists for the call, =workgroup rules out a wave per unit; for tests and measurements (codes and scales
 * do not depend on it; the statistics are summed in another fixed order). */
snip_status snip_quantize_both(const void* x, int64_t rows, int64_t cols, int64_t ld,
                               snip_scale_rule rule, const snip_qtensor* out_row,
                               const snip_qtensor* out_col, snip_stats* stats_row,
                               snip_stats* stats_col, snip_stats_scope scope, void* workspace,
                               size_t workspace_bytes, void* stream);

/* Quantize to FP4 with stochastic rounding (Sec. 5.1 "Quantization Format and Implementation":
 * FP4 output gradients are rounded probabilistically to the two nearest values).  Arguments,
 * layout, scales (bit-identical to snip_quantize with SNIP_FP4_E2M1) and error behaviour as for
 * snip_quantize; out->fmt must be SNIP_FP4_E2M1.  The rounding is a pure function of (x, seed):
 *   - element i (row-major position in the STORED matrix) draws the random byte rnd = byte
 *     (i mod 8) of the 64 bits Threefry-2x32-20(counter = i div 8, key = seed) (Salmon et al.,
 *     SC'11; counter and key low word first; output word 0 first, least significant byte first);
 *   - with lo <= |v| <= hi the grid magnitudes next to the scaled element v and
 *     p = (|v| - lo) / (hi - lo), the magnitude becomes hi iff rnd < floor(256 p), else lo.
 * Grid values are kept for every seed; the expectation over rnd equals v exactly for
 * |v| >= 0.25 (p then has at most 8 bits) and lies within 0.5/256 below |v| otherwise.
 * Use a fresh seed per tensor and step. */
snip_status snip_quantize_sr_fp4(const void* x, int64_t rows, int64_t cols, int64_t ld,
                                 snip_axis axis, snip_scale_rule rule, uint64_t seed,
                                 const snip_qtensor* out, void* stream);

/* ---- the three GEMMs (Sec. 2.2; shapes Sec. 4.1 / 4.3.1) ----------------------------- */
/* All three contract the stored `cols` of both operands: C[i][j] = sum_r A[i][r] * B[j][r]
 * with a = code * 2^(scale-127), accumulated in fp32 and rounded once (nearest even) to the
 * output type.  Operands must have equal cols (SNIP_ERR_LAYOUT otherwise) and the formats the
 * plan names for that GEMM (SNIP_ERR_FORMAT otherwise).  The output is row-major with leading
 * dimension ld_out (elements), 16-byte aligned rows.  `workspace` is reserved (may be NULL).
 *
 *   fwd  : Xq  = quantize(X,  ROW) [M,K],  Wq  = quantize(W,  ROW) [N,K]  ->  Y  [M,N]
 *   dgrad: dYq = quantize(dY, ROW) [M,N],  Wq  = quantize(W,  COL) [K,N]  ->  dX [M,K]
 *   wgrad: dYq = quantize(dY, COL) [N,M],  Xq  = quantize(X,  COL) [K,M]  ->  dW [N,K]
 *
 * Every output element sums its products in one fixed order, whichever kernel and workgroup tile
 * the launcher picks for the shape.  The matrix-core kernels have tiles from 256 x 256 down to
 * 32 x 32 outputs per workgroup; the environment variable
 * SNIP_GEMM_TILE=big|wide|ahead|128x128|64x64|64x32|32x32|general (big = 256 x 256, wide = 256 x 128,
 * ahead is another name of wide), read at every call, fixes the tile where it can
 * serve the call, for measurements and tests, and never changes a result. */
snip_status snip_gemm_fwd(const snip_layer_plan* plan, const snip_qtensor* xq_row,
                          const snip_qtensor* wq_row, void* y, int64_t ld_out,
                          snip_out_dtype out_dtype, void* workspace, size_t workspace_bytes,
                          void* stream);
snip_status snip_gemm_dgrad(const snip_layer_plan* plan, const snip_qtensor* dyq_row,
                            const snip_qtensor* wq_col, void* dx, int64_t ld_out,
                            snip_out_dtype out_dtype, void* workspace, size_t workspace_bytes,
                            void* stream);
snip_status snip_gemm_wgrad(const snip_layer_plan* plan, const snip_qtensor* dyq_col,
                            const snip_qtensor* xq_col, void* dw, int64_t ld_out,
                            snip_out_dtype out_dtype, void* workspace, size_t workspace_bytes,
                            void* stream);

/* ---- GEMMs that also deliver the norm of their output (Sec. 3.1 Step 1) --------------- */
/* Step 1 of the paper collects the Frobenius norms of Y, dX and dW next to those of the GEMM
 * inputs; ||dX|| and ||dW|| are the gradient factors of the loss-divergence estimate (Sec. 4.2
 * "Loss Divergence in Forward Pass").  These variants compute exactly what the plain calls do and,
 * from the same accumulators, the squared Frobenius norm of the output AS STORED (every element
 * rounded to the output type first; elements outside the matrix do not count).
 *   sum_sq   : device, one double.
 *   workspace: device, required, >= snip_gemm_workspace_bytes(out rows, out cols) bytes, 16-byte
 *              aligned, no initialisation needed; calls that overlap in time must not share it.
 * The sum is formed per lane (128 or 64 squares), per wave and per workgroup in fp32 and across
 * workgroups in double, all in a fixed order: results are identical from run to run. */
size_t snip_gemm_workspace_bytes(int64_t out_rows, int64_t out_cols);
snip_status snip_gemm_fwd_norm(const snip_layer_plan* plan, const snip_qtensor* xq_row,
                               const snip_qtensor* wq_row, void* y, int64_t ld_out,
                               snip_out_dtype out_dtype, double* sum_sq, void* workspace,
                               size_t workspace_bytes, void* stream);
snip_status snip_gemm_dgrad_norm(const snip_layer_plan* plan, const snip_qtensor* dyq_row,
                                 const snip_qtensor* wq_col, void* dx, int64_t ld_out,
                                 snip_out_dtype out_dtype, double* sum_sq, void* workspace,
                                 size_t workspace_bytes, void* stream);
snip_status snip_gemm_wgrad_norm(const snip_layer_plan* plan, const snip_qtensor* dyq_col,
                                 const snip_qtensor* xq_col, void* dw, int64_t ld_out,
                                 snip_out_dtype out_dtype, double* sum_sq, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* Host, pure.  The paper's estimate of the loss change caused by quantizing the inputs X [m,k]
 * and weights W [n,k] of one linear layer (Sec. 4.2 "Loss Divergence in Forward Pass"):
 *     sqrt( (||dX|| ||q(X)-X|| / sqrt(m k))^2 + (||dW|| ||q(W)-W|| / sqrt(n k))^2 )
 * from SQUARED Frobenius norms: grad_x_sq / grad_w_sq are the sum_sq of the dgrad / wgrad calls
 * above, err_x_sq / err_w_sq the err_sq_* fields of snip_stats for the format in question.
 * Returns NaN for a non-positive extent or a negative or NaN argument. */
double snip_loss_divergence(double grad_x_sq, double err_x_sq, int64_t m,
                            double grad_w_sq, double err_w_sq, int64_t n, int64_t k);

/* ---- the paper's own quantization recipe (Sec. 2.3, Sec. 5.1) -------------------------- */
/* Sec. 2.3 scales a group by the real number s = FPX_MAX / max|x|, casts x * s to FPX and divides
 * by s afterwards; Sec. 5.1 uses 1x128 tiles for activations and gradients and 128x128 blocks
 * for weights.  These calls implement exactly that, next to the power-of-two 32-element blocks
 * of snip_quantize, so that the error statistics of the paper's configuration can be produced.
 * s and x * s are formed in fp32 (one correctly rounded division, one correctly rounded
 * product), then rounded to nearest even onto the FPX grid, saturating; s = 1 for an all-zero
 * group, s is capped at 2^126, and a group with an infinity or NaN gets s = NaN and zero codes.
 *   x, rows, cols, ld, axis: as for snip_quantize, but the blocked extent (cols for AXIS_ROW,
 *           rows for AXIS_COL) must be a multiple of 128.
 *   codes : device, layout as snip_qtensor.codes (stored orientation), 16-byte aligned.
 *   scales: device, fp32, [stored rows][stored cols / 128] for tiles,
 *           [ceil(stored rows / 128)][stored cols / 128] for blocks; snip_paper_scale_bytes.
 * The codes are consumed by snip_gemm_paper below, not by snip_gemm_fwd/dgrad/wgrad (the matrix
 * instruction applies power-of-two scales to 32-element blocks only). */
size_t snip_paper_scale_bytes(int64_t stored_rows, int64_t stored_cols, snip_group group);
snip_status snip_quantize_paper(const void* x, int64_t rows, int64_t cols, int64_t ld,
                                snip_fmt fmt, snip_axis axis, snip_group group,
                                void* codes, float* scales, void* stream);

/* A matrix quantized by snip_quantize_paper, in its stored orientation (cols = contraction extent,
 * a multiple of 128); scales as that call lays them out for `group`. */
typedef struct {
    const void*  codes;
    const float* scales;
    int64_t      rows, cols;
    int32_t      fmt;      /* snip_fmt */
    int32_t      group;    /* snip_group */
} snip_ptensor;

/* C[i][j] = sum_r (A[i][r] / sa) * (B[j][r] / sb) for operands of that recipe: the real-valued
 * scales are applied in software once per 128-element slab of the contraction (the codes of a
 * slab are multiplied on the matrix cores with unit scales into a fresh fp32 accumulator, which
 * is folded into the result with the factor (1/sa)(1/sb)); fp32 accumulation, one rounding to
 * the output type.  The three GEMMs of a linear layer are this call with the operand pairs
 * listed for snip_gemm_fwd / dgrad / wgrad.  A NaN scale makes the rows or columns it covers NaN.
 * Output layout and alignment as for the other GEMMs. */
snip_status snip_gemm_paper(const snip_ptensor* a, const snip_ptensor* b, void* c, int64_t ld_out,
                            snip_out_dtype out_dtype, void* stream);

/* Squared Frobenius norms of x and of q(x) - x for both formats under that recipe (q(x) = code / s).
 *   out: device, one snip_stats.  workspace: device, required,
 *   >= snip_paper_workspace_bytes(rows, cols), 16-byte aligned. */
size_t snip_paper_workspace_bytes(int64_t rows, int64_t cols);
snip_status snip_quant_error_stats_paper(const void* x, int64_t rows, int64_t cols, int64_t ld,
                                         snip_axis axis, snip_group group, snip_stats* out,
                                         void* workspace, size_t workspace_bytes, void* stream);

/* ---- AdamW factor of the weight-divergence estimate (Sec. 4.3.2) ---------------------- */
/* With m = beta1 m' + (1-beta1) g and v = beta2 v' + (1-beta2) g^2 (the AdamW moments after the
 * step's update) the update direction h(g) = m / (sqrt(v) + eps) has the element-wise derivative
 *     (1-beta1) / (sqrt(v)+eps)  -  (1-beta2) m g / ( sqrt(v) (sqrt(v)+eps)^2 );
 * Step 1 collects the Frobenius norm of that term (Sec. 4.3.2 "Impact on Weight Divergence").
 * This call writes its SQUARE to *sum_sq.
 *   m, v : device, fp32 [n], 16-byte aligned.  Where v is zero the second part counts as zero.
 *   g    : device, [n], fp32 (g_dtype = SNIP_OUT_FP32, 16-byte aligned) or bf16 (SNIP_OUT_BF16,
 *          8-byte aligned; e.g. the dW a wgrad call produced).
 *   beta1, beta2 in [0, 1), eps >= 0 (SNIP_ERR_FORMAT otherwise).
 *   sum_sq: device, one double.  workspace: device, required, >= snip_workspace_bytes(0, 0).
 * fp32 arithmetic.  Each of the two parts of an element's term is within 5e-7 of its value: correctly rounded root
 * and quotients, or, where v is zero or in [2^-96, 2^96] and eps in [2^-96, 1], approximated ones that are as close
 * (root and eps are rounded together there).  Infinities, NaNs and negative v reach the sum as in the expression.
 * Fixed summation order. */
snip_status snip_adamw_sensitivity(const float* m, const float* v, const void* g,
                                   snip_out_dtype g_dtype, int64_t n, float beta1, float beta2,
                                   float eps, double* sum_sq, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* Host, pure.  The per-layer weight-divergence estimate the factor feeds (same section):
 *     alpha sqrt(1 - beta2^t) / (1 - beta1^t) * sqrt(sens_sq) * sqrt(err_g_sq) / sqrt(n k)
 * for a weight of n x k elements at optimizer step t >= 1; sens_sq from snip_adamw_sensitivity,
 * err_g_sq the squared Frobenius norm of the perturbation of the weight gradient.  NaN on a
 * bad argument. */
double snip_weight_divergence(double alpha, double beta1, double beta2, int64_t t, double sens_sq,
                              double err_g_sq, int64_t n, int64_t k);

/* ---- RMS norm in front of a linear layer ------------------------------------------------ */
/* What makes the X operand of the linears behind a norm, with the residual's addition in front of it:
 *     h = bf16(x + residual)   (h = x without a residual)
 *     rstd = 1 / sqrt(mean(h^2) + eps) of every row,   y = h * weight * rstd.
 * The norm is that of h as it is stored, so that the backward call differentiates what was computed.  Sums
 * and statistics are fp32; y is rounded once, from fp32, to each output asked for:
 *   x, residual: device, bf16 [rows][ld], 16-byte aligned, ld >= cols and a multiple of 8; residual may be NULL.
 *   weight  : device, [cols], bf16 or fp32 (weight_dtype), 16-byte aligned.
 *   eps     : finite, >= 0.  With eps = 0 a row of zeros is 0 * infinity: NaN.
 *   sum     : device, bf16 [rows][ld_sum], h; NULL, or with a residual only (SNIP_ERR_NULL otherwise).  May be x or residual
 *             itself (same ld).
 *   rstd    : device, fp32 [rows], or NULL.
 *   y       : device, bf16 [rows][ld_y], or NULL.
 *   out_row : y quantized in blocks along rows, as by snip_quantize(..., SNIP_AXIS_ROW, rule, ...), but from fp32; cols a
 *             multiple of 32.  NULL if not wanted.
 *   out_col : the same down columns, stored transposed (cols x rows), the operand of snip_gemm_wgrad; rows a multiple of 32, cols
 *             even.  Needs rstd, and with a residual sum (SNIP_ERR_NULL otherwise).  The two formats may differ.
 * At least one output has to be given (SNIP_ERR_NULL).  A row with a NaN gets NaNs.  Where a row's squares add up to more than fp32
 * holds (3.4e38: an infinity, or numbers from 1.8e19 on) rstd is 0: finite elements become 0, infinite ones NaN, and no error is
 * raised; squares below fp32's normal numbers may count as zero.  Blocks that hold an infinity or a NaN get scale byte 0xFF and zero
 * codes, as in snip_quantize.  Columns >= cols of sum and y are not touched.  But for sum no output may overlap an input or another output. */
snip_status snip_rms_norm(const void* x, int64_t rows, int64_t cols, int64_t ld, const void* residual, int64_t ld_residual,
                          const void* weight, snip_out_dtype weight_dtype, float eps, snip_scale_rule rule,
                          void* sum, int64_t ld_sum, float* rstd, void* y, int64_t ld_y,
                          const snip_qtensor* out_row, const snip_qtensor* out_col, void* stream);

/* Its gradient.  With g = dy * weight:
 *     dx = rstd * (g - h * rstd^2 * mean(g h)) + dsum        (of x and of the residual alike)
 *     dweight = sum over rows of dy * h * rstd
 *   dy, h, dsum, dx: device, bf16, rows and pitches as above; h is `sum` (or x) and rstd that of the forward call; dsum, the
 *             gradient that reaches h past the norm, may be NULL.  dx may be dy or dsum itself.
 *   dweight : device, fp32 [cols], or NULL.
 *   workspace: device, needed with dweight, >= snip_rms_norm_workspace_bytes(rows, cols) bytes, 16-byte aligned.  The size never falls as
 *             rows or cols grow: a workspace for the largest matrix serves all that are no larger in either extent.
 * Sums are fp32 and added in a fixed order (the last 32 of each column in double). */
size_t snip_rms_norm_workspace_bytes(int64_t rows, int64_t cols);
snip_status snip_rms_norm_backward(const void* dy, int64_t rows, int64_t cols, int64_t ld_dy, const void* h, int64_t ld_h,
                                   const void* weight, snip_out_dtype weight_dtype, const float* rstd,
                                   const void* dsum, int64_t ld_dsum, void* dx, int64_t ld_dx, float* dweight,
                                   void* workspace, size_t workspace_bytes, void* stream);

/* ---- AdamW step ------------------------------------------------------------------------- */
/* One parameter tensor.  Arrays are contiguous and may start at any element.
 *   param  : device, fp32 [n], the master weights, updated.
 *   grad   : device, [n], fp32 or bf16 (grad_dtype): the dW of a wgrad call, the dweight of a norm.
 *   m, v   : device, the moments, updated; zeros before the first step.  fp32 [n], or, where m_scale and v_scale are
 *            given, 8 bits per element in groups of 128 (the last one may be shorter):
 *              m       : E4M3 numbers; the moment is number * m_scale[i / 128]
 *              v       : unsigned numbers c of 4 exponent and 4 mantissa bits, value (c >> 4 ? 2^((c >> 4) - 15) (1 + (c & 15) / 16) :
 *                        (c & 15) 2^-18), i.e. the half-precision number of bits c << 6; the moment is (value * v_scale[i / 128])^2
 *   copy   : device, bf16 [n], the new param rounded to nearest even, what the quantize calls read; or NULL.
 *   m_scale, v_scale: device, fp32 [ceil(n / 128)], both or neither.
 *   n      : 0 <= n < 2^34. */
typedef struct {
    float*      param;
    const void* grad;
    void*       m;
    void*       v;
    void*       copy;
    float*      m_scale;
    float*      v_scale;
    int64_t     n;
    float       weight_decay;
    int32_t     grad_dtype;      /* snip_out_dtype */
} snip_adamw_tensor;

/* AdamW with decoupled weight decay over `count` tensors (host array), 40 of them per launch:
 *     g = grad * *grad_scale;   m = beta1 m + (1 - beta1) g;   v = beta2 v + (1 - beta2) g^2
 *     param = param (1 - lr weight_decay) - lr / (1 - beta1^step) m / (sqrt(v / (1 - beta2^step)) + eps)
 * in fp32 (the coefficients formed in double), one rounding per operation.  param is updated with the moments before they are rounded to 8 bits.
 *   step       : counts from 1.  It and lr are arguments of the launch: a captured graph repeats them.
 *   grad_scale : device, one fp32 (a clipping coefficient, the inverse of a loss scale), or NULL for 1.
 *   seed       : moments of 8 bits: numbers of sqrt(v) are rounded stochastically, up where the bits that are dropped and 16
 *                random ones carry; element i of tensor k takes bits 16 (i mod 4) on of the 64 of Threefry-2x32-20 (counter = (i
 *                div 4, k), key = seed; words and counter as for snip_quantize_sr_fp4).  Take a fresh seed for every step.  Numbers of m are
 *                rounded to nearest even.  What is not zero keeps a number of sqrt(v) above zero.
 * What 8 bits do over steps: m keeps its number while (1 - beta1) |g - m| is below half the distance to the next one, up to |m| / 16
 * (2^-10 m_scale below 2^-6 m_scale).  Under gradients that do not change it can stop up to |m| / (16 (1 - beta1)) from them: 0.63 |m|
 * for beta1 = 0.9, and from 0.9375 on a moment whose gradients have become zero may stay for good.  Gradients that vary from step to
 * step move it all the same; where that cannot be relied on, and for beta1 above 0.9, take moments of 32 bits.  sqrt(v) is rounded without
 * bias, v is thus too large in the mean: 0.1 % under gradients that do not change, 0.9 % (beta2 = 0.95) to 2.1 % (0.999) under normally
 * distributed ones.
 * Scales are largest / 448 (m) and largest / 1.9375 (sqrt(v)), as products with the rounded reciprocals; a group whose scale would be
 * below 2^-126 becomes zero, and one with an infinity or NaN becomes NaN altogether.
 * beta1, beta2 in [0, 1), eps >= 0, lr and weight_decay finite, step >= 1 (SNIP_ERR_FORMAT otherwise). */
snip_status snip_adamw_step(const snip_adamw_tensor* tensors, int32_t count, double lr, double beta1, double beta2,
                            double eps, int64_t step, const float* grad_scale, uint64_t seed, void* stream);

/* ---- few tokens against quantized weights ----------------------------------------------- */
/* Y_i [m, n_i] = X [m, k] * W_i [n_i, k]^T for `count` weights that share X (q, k and v; gate and up), X in bf16 and not quantized: what
 * a model generates with, a token of each sequence at a time.
 *   x    : device, bf16 [m][ld], 16-byte aligned, ld >= k and a multiple of 8.
 *   w    : host array; quantize(W, ROW) of every weight (FP4 or FP8, formats may differ), all with cols == k (SNIP_ERR_LAYOUT
 *          otherwise); scales_g4 is not used.
 *   y    : host array of device pointers; Y_i is row-major with leading dimension ld_y[i], 16-byte aligned rows as for the GEMMs
 *          (ld_y is not read for a single token).
 * Weights become bf16: exactly within its normal numbers, below them (2^-126) to its nearest subnormal one, 2^-134 off at most (FP4, and
 * FP8 under scale bytes from 3 on, exactly there too), beyond them infinite.  Products are exact and sums fp32, added in a fixed order.  A scale byte of 0xFF makes its row NaN.  Meant for up to 64 tokens (m <= 65536 are served, 64 at a time, weights
 * read anew for each); the calls above are for more.  n_i <= 2^27. */
snip_status snip_gemv(const void* x, int64_t m, int64_t k, int64_t ld, const snip_qtensor* w, void* const* y,
                      const int64_t* ld_y, int32_t count, snip_out_dtype out_dtype, void* stream);

/* ---- both ends of a language model -------------------------------------------------------- */
/* What comes in front of the first layer and behind the last one: rows of the embedding, and the loss over the vocabulary with its
 * gradients, for the head's weights in bf16 and without keeping the logits.
 * Token numbers (`ids`, `targets`, `indices`) are 32- or 64-bit integers on the device, aligned to their size.  A number outside
 * [0, vocab) is no token: it has no row, no loss and no gradient (padding; a target of -100). */
typedef enum { SNIP_INDEX_I32 = 0, SNIP_INDEX_I64 = 1 } snip_index_dtype;

/* y[t] = scale * w[ids[t]], a product in fp32 that is rounded to bf16; zeros where ids[t] is no token.
 *   w    : device, bf16 or fp32 (w_dtype) [vocab][ld_w], 16-byte aligned; cols < 2^20 and ld_w >= cols multiples of 8; 0 < vocab < 2^31.
 *   scale: finite.
 *   y    : device, bf16 [tokens][ld_y], 16-byte aligned, ld_y >= cols, a multiple of 8.  Columns >= cols are not touched. */
snip_status snip_embed(const void* w, snip_out_dtype w_dtype, int64_t vocab, int64_t cols, int64_t ld_w, const void* ids,
                       snip_index_dtype id_dtype, int64_t tokens, float scale, void* y, int64_t ld_y, void* stream);

/* Its gradient: dw[v] = scale * (sum of dy[t] over the t with ids[t] == v), or, with `accumulate`, that added to what dw holds (a second
 * micro-batch; a table that is the head's weight too).
 *   dy  : device, bf16 [tokens][ld_dy], 16-byte aligned, ld_dy >= cols, a multiple of 8; tokens < 2^30, vocab <= 2^30.
 *   dw  : device, bf16 or fp32 (dw_dtype) [vocab][ld_dw], 16-byte aligned, ld_dw a multiple of 8.  Rows that no token names become
 *         zero, or with `accumulate` are not touched.
 *   workspace: device, >= snip_embed_workspace_bytes(tokens, cols, vocab) bytes, 16-byte aligned.  The size never falls as an extent grows.
 * Sums are fp32, of the tokens in their order (in parts of up to 64 where a row has more), and rounded once: results are the same from run to run.
 * More than 2048 tokens are put in order by a pass over all of them for each 512 entries of the table: 17 us for 16384 tokens and 32000 entries, 1.6 ms for
 * 2^20 tokens and 256000 entries. */
size_t snip_embed_workspace_bytes(int64_t tokens, int64_t cols, int64_t vocab);
snip_status snip_embed_backward(const void* dy, int64_t tokens, int64_t cols, int64_t ld_dy, const void* ids,
                                snip_index_dtype id_dtype, int64_t vocab, float scale, void* dw, snip_out_dtype dw_dtype,
                                int64_t ld_dw, int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream);

/* Softmax cross entropy of x [tokens][cols] against the head's weight w [vocab][cols], z = x w^T never being stored:
 *     lse[t] = log(sum over v of exp(z[t][v])),   loss[t] = lse[t] - z[t][targets[t]],   0 where targets[t] is no token.
 *   x, w   : device, bf16 [rows][ld], 16-byte aligned; cols and both ld >= cols multiples of 8; cols < 2^20, ld < 2^22; up to 2^21 tokens;
 *            0 < vocab <= 2^21; tokens * vocab and tokens * cols up to 2^37.
 *   targets: device, [tokens].
 *   loss, lse: device, fp32 [tokens]; lse is what the backward call needs.  Either may be NULL.
 *   workspace: device, >= snip_vocab_loss_workspace_bytes(tokens, cols, vocab, 1) bytes, 16-byte aligned.  The size never falls as an extent grows;
 *            calls that overlap in time must not share it.
 * Products are exact, sums, exponentials and logarithms fp32, in a fixed order.  Infinite logits count as the formulas have it: one of minus infinity adds
 * nothing (an entry that is masked out by its weights), one of plus infinity makes lse infinite.  lse is fp32 too: of a logit s the exponential that a gradient forms,
 * exp(s - lse), is off by up to |s| 2^-22 of itself, so gradients want |s| below some 2^13; from 2^29 on they need not be finite (the losses are). */
size_t snip_vocab_loss_workspace_bytes(int64_t tokens, int64_t cols, int64_t vocab, int64_t k);
snip_status snip_cross_entropy(const void* x, int64_t tokens, int64_t cols, int64_t ld_x, const void* w, int64_t vocab, int64_t ld_w,
                               const void* targets, snip_index_dtype index_dtype, float* loss, float* lse, void* workspace,
                               size_t workspace_bytes, void* stream);

/* Its gradients, from the same x, w and targets and the forward call's lse.  The logits are formed anew, a piece of the vocabulary at a time:
 *     dz[t][v] = dloss[t] * (exp(z[t][v] - lse[t]) - [v == targets[t]]),   dx = dz w,   dw = dz^T x.
 *   dloss: device, fp32 [tokens], the loss's gradient of every token (1 / count for a mean), or NULL for 1.  A token without a target, or
 *          whose dloss is zero, takes no part, whatever its x holds: its dx is zero, dw has nothing of it, and no product is formed for it.
 *   dx   : device, bf16 [tokens][ld_dx], 16-byte aligned, ld_dx a multiple of 8, or NULL.
 *   dw   : device, bf16 or fp32 (dw_dtype) [vocab][ld_dw], 16-byte aligned, ld_dw a multiple of 8, or NULL (a frozen head); with
 *          `accumulate` the gradient is added to what dw holds.
 *   workspace: as above, >= snip_vocab_loss_backward_workspace_bytes(tokens, cols, vocab, 1) bytes.  It holds dz of one piece, up to 2^28 elements of bf16 (all of
 *          dz where tokens * vocab is no more), partial sums of dx in fp32 and x of the tokens that take part: 743 MB for 8192 tokens of 4096 columns and 128000 entries.
 * dz is rounded to bf16 once, before the products with w and x (relative 2^-8 of each, also of an fp32 dw), in units of the largest finite |dloss|
 * (distillation: dloss * temperature): of equal weights the entry that is wanted loses least, and what is below 2^-126 of that unit may
 * become zero.  Sums are fp32, in a fixed order. */
size_t snip_vocab_loss_backward_workspace_bytes(int64_t tokens, int64_t cols, int64_t vocab, int64_t k);
snip_status snip_cross_entropy_backward(const void* x, int64_t tokens, int64_t cols, int64_t ld_x, const void* w, int64_t vocab,
                                        int64_t ld_w, const void* targets, snip_index_dtype index_dtype, const float* lse,
                                        const float* dloss, void* dx, int64_t ld_dx, void* dw, snip_out_dtype dw_dtype, int64_t ld_dw,
                                        int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream);

/* Distillation from the k largest logits of a teacher for every token.  With s = z / temperature and q[t] = softmax(teacher[t] /
 * temperature) over the entries whose index is a token:
 *     lse[t] = log(sum over v of exp(s[t][v])),
 *     loss[t] = temperature^2 * sum over j of q[t][j] * (log q[t][j] - s[t][indices[t][j]] + lse[t]),
 * the Kullback-Leibler divergence of the student, over the whole vocabulary, from the teacher's k; 0 where no index is a token.
 *   indices: device, [tokens][k], contiguous.  An index may come twice: both entries count.
 *   teacher: device, fp32 or bf16 (teacher_dtype) [tokens][k], contiguous.  An entry of minus infinity has q = 0; a row of nothing else is
 *            one without a token.
 *   k      : 1 to 1024, tokens * k < 2^31.   temperature: > 0; its square, which is normal, is an fp32 number too (1.1e-19 to 1.8e19).
 * Other arguments as for snip_cross_entropy; workspace for this k. */
snip_status snip_distill(const void* x, int64_t tokens, int64_t cols, int64_t ld_x, const void* w, int64_t vocab, int64_t ld_w,
                         const void* indices, snip_index_dtype index_dtype, const void* teacher, snip_out_dtype teacher_dtype, int64_t k,
                         float temperature, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* Its gradients, as for snip_cross_entropy_backward with
 *     dz[t][v] = dloss[t] * temperature * (exp(s[t][v] - lse[t]) - sum of q[t][j] over the j with indices[t][j] == v). */
snip_status snip_distill_backward(const void* x, int64_t tokens, int64_t cols, int64_t ld_x, const void* w, int64_t vocab, int64_t ld_w,
                                  const void* indices, snip_index_dtype index_dtype, const void* teacher, snip_out_dtype teacher_dtype,
                                  int64_t k, float temperature, const float* lse, const float* dloss, void* dx, int64_t ld_dx, void* dw,
                                  snip_out_dtype dw_dtype, int64_t ld_dw, int32_t accumulate, void* workspace, size_t workspace_bytes,
                                  void* stream);

/* ---- quantization-error statistics (Sec. 3.1 Step 1; row-wise form: Sec. 5.3) -------- */

/* One read of a bf16 matrix; for blocks along `axis` produces the squared Frobenius norm of x
 * and of q(x) - x for BOTH formats (the ILP needs the error of options that are not currently
 * selected, Sec. 4.2).
 *   out      : device, one snip_stats.
 *   per_line : device or NULL; float [L][3] = {sum x^2, err^2 fp4, err^2 fp8} for every line of
 *              the stored matrix: L = rows (one per source row) for AXIS_ROW, L = cols (one per
 *              source column) for AXIS_COL.
 *   workspace: device, required, >= snip_workspace_bytes(rows, cols). */
snip_status snip_quant_error_stats(const void* x, int64_t rows, int64_t cols, int64_t ld,
                                   snip_axis axis, snip_scale_rule rule,
                                   snip_stats* out, float* per_line,
                                   void* workspace, size_t workspace_bytes, void* stream);

/* The same statistics for BOTH block directions from one read of the matrix: *out_row is what
 * snip_quant_error_stats(..., SNIP_AXIS_ROW, ...) delivers and *out_col what SNIP_AXIS_COL
 * delivers (to the tolerance of the statistics; the sums are grouped differently).  A tensor's
 * forward operand is blocked along rows and its backward operands down columns (Sec. 2.2), so
 * this is the complete Step-1 record of a tensor.  rows and cols must both be multiples of 32;
 * no per-line sums.  workspace: >= snip_workspace_bytes(rows, cols). */
snip_status snip_quant_error_stats_both(const void* x, int64_t rows, int64_t cols, int64_t ld,
                                        snip_scale_rule rule, snip_stats* out_row,
                                        snip_stats* out_col, void* workspace,
                                        size_t workspace_bytes, void* stream);

/* For callers that cannot allocate device memory or pass a workspace (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): snip_quant_error_stats with its workspace
 * taken from an array that is part of the library's device image (about 24 MiB, resident on every
 * GPU the library is used on until the process ends).  Same arguments, results and error behaviour
 * as snip_quant_error_stats without the workspace pair, except:
 *   - cols must not exceed snip_noalloc_max_cols() (32768): SNIP_ERR_WORKSPACE otherwise;
 *   - the device is the current one (hipGetDevice) and `stream` must belong to it;
 *   - all calls on one GPU share the array: calls that overlap in time on one GPU (different
 *     streams, different threads) race and must be serialized by the caller.  Nothing in the
 *     array has to start at zero; every word a call reads it has written itself.
 * The call allocates nothing and frees nothing; the first call on a device looks up the array's
 * device address (hipGetSymbolAddress), later calls reuse it. */
size_t snip_noalloc_max_cols(void);
snip_status snip_quant_error_stats_noalloc(const void* x, int64_t rows, int64_t cols, int64_t ld,
                                           snip_axis axis, snip_scale_rule rule,
                                           snip_stats* out, float* per_line, void* stream);

const char* snip_status_string(snip_status s);

#ifdef __cplusplus
}
#endif
#endif /* SNIP_H */
