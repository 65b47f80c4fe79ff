// C-ABI layer: argument validation and dispatch.  No kernel code here.
#include "../../include/snip.h"
#include "snip_internal.h"
#include <algorithm>
#include <cmath>
#include <mutex>

using namespace snip;

// Scratch of snip_quant_error_stats_noalloc: the workspace of the statistics kernels for a source of up to
// kNoallocMaxCols columns, resident on every device the library is used on.  In host code this name is only a
// handle for hipGetSymbolAddress; kernels and launchers get the device address kept in g_scratch_ptr.
constexpr int64_t kNoallocMaxCols = 32768;
constexpr size_t kScratchBytes = stream_workspace_bytes(kNoallocMaxCols);
static __device__ __align__(256) unsigned char scratch[kScratchBytes];

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool valid_fmt(int f) { return f == SNIP_FP8_E4M3 || f == SNIP_FP4_E2M1; }

snip_status check_source(const void* x, int64_t rows, int64_t cols, int64_t ld, int axis, int rule)
{
    if (!x && rows > 0 && cols > 0) return SNIP_ERR_NULL;   // an empty matrix may have no storage
    if (axis != SNIP_AXIS_ROW && axis != SNIP_AXIS_COL) return SNIP_ERR_FORMAT;
    if (rule != SNIP_SCALE_NO_OVERFLOW && rule != SNIP_SCALE_OCP_FLOOR) return SNIP_ERR_FORMAT;
    if (rows < 0 || cols < 0 || ld < cols) return SNIP_ERR_SHAPE;
    if (axis == SNIP_AXIS_ROW && cols % 32 != 0) return SNIP_ERR_SHAPE;
    if (axis == SNIP_AXIS_COL && (rows % 32 != 0 || cols % 2 != 0)) return SNIP_ERR_SHAPE;
    // kernels index work units with 32-bit integers
    if (rows >= (int64_t)1 << 31 || cols >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    if ((rows + 31) / 32 * ((cols + 127) / 128) >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    if (rows * ((cols + 511) / 512) >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    if (!aligned16(x) || ld % 8 != 0) return SNIP_ERR_LAYOUT;
    return SNIP_OK;
}

snip_status check_qtensor(const snip_qtensor* q)
{
    if (!q) return SNIP_ERR_NULL;
    if ((!q->codes || !q->scales) && q->rows > 0) return SNIP_ERR_NULL;      // an empty matrix may have no storage
    if (!valid_fmt(q->fmt)) return SNIP_ERR_FORMAT;
    if (q->rows < 0 || q->cols <= 0 || q->cols % 32 != 0) return SNIP_ERR_SHAPE;
    if (q->rows >= (int64_t)1 << 31 || q->cols >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    if (!aligned16(q->codes)) return SNIP_ERR_LAYOUT;
    if (q->scales_g4 && !aligned16(q->scales_g4)) return SNIP_ERR_LAYOUT;      // written with 16-byte stores
    if (reinterpret_cast<uintptr_t>(q->scales) & 3u) return SNIP_ERR_LAYOUT;
    return SNIP_OK;
}

size_t gemm_ws_bytes(int64_t I, int64_t J) { return (size_t)gemm_norm_partials(I, J) * sizeof(float) + 16; }

snip_status gemm(const snip_qtensor* a, int fmt_a, const snip_qtensor* b, int fmt_b, void* c, int64_t ldc,
                 int out_dtype, void* stream, bool want_norm = false, double* sum_sq = nullptr,
                 void* workspace = nullptr, size_t workspace_bytes_ = 0)
{
    snip_status st = check_qtensor(a);
    if (st != SNIP_OK) return st;
    st = check_qtensor(b);
    if (st != SNIP_OK) return st;
    if (!c && a->rows > 0 && b->rows > 0) return SNIP_ERR_NULL;
    if (!valid_fmt(fmt_a) || !valid_fmt(fmt_b)) return SNIP_ERR_FORMAT;
    if (out_dtype != SNIP_OUT_BF16 && out_dtype != SNIP_OUT_FP32) return SNIP_ERR_FORMAT;
    if (a->fmt != fmt_a || b->fmt != fmt_b) return SNIP_ERR_FORMAT;
    if (a->cols != b->cols) return SNIP_ERR_LAYOUT;
    if (ldc < b->rows) return SNIP_ERR_SHAPE;
    if ((a->rows + 127) / 128 * ((b->rows + 127) / 128) >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    const int64_t align_elems = out_dtype == SNIP_OUT_BF16 ? 8 : 4;
    if (!aligned16(c) || ldc % align_elems != 0) return SNIP_ERR_LAYOUT;
    GemmArgs g;
    g.a_codes = (const uint8_t*)a->codes; g.a_scales = a->scales; g.a_scales_g4 = a->scales_g4; g.fmt_a = fmt_a;
    g.b_codes = (const uint8_t*)b->codes; g.b_scales = b->scales; g.b_scales_g4 = b->scales_g4; g.fmt_b = fmt_b;
    g.I = a->rows; g.J = b->rows; g.R = a->cols;
    g.c = c; g.ldc = ldc; g.out_fp32 = out_dtype == SNIP_OUT_FP32;
    if (want_norm) {
        if (!sum_sq) return SNIP_ERR_NULL;
        if (!workspace || workspace_bytes_ < gemm_ws_bytes(g.I, g.J)) return SNIP_ERR_WORKSPACE;
        if (!aligned16(workspace)) return SNIP_ERR_LAYOUT;
        g.norm_partials = (float*)workspace;
        g.norm_out = sum_sq;
    }
    return launch_gemm(g, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

// A bf16 matrix of a norm: `rows` rows `ld` apart.
snip_status check_rows(const void* p, int64_t rows, int64_t cols, int64_t ld)
{
    if (!p && rows > 0) return SNIP_ERR_NULL;
    if (ld < cols) return SNIP_ERR_SHAPE;
    if (!aligned16(p) || ld % 8 != 0) return SNIP_ERR_LAYOUT;
    return SNIP_OK;
}
snip_status check_norm(int64_t rows, int64_t cols, const void* weight, int weight_dtype)
{
    if (weight_dtype != SNIP_OUT_BF16 && weight_dtype != SNIP_OUT_FP32) return SNIP_ERR_FORMAT;
    if (rows < 0 || cols <= 0 || rows >= (int64_t)1 << 31 || cols >= (int64_t)1 << 30) return SNIP_ERR_SHAPE;
    if (!weight) return SNIP_ERR_NULL;
    return aligned16(weight) ? SNIP_OK : SNIP_ERR_LAYOUT;
}
snip_status check_out(const snip_qtensor* o, int64_t stored_rows, int64_t stored_cols)
{
    if (!valid_fmt(o->fmt)) return SNIP_ERR_FORMAT;
    if (o->rows != stored_rows || o->cols != stored_cols || stored_cols % 32 != 0) return SNIP_ERR_SHAPE;
    if ((!o->codes || !o->scales) && stored_rows > 0 && stored_cols > 0) return SNIP_ERR_NULL;
    if (!aligned16(o->codes) || !aligned16(o->scales_g4) || (reinterpret_cast<uintptr_t>(o->scales) & 3u)) return SNIP_ERR_LAYOUT;
    return SNIP_OK;
}

// Operands of the calls at both ends of a model: rows of a table or of tokens, whole pieces of 16 bytes.
constexpr int64_t kMostTokens = 1 << 21, kMostLd = 1 << 22, kMostVocab = (int64_t)1 << 31, kMostHead = 1 << 21, kMostWidth = 1 << 20;
// what their grids hold: 2^32 threads
constexpr int64_t kMostTable = (int64_t)1 << 30, kMostLogits = (int64_t)1 << 37;
bool valid_type(int t) { return t == SNIP_OUT_BF16 || t == SNIP_OUT_FP32; }
snip_status check_index(const void* p, int type, int64_t n)
{
    if (type != SNIP_INDEX_I32 && type != SNIP_INDEX_I64) return SNIP_ERR_FORMAT;
    if (!p && n > 0) return SNIP_ERR_NULL;
    return reinterpret_cast<uintptr_t>(p) & (type == SNIP_INDEX_I64 ? 7u : 3u) ? SNIP_ERR_LAYOUT : SNIP_OK;
}
snip_status check_vocab_loss(const VocabLossArgs& a, int index_type)
{
    if (a.tokens < 0 || a.tokens > kMostTokens || a.vocab <= 0 || a.vocab > kMostHead || a.cols <= 0 || a.cols >= kMostWidth || a.cols % 8 != 0) return SNIP_ERR_SHAPE;
    if (a.ldx >= kMostLd || a.ldw >= kMostLd || a.tokens * std::max(a.vocab, (int64_t)a.cols) > kMostLogits) return SNIP_ERR_SHAPE;
    if (a.k < 1 || a.k > 1024 || a.tokens * a.k >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    if (!(a.tau > 0.f) || !std::isfinite(1.f / a.tau) || !std::isnormal(a.tau * a.tau)) return SNIP_ERR_FORMAT;
    snip_status st = check_rows(a.x, a.tokens, a.cols, a.ldx);
    if (st == SNIP_OK) st = check_rows(a.w, a.vocab, a.cols, a.ldw);
    if (st == SNIP_OK) st = check_index(a.indices, index_type, a.tokens);
    if (st == SNIP_OK && ((reinterpret_cast<uintptr_t>(a.loss) | reinterpret_cast<uintptr_t>(a.lse) | reinterpret_cast<uintptr_t>(a.lse_in) | reinterpret_cast<uintptr_t>(a.dloss)) & 3u))
        st = SNIP_ERR_LAYOUT;
    return st;
}
snip_status check_teacher(const void* teacher, int type, int64_t tokens)
{
    if (!valid_type(type)) return SNIP_ERR_FORMAT;
    if (!teacher && tokens > 0) return SNIP_ERR_NULL;
    return reinterpret_cast<uintptr_t>(teacher) & (type == SNIP_OUT_FP32 ? 3u : 1u) ? SNIP_ERR_LAYOUT : SNIP_OK;
}
snip_status check_workspace(const void* p, size_t bytes, size_t needed)
{
    if (!p || bytes < needed) return SNIP_ERR_WORKSPACE;
    return aligned16(p) ? SNIP_OK : SNIP_ERR_LAYOUT;
}
snip_status vocab_loss(const VocabLossArgs& a, int index_type, size_t workspace_bytes_, void* stream)
{
    snip_status st = check_vocab_loss(a, index_type);
    if (st != SNIP_OK) return st;
    if (a.tokens == 0) return SNIP_OK;
    if (!a.loss && !a.lse) return SNIP_ERR_NULL;
    if ((st = check_workspace(a.workspace, workspace_bytes_, vocab_loss_needed(a))) != SNIP_OK) return st;
    return launch_vocab_loss(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}
snip_status vocab_loss_backward(const VocabLossArgs& a, int index_type, int dw_type, size_t workspace_bytes_, void* stream)
{
    snip_status st = check_vocab_loss(a, index_type);
    if (st != SNIP_OK) return st;
    if (!valid_type(dw_type)) return SNIP_ERR_FORMAT;
    if (!a.lse_in && a.tokens > 0) return SNIP_ERR_NULL;
    if (!a.dx && !a.dw && a.tokens > 0) return SNIP_ERR_NULL;
    if (a.dx && (st = check_rows(a.dx, a.tokens, a.cols, a.lddx)) != SNIP_OK) return st;
    if (a.dw && (st = check_rows(a.dw, a.vocab, a.cols, a.lddw)) != SNIP_OK) return st;
    if (a.tokens > 0 && (st = check_workspace(a.workspace, workspace_bytes_, vocab_loss_backward_needed(a))) != SNIP_OK) return st;
    return launch_vocab_loss_backward(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

}  // namespace

extern "C" {

size_t snip_qtensor_code_bytes(int64_t rows, int64_t cols, snip_fmt fmt)
{
    if (rows < 0 || cols < 0 || cols % 32 != 0 || !valid_fmt(fmt)) return 0;
    const size_t n = (size_t)rows * (size_t)cols;
    return fmt == SNIP_FP8_E4M3 ? n : n / 2;
}

size_t snip_qtensor_scale_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || cols % 32 != 0) return 0;
    return (size_t)rows * (size_t)(cols / 32);
}

size_t snip_qtensor_scale_g4_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || cols % 32 != 0) return 0;
    return (size_t)g4_pitch(rows) * (size_t)((cols + 127) / 128) * 4;
}

size_t snip_workspace_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0) return 0;
    return workspace_bytes(rows, cols);
}

snip_status snip_quantize(const void* x, int64_t rows, int64_t cols, int64_t ld, snip_fmt fmt, snip_axis axis,
                          snip_scale_rule rule, const snip_qtensor* out, snip_stats* stats, void* workspace,
                          size_t workspace_bytes_, void* stream)
{
    if (!valid_fmt(fmt)) return SNIP_ERR_FORMAT;
    snip_status st = check_source(x, rows, cols, ld, axis, rule);
    if (st != SNIP_OK) return st;
    if (!out) return SNIP_ERR_NULL;
    if ((!out->codes || !out->scales) && rows > 0 && cols > 0) return SNIP_ERR_NULL;
    if (out->fmt != (int32_t)fmt) return SNIP_ERR_FORMAT;
    const int64_t sr = axis == SNIP_AXIS_ROW ? rows : cols, sc = axis == SNIP_AXIS_ROW ? cols : rows;
    if (out->rows != sr || out->cols != sc) return SNIP_ERR_SHAPE;
    if (!aligned16(out->codes)) return SNIP_ERR_LAYOUT;
    if (out->scales_g4 && !aligned16(out->scales_g4)) return SNIP_ERR_LAYOUT;
    if (reinterpret_cast<uintptr_t>(out->scales) & 3u) return SNIP_ERR_LAYOUT;
    if (stats) {
        if (!workspace || workspace_bytes_ < workspace_bytes(rows, cols)) return SNIP_ERR_WORKSPACE;
        if (!aligned16(workspace)) return SNIP_ERR_LAYOUT;
    }
    QuantArgs a;
    a.x = (const uint16_t*)x; a.rows = rows; a.cols = cols; a.ld = ld;
    a.fmt = fmt; a.axis = axis; a.rule = rule;
    a.codes = (uint8_t*)out->codes; a.scales = out->scales; a.scales_g4 = out->scales_g4;
    a.stats = (double*)stats; a.workspace = workspace;
    return launch_quantize(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

snip_status snip_quantize_both(const void* x, int64_t rows, int64_t cols, int64_t ld, snip_scale_rule rule,
                               const snip_qtensor* out_row, const snip_qtensor* out_col, snip_stats* stats_row,
                               snip_stats* stats_col, snip_stats_scope scope, void* workspace, size_t workspace_bytes_,
                               void* stream)
{
    if (scope != SNIP_STATS_CHOSEN_FORMAT && scope != SNIP_STATS_BOTH_FORMATS) return SNIP_ERR_FORMAT;
    // both orientations: every extent constraint of the two single-orientation calls at once
    snip_status st = check_source(x, rows, cols, ld, SNIP_AXIS_ROW, rule);
    if (st == SNIP_OK) st = check_source(x, rows, cols, ld, SNIP_AXIS_COL, rule);
    if (st != SNIP_OK) return st;
    if (!out_row || !out_col) return SNIP_ERR_NULL;
    if ((stats_row == nullptr) != (stats_col == nullptr)) return SNIP_ERR_NULL;
    const snip_qtensor* outs[2] = {out_row, out_col};
    for (int i = 0; i < 2; ++i) {
        const snip_qtensor* o = outs[i];
        if ((!o->codes || !o->scales) && rows > 0 && cols > 0) return SNIP_ERR_NULL;
        if (!valid_fmt((snip_fmt)o->fmt)) return SNIP_ERR_FORMAT;
        if (o->rows != (i == 0 ? rows : cols) || o->cols != (i == 0 ? cols : rows)) return SNIP_ERR_SHAPE;
        if (!aligned16(o->codes)) return SNIP_ERR_LAYOUT;
        if (o->scales_g4 && !aligned16(o->scales_g4)) return SNIP_ERR_LAYOUT;
        if (reinterpret_cast<uintptr_t>(o->scales) & 3u) return SNIP_ERR_LAYOUT;
    }
    if (stats_row) {
        if (!workspace || workspace_bytes_ < workspace_bytes(rows, cols)) return SNIP_ERR_WORKSPACE;
        if (!aligned16(workspace)) return SNIP_ERR_LAYOUT;
    }
    QuantBothArgs a;
    a.x = (const uint16_t*)x; a.rows = rows; a.cols = cols; a.ld = ld; a.rule = rule;
    a.fmt_r = out_row->fmt; a.codes_r = (uint8_t*)out_row->codes; a.scales_r = out_row->scales; a.g4_r = out_row->scales_g4;
    a.fmt_c = out_col->fmt; a.codes_c = (uint8_t*)out_col->codes; a.scales_c = out_col->scales; a.g4_c = out_col->scales_g4;
    a.stats_r = (double*)stats_row; a.stats_c = (double*)stats_col; a.workspace = workspace;
    a.both_formats = scope == SNIP_STATS_BOTH_FORMATS;
    return launch_quantize_both(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

snip_status snip_quantize_sr_fp4(const void* x, int64_t rows, int64_t cols, int64_t ld, snip_axis axis,
                                 snip_scale_rule rule, uint64_t seed, const snip_qtensor* out, void* stream)
{
    snip_status st = check_source(x, rows, cols, ld, axis, rule);
    if (st != SNIP_OK) return st;
    if (!out) return SNIP_ERR_NULL;
    if ((!out->codes || !out->scales) && rows > 0 && cols > 0) return SNIP_ERR_NULL;
    if (out->fmt != (int32_t)SNIP_FP4_E2M1) return SNIP_ERR_FORMAT;
    const int64_t sr = axis == SNIP_AXIS_ROW ? rows : cols, sc = axis == SNIP_AXIS_ROW ? cols : rows;
    if (out->rows != sr || out->cols != sc) return SNIP_ERR_SHAPE;
    if (!aligned16(out->codes)) return SNIP_ERR_LAYOUT;
    if (out->scales_g4 && !aligned16(out->scales_g4)) return SNIP_ERR_LAYOUT;
    if (reinterpret_cast<uintptr_t>(out->scales) & 3u) return SNIP_ERR_LAYOUT;
    QuantArgs a;
    a.x = (const uint16_t*)x; a.rows = rows; a.cols = cols; a.ld = ld;
    a.fmt = SNIP_FP4_E2M1; a.axis = axis; a.rule = rule;
    a.codes = (uint8_t*)out->codes; a.scales = out->scales; a.scales_g4 = out->scales_g4;
    a.stats = nullptr; a.workspace = nullptr;
    a.stochastic = true; a.sr_seed = seed;
    return launch_quantize(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

snip_status snip_gemm_fwd(const snip_layer_plan* plan, const snip_qtensor* xq_row, const snip_qtensor* wq_row,
                          void* y, int64_t ld_out, snip_out_dtype out_dtype, void*, size_t, void* stream)
{
    if (!plan) return SNIP_ERR_NULL;
    return gemm(xq_row, plan->fwd_x, wq_row, plan->fwd_w, y, ld_out, out_dtype, stream);
}

snip_status snip_gemm_dgrad(const snip_layer_plan* plan, const snip_qtensor* dyq_row, const snip_qtensor* wq_col,
                            void* dx, int64_t ld_out, snip_out_dtype out_dtype, void*, size_t, void* stream)
{
    if (!plan) return SNIP_ERR_NULL;
    return gemm(dyq_row, plan->dgrad_dy, wq_col, plan->dgrad_w, dx, ld_out, out_dtype, stream);
}

snip_status snip_gemm_wgrad(const snip_layer_plan* plan, const snip_qtensor* dyq_col, const snip_qtensor* xq_col,
                            void* dw, int64_t ld_out, snip_out_dtype out_dtype, void*, size_t, void* stream)
{
    if (!plan) return SNIP_ERR_NULL;
    return gemm(dyq_col, plan->wgrad_dy, xq_col, plan->wgrad_x, dw, ld_out, out_dtype, stream);
}

size_t snip_gemm_workspace_bytes(int64_t out_rows, int64_t out_cols)
{
    if (out_rows < 0 || out_cols < 0) return 0;
    return gemm_ws_bytes(out_rows, out_cols);
}

snip_status snip_gemm_fwd_norm(const snip_layer_plan* plan, const snip_qtensor* xq_row, const snip_qtensor* wq_row,
                               void* y, int64_t ld_out, snip_out_dtype out_dtype, double* sum_sq, void* workspace,
                               size_t workspace_bytes_, void* stream)
{
    if (!plan) return SNIP_ERR_NULL;
    return gemm(xq_row, plan->fwd_x, wq_row, plan->fwd_w, y, ld_out, out_dtype, stream, true, sum_sq, workspace, workspace_bytes_);
}

snip_status snip_gemm_dgrad_norm(const snip_layer_plan* plan, const snip_qtensor* dyq_row, const snip_qtensor* wq_col,
                                 void* dx, int64_t ld_out, snip_out_dtype out_dtype, double* sum_sq, void* workspace,
                                 size_t workspace_bytes_, void* stream)
{
    if (!plan) return SNIP_ERR_NULL;
    return gemm(dyq_row, plan->dgrad_dy, wq_col, plan->dgrad_w, dx, ld_out, out_dtype, stream, true, sum_sq, workspace, workspace_bytes_);
}

snip_status snip_gemm_wgrad_norm(const snip_layer_plan* plan, const snip_qtensor* dyq_col, const snip_qtensor* xq_col,
                                 void* dw, int64_t ld_out, snip_out_dtype out_dtype, double* sum_sq, void* workspace,
                                 size_t workspace_bytes_, void* stream)
{
    if (!plan) return SNIP_ERR_NULL;
    return gemm(dyq_col, plan->wgrad_dy, xq_col, plan->wgrad_x, dw, ld_out, out_dtype, stream, true, sum_sq, workspace, workspace_bytes_);
}

double snip_loss_divergence(double grad_x_sq, double err_x_sq, int64_t m, double grad_w_sq, double err_w_sq,
                            int64_t n, int64_t k)
{
    if (m <= 0 || n <= 0 || k <= 0 || !(grad_x_sq >= 0.0) || !(err_x_sq >= 0.0) || !(grad_w_sq >= 0.0) || !(err_w_sq >= 0.0))
        return std::nan("");
    // each term is a product of two Frobenius norms over the square root of the element count
    const double tx = std::sqrt(grad_x_sq * err_x_sq / ((double)m * (double)k));
    const double tw = std::sqrt(grad_w_sq * err_w_sq / ((double)n * (double)k));
    return std::hypot(tx, tw);
}

static snip_status check_paper(const void* x, int64_t rows, int64_t cols, int64_t ld, int axis, int group)
{
    snip_status st = check_source(x, rows, cols, ld, axis, SNIP_SCALE_NO_OVERFLOW);
    if (st != SNIP_OK) return st;
    if (group != SNIP_GROUP_TILE_1x128 && group != SNIP_GROUP_BLOCK_128x128) return SNIP_ERR_FORMAT;
    if ((axis == SNIP_AXIS_ROW ? cols : rows) % 128 != 0) return SNIP_ERR_SHAPE;
    return SNIP_OK;
}

size_t snip_paper_scale_bytes(int64_t stored_rows, int64_t stored_cols, snip_group group)
{
    if (stored_rows < 0 || stored_cols < 0 || stored_cols % 128 != 0) return 0;
    if (group != SNIP_GROUP_TILE_1x128 && group != SNIP_GROUP_BLOCK_128x128) return 0;
    const int64_t gr = group == SNIP_GROUP_TILE_1x128 ? stored_rows : (stored_rows + 127) / 128;
    return (size_t)gr * (size_t)(stored_cols / 128) * sizeof(float);
}

size_t snip_paper_workspace_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0) return 0;
    return paper_workspace_bytes(rows, cols);
}

snip_status snip_quantize_paper(const void* x, int64_t rows, int64_t cols, int64_t ld, snip_fmt fmt, snip_axis axis,
                                snip_group group, void* codes, float* scales, void* stream)
{
    if (!valid_fmt(fmt)) return SNIP_ERR_FORMAT;
    snip_status st = check_paper(x, rows, cols, ld, axis, group);
    if (st != SNIP_OK) return st;
    if ((!codes || !scales) && rows > 0 && cols > 0) return SNIP_ERR_NULL;
    if (!aligned16(codes) || (reinterpret_cast<uintptr_t>(scales) & 3u)) return SNIP_ERR_LAYOUT;
    PaperArgs a;
    a.x = (const uint16_t*)x; a.rows = rows; a.cols = cols; a.ld = ld; a.fmt = fmt; a.axis = axis;
    a.blocks = group == SNIP_GROUP_BLOCK_128x128;
    a.codes = (uint8_t*)codes; a.scales = scales; a.stats = nullptr; a.workspace = nullptr;
    return launch_paper(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

snip_status snip_quant_error_stats_paper(const void* x, int64_t rows, int64_t cols, int64_t ld, snip_axis axis,
                                         snip_group group, snip_stats* out, void* workspace, size_t workspace_bytes_,
                                         void* stream)
{
    snip_status st = check_paper(x, rows, cols, ld, axis, group);
    if (st != SNIP_OK) return st;
    if (!out) return SNIP_ERR_NULL;
    if (!workspace || workspace_bytes_ < paper_workspace_bytes(rows, cols)) return SNIP_ERR_WORKSPACE;
    if (!aligned16(workspace)) return SNIP_ERR_LAYOUT;
    PaperArgs a;
    a.x = (const uint16_t*)x; a.rows = rows; a.cols = cols; a.ld = ld; a.fmt = SNIP_FP8_E4M3; a.axis = axis;
    a.blocks = group == SNIP_GROUP_BLOCK_128x128;
    a.codes = nullptr; a.scales = nullptr; a.stats = (double*)out; a.workspace = workspace;
    return launch_paper(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

static snip_status check_ptensor(const snip_ptensor* q)
{
    if (!q) return SNIP_ERR_NULL;
    if ((!q->codes || !q->scales) && q->rows > 0) return SNIP_ERR_NULL;
    if (!valid_fmt(q->fmt)) return SNIP_ERR_FORMAT;
    if (q->group != SNIP_GROUP_TILE_1x128 && q->group != SNIP_GROUP_BLOCK_128x128) return SNIP_ERR_FORMAT;
    if (q->rows < 0 || q->cols <= 0 || q->cols % 128 != 0) return SNIP_ERR_SHAPE;
    if (q->rows >= (int64_t)1 << 31 || q->cols >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    if (!aligned16(q->codes) || (reinterpret_cast<uintptr_t>(q->scales) & 3u)) return SNIP_ERR_LAYOUT;
    return SNIP_OK;
}

snip_status snip_gemm_paper(const snip_ptensor* a, const snip_ptensor* b, void* c, int64_t ld_out,
                            snip_out_dtype out_dtype, void* stream)
{
    snip_status st = check_ptensor(a);
    if (st != SNIP_OK) return st;
    st = check_ptensor(b);
    if (st != SNIP_OK) return st;
    if (!c && a->rows > 0 && b->rows > 0) return SNIP_ERR_NULL;
    if (out_dtype != SNIP_OUT_BF16 && out_dtype != SNIP_OUT_FP32) return SNIP_ERR_FORMAT;
    if (a->cols != b->cols) return SNIP_ERR_LAYOUT;
    if (ld_out < b->rows) return SNIP_ERR_SHAPE;
    if ((a->rows + 127) / 128 * ((b->rows + 127) / 128) >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    if (!aligned16(c) || ld_out % (out_dtype == SNIP_OUT_BF16 ? 8 : 4) != 0) return SNIP_ERR_LAYOUT;
    GemmPaperArgs g;
    g.a_codes = (const uint8_t*)a->codes; g.a_scales = a->scales; g.a_group = a->group; g.fmt_a = a->fmt;
    g.b_codes = (const uint8_t*)b->codes; g.b_scales = b->scales; g.b_group = b->group; g.fmt_b = b->fmt;
    g.I = a->rows; g.J = b->rows; g.R = a->cols;
    g.c = c; g.ldc = ld_out; g.out_fp32 = out_dtype == SNIP_OUT_FP32;
    return launch_gemm_paper(g, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

snip_status snip_adamw_sensitivity(const float* m, const float* v, const void* g, snip_out_dtype g_dtype,
                                   int64_t n, float beta1, float beta2, float eps, double* sum_sq,
                                   void* workspace, size_t workspace_bytes_, void* stream)
{
    if (n < 0) return SNIP_ERR_SHAPE;
    if ((!m || !v || !g) && n > 0) return SNIP_ERR_NULL;
    if (!sum_sq) return SNIP_ERR_NULL;
    if (g_dtype != SNIP_OUT_BF16 && g_dtype != SNIP_OUT_FP32) return SNIP_ERR_FORMAT;
    if (!(beta1 >= 0.f && beta1 < 1.f) || !(beta2 >= 0.f && beta2 < 1.f) || !(eps >= 0.f)) return SNIP_ERR_FORMAT;
    if (!aligned16(m) || !aligned16(v)) return SNIP_ERR_LAYOUT;
    if (reinterpret_cast<uintptr_t>(g) & (g_dtype == SNIP_OUT_BF16 ? 7u : 15u)) return SNIP_ERR_LAYOUT;
    if (!workspace || workspace_bytes_ < workspace_bytes(0, 0)) return SNIP_ERR_WORKSPACE;
    if (!aligned16(workspace)) return SNIP_ERR_LAYOUT;
    AdamwArgs a;
    a.m = m; a.v = v; a.g = g; a.g_bf16 = g_dtype == SNIP_OUT_BF16; a.n = n;
    a.beta1 = beta1; a.beta2 = beta2; a.eps = eps; a.out = sum_sq; a.workspace = workspace;
    return launch_adamw_sensitivity(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

double snip_weight_divergence(double alpha, double beta1, double beta2, int64_t t, double sens_sq,
                              double err_g_sq, int64_t n, int64_t k)
{
    if (t <= 0 || n <= 0 || k <= 0 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) ||
        !(sens_sq >= 0.0) || !(err_g_sq >= 0.0))
        return std::nan("");
    const double corr = std::sqrt(1.0 - std::pow(beta2, (double)t)) / (1.0 - std::pow(beta1, (double)t));
    return alpha * corr * std::sqrt(sens_sq * err_g_sq / ((double)n * (double)k));
}

snip_status snip_quant_error_stats(const void* x, int64_t rows, int64_t cols, int64_t ld, snip_axis axis,
                                   snip_scale_rule rule, snip_stats* out, float* per_line, void* workspace,
                                   size_t workspace_bytes_, void* stream)
{
    snip_status st = check_source(x, rows, cols, ld, axis, rule);
    if (st != SNIP_OK) return st;
    if (!out) return SNIP_ERR_NULL;
    if (!workspace || workspace_bytes_ < workspace_bytes(rows, cols)) return SNIP_ERR_WORKSPACE;
    if (!aligned16(workspace)) return SNIP_ERR_LAYOUT;
    StatsArgs a;
    a.x = (const uint16_t*)x; a.rows = rows; a.cols = cols; a.ld = ld; a.axis = axis; a.rule = rule;
    a.stats = (double*)out; a.per_line = per_line; a.workspace = workspace;
    return launch_stats(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

snip_status snip_quant_error_stats_both(const void* x, int64_t rows, int64_t cols, int64_t ld, snip_scale_rule rule,
                                        snip_stats* out_row, snip_stats* out_col, void* workspace,
                                        size_t workspace_bytes_, void* stream)
{
    snip_status st = check_source(x, rows, cols, ld, SNIP_AXIS_ROW, rule);
    if (st != SNIP_OK) return st;
    st = check_source(x, rows, cols, ld, SNIP_AXIS_COL, rule);
    if (st != SNIP_OK) return st;
    if (!out_row || !out_col) return SNIP_ERR_NULL;
    if (!workspace || workspace_bytes_ < workspace_bytes(rows, cols)) return SNIP_ERR_WORKSPACE;
    if (!aligned16(workspace)) return SNIP_ERR_LAYOUT;
    StatsArgs a;
    a.x = (const uint16_t*)x; a.rows = rows; a.cols = cols; a.ld = ld; a.axis = SNIP_AXIS_ROW; a.rule = rule;
    a.stats = (double*)out_row; a.per_line = nullptr; a.workspace = workspace;
    return launch_stats_both(a, (double*)out_col, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

snip_status snip_rms_norm(const void* x, int64_t rows, int64_t cols, int64_t ld, const void* residual, int64_t ld_residual,
                          const void* weight, snip_out_dtype weight_dtype, float eps, snip_scale_rule rule, void* sum,
                          int64_t ld_sum, float* rstd, void* y, int64_t ld_y, const snip_qtensor* out_row,
                          const snip_qtensor* out_col, void* stream)
{
    if (rule != SNIP_SCALE_NO_OVERFLOW && rule != SNIP_SCALE_OCP_FLOOR) return SNIP_ERR_FORMAT;
    if (!(eps >= 0.f && eps <= 3.402823466e38f)) return SNIP_ERR_FORMAT;
    snip_status st = check_norm(rows, cols, weight, weight_dtype);
    if (st == SNIP_OK) st = check_rows(x, rows, cols, ld);
    if (st == SNIP_OK && residual) st = check_rows(residual, rows, cols, ld_residual);
    if (st == SNIP_OK && sum) st = residual ? check_rows(sum, rows, cols, ld_sum) : SNIP_ERR_NULL;
    if (st == SNIP_OK && y) st = check_rows(y, rows, cols, ld_y);
    if (st != SNIP_OK) return st;
    if (rows > 0 && !sum && !rstd && !y && !out_row && !out_col) return SNIP_ERR_NULL;      // (an empty vector may have no storage)
    if (reinterpret_cast<uintptr_t>(rstd) & 3u) return SNIP_ERR_LAYOUT;
    if (out_row && (st = check_out(out_row, rows, cols)) != SNIP_OK) return st;
    if (out_col) {
        if (cols % 2 != 0) return SNIP_ERR_SHAPE;
        if ((st = check_out(out_col, cols, rows)) != SNIP_OK) return st;
        if (rows > 0 && (!rstd || (residual && !sum))) return SNIP_ERR_NULL;
        if ((rows + 31) / 32 * ((cols + 127) / 128) >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    }
    NormArgs a = {};
    a.x = (const uint16_t*)x; a.ldx = ld; a.r = (const uint16_t*)residual; a.ldr = ld_residual;
    a.gain = weight; a.gain_fp32 = weight_dtype == SNIP_OUT_FP32; a.rows = (int)rows; a.cols = (int)cols; a.eps = eps;
    a.sum = (uint16_t*)sum; a.lds = ld_sum; a.rstd = rstd; a.y = (uint16_t*)y; a.ldy = ld_y; a.rule = rule;
    if (out_row) {
        a.fmt_r = out_row->fmt; a.codes_r = (uint8_t*)out_row->codes; a.scales_r = out_row->scales; a.g4_r = out_row->scales_g4;
        a.pitch_r = g4_pitch(rows);
    }
    if (out_col) {
        a.fmt_c = out_col->fmt; a.codes_c = (uint8_t*)out_col->codes; a.scales_c = out_col->scales; a.g4_c = out_col->scales_g4;
        a.pitch_c = g4_pitch(cols);
    }
    return launch_rms_norm(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

size_t snip_rms_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols <= 0) return 0;
    return norm_workspace_bytes(rows, cols);
}

snip_status snip_rms_norm_backward(const void* dy, int64_t rows, int64_t cols, int64_t ld_dy, const void* h, int64_t ld_h,
                                   const void* weight, snip_out_dtype weight_dtype, const float* rstd, const void* dsum,
                                   int64_t ld_dsum, void* dx, int64_t ld_dx, float* dweight, void* workspace,
                                   size_t workspace_bytes_, void* stream)
{
    snip_status st = check_norm(rows, cols, weight, weight_dtype);
    if (st == SNIP_OK) st = check_rows(dy, rows, cols, ld_dy);
    if (st == SNIP_OK) st = check_rows(h, rows, cols, ld_h);
    if (st == SNIP_OK && dsum) st = check_rows(dsum, rows, cols, ld_dsum);
    if (st == SNIP_OK) st = check_rows(dx, rows, cols, ld_dx);
    if (st != SNIP_OK) return st;
    if (!rstd && rows > 0) return SNIP_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(rstd) | reinterpret_cast<uintptr_t>(dweight)) & 3u) return SNIP_ERR_LAYOUT;
    if (dweight && rows > 0) {
        if (!workspace || workspace_bytes_ < norm_workspace_needed(rows, cols)) return SNIP_ERR_WORKSPACE;
        if (!aligned16(workspace)) return SNIP_ERR_LAYOUT;
    }
    NormGradArgs a = {};
    a.dy = (const uint16_t*)dy; a.lddy = ld_dy; a.h = (const uint16_t*)h; a.ldh = ld_h;
    a.gain = weight; a.gain_fp32 = weight_dtype == SNIP_OUT_FP32; a.rstd = rstd;
    a.dsum = (const uint16_t*)dsum; a.ldds = ld_dsum; a.dx = (uint16_t*)dx; a.lddx = ld_dx;
    a.dgain = dweight; a.partials = dweight ? (float*)workspace : nullptr; a.rows = (int)rows; a.cols = (int)cols;
    return launch_rms_norm_backward(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

snip_status snip_adamw_step(const snip_adamw_tensor* tensors, int32_t count, double lr, double beta1, double beta2,
                            double eps, int64_t step, const float* grad_scale, uint64_t seed, void* stream)
{
    if (count < 0 || step < 1) return count < 0 ? SNIP_ERR_SHAPE : SNIP_ERR_FORMAT;
    if (!tensors && count > 0) return SNIP_ERR_NULL;
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0 && eps >= 0.0) || !std::isfinite(eps) || !std::isfinite(lr)) return SNIP_ERR_FORMAT;
    if (reinterpret_cast<uintptr_t>(grad_scale) & 3u) return SNIP_ERR_LAYOUT;
    for (int32_t i = 0; i < count; ++i) {
        const snip_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n >= (int64_t)1 << 34) return SNIP_ERR_SHAPE;
        if (t.grad_dtype != SNIP_OUT_BF16 && t.grad_dtype != SNIP_OUT_FP32) return SNIP_ERR_FORMAT;
        if (!std::isfinite(t.weight_decay)) return SNIP_ERR_FORMAT;
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v || !t.m_scale != !t.v_scale) return SNIP_ERR_NULL;
        const uintptr_t fp32 = reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(t.m_scale) | reinterpret_cast<uintptr_t>(t.v_scale) |
                               (t.m_scale ? 0 : reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v)) |
                               (t.grad_dtype == SNIP_OUT_FP32 ? reinterpret_cast<uintptr_t>(t.grad) : 0);
        if ((fp32 & 3u) || ((reinterpret_cast<uintptr_t>(t.copy) | reinterpret_cast<uintptr_t>(t.grad)) & 1u)) return SNIP_ERR_LAYOUT;
    }
    AdamwStepArgs a = {};
    a.beta1 = (float)beta1; a.rest1 = (float)(1.0 - beta1); a.beta2 = (float)beta2; a.rest2 = (float)(1.0 - beta2);
    a.step_size = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    a.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    a.eps = (float)eps; a.grad_scale = grad_scale; a.seed = make_uint2((unsigned)seed, (unsigned)(seed >> 32));
    for (int small = 0; small < 2; ++small) {
        int64_t chunks = 0;
        a.count = 0;
        auto launch = [&] {
            a.chunks = (unsigned)chunks;
            const hipError_t e = launch_adamw_step(a, small != 0, (hipStream_t)stream);
            a.count = 0;
            chunks = 0;
            return e == hipSuccess;
        };
        for (int32_t i = 0; i < count; ++i) {
            const snip_adamw_tensor& t = tensors[i];
            if (t.n == 0 || (t.m_scale != nullptr) != (small != 0)) continue;
            AdamwStepTensor& d = a.t[a.count];
            d.p = t.param; d.g = t.grad; d.m = t.m; d.v = t.v; d.copy = (uint16_t*)t.copy; d.m_scale = t.m_scale; d.v_scale = t.v_scale; d.n = t.n;
            d.keep = (float)(1.0 - lr * t.weight_decay); d.g_bf16 = t.grad_dtype == SNIP_OUT_BF16; d.index = (unsigned)i;
            a.first[a.count++] = (unsigned)chunks;
            chunks += adamw_step_chunks(t.n);
            if (a.count == kStepTensors && !launch()) return SNIP_ERR_HIP;
        }
        if (a.count > 0 && !launch()) return SNIP_ERR_HIP;
    }
    return SNIP_OK;
}

snip_status snip_gemv(const void* x, int64_t m, int64_t k, int64_t ld, const snip_qtensor* w, void* const* y,
                      const int64_t* ld_y, int32_t count, snip_out_dtype out_dtype, void* stream)
{
    if (out_dtype != SNIP_OUT_BF16 && out_dtype != SNIP_OUT_FP32) return SNIP_ERR_FORMAT;
    if (m < 0 || k <= 0 || k % 32 != 0 || count < 0 || m > 65536 || k >= (int64_t)1 << 31) return SNIP_ERR_SHAPE;
    snip_status st = check_rows(x, m, k, ld);
    if (st != SNIP_OK) return st;
    if ((!w || !y || !ld_y) && count > 0) return SNIP_ERR_NULL;
    for (int32_t i = 0; i < count; ++i) {
        if ((st = check_qtensor(&w[i])) != SNIP_OK) return st;
        if (w[i].cols != k) return SNIP_ERR_LAYOUT;
        if (w[i].rows > (int64_t)1 << 27) return SNIP_ERR_SHAPE;                 // (eight of them: workgroups of a launch)
        if (w[i].rows == 0) continue;
        if (!y[i] && m > 0) return SNIP_ERR_NULL;
        if (m > 1 && ld_y[i] < w[i].rows) return SNIP_ERR_SHAPE;                 // (a single row has no pitch)
        if (!aligned16(y[i]) || (m > 1 && ld_y[i] % (out_dtype == SNIP_OUT_BF16 ? 8 : 4) != 0)) return SNIP_ERR_LAYOUT;
    }
    GemvArgs a = {};
    a.x = (const uint16_t*)x; a.ldx = ld; a.m = (int)m; a.k = (int)k; a.out_fp32 = out_dtype == SNIP_OUT_FP32;
    for (int32_t i = 0; i < count; ++i) {
        if (w[i].rows > 0) {
            GemvWeight& g = a.w[a.count++];
            g.codes = (const uint8_t*)w[i].codes; g.scales = w[i].scales; g.y = y[i]; g.ldy = ld_y[i]; g.n = (int)w[i].rows; g.fmt = w[i].fmt;
        }
        if (a.count == kGemvWeights || i + 1 == count) {
            if (launch_gemv(a, (hipStream_t)stream) != hipSuccess) return SNIP_ERR_HIP;
            a.count = 0;
        }
    }
    return SNIP_OK;
}

snip_status snip_embed(const void* w, snip_out_dtype w_dtype, int64_t vocab, int64_t cols, int64_t ld_w, const void* ids,
                       snip_index_dtype id_dtype, int64_t tokens, float scale, void* y, int64_t ld_y, void* stream)
{
    if (!valid_type(w_dtype) || !std::isfinite(scale)) return SNIP_ERR_FORMAT;
    if (tokens < 0 || vocab <= 0 || vocab >= kMostVocab || cols <= 0 || cols >= kMostWidth || cols % 8 != 0) return SNIP_ERR_SHAPE;
    snip_status st = check_rows(w, vocab, cols, ld_w);
    if (st == SNIP_OK) st = check_rows(y, tokens, cols, ld_y);
    if (st == SNIP_OK) st = check_index(ids, id_dtype, tokens);
    if (st != SNIP_OK) return st;
    EmbedArgs a = {};
    a.w = w; a.w_fp32 = w_dtype == SNIP_OUT_FP32; a.vocab = vocab; a.ldw = ld_w; a.ids = ids; a.ids64 = id_dtype == SNIP_INDEX_I64;
    a.tokens = tokens; a.cols = (int)cols; a.scale = scale; a.y = (uint16_t*)y; a.ldy = ld_y;
    return launch_embed(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

size_t snip_embed_workspace_bytes(int64_t tokens, int64_t cols, int64_t vocab)
{
    return tokens < 0 || cols <= 0 || vocab <= 0 ? 0 : embed_workspace_bytes(tokens, cols, vocab);
}

snip_status snip_embed_backward(const void* dy, int64_t tokens, int64_t cols, int64_t ld_dy, const void* ids,
                                snip_index_dtype id_dtype, int64_t vocab, float scale, void* dw, snip_out_dtype dw_dtype,
                                int64_t ld_dw, int32_t accumulate, void* workspace, size_t workspace_bytes_, void* stream)
{
    if (!valid_type(dw_dtype) || !std::isfinite(scale)) return SNIP_ERR_FORMAT;
    if (tokens < 0 || tokens >= (int64_t)1 << 30 || vocab <= 0 || vocab > kMostTable || cols <= 0 || cols >= kMostWidth || cols % 8 != 0) return SNIP_ERR_SHAPE;
    snip_status st = check_rows(dy, tokens, cols, ld_dy);
    if (st == SNIP_OK) st = check_rows(dw, vocab, cols, ld_dw);
    if (st == SNIP_OK) st = check_index(ids, id_dtype, tokens);
    if (st == SNIP_OK) st = check_workspace(workspace, workspace_bytes_, embed_workspace_bytes(tokens, cols, vocab));
    if (st != SNIP_OK) return st;
    EmbedGradArgs a = {};
    a.dy = (const uint16_t*)dy; a.ld = ld_dy; a.ids = ids; a.ids64 = id_dtype == SNIP_INDEX_I64; a.tokens = tokens; a.vocab = vocab; a.cols = (int)cols;
    a.scale = scale; a.dw = dw; a.dw_fp32 = dw_dtype == SNIP_OUT_FP32; a.lddw = ld_dw; a.add = accumulate != 0; a.workspace = workspace;
    return launch_embed_backward(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

static bool vocab_extents(int64_t tokens, int64_t cols, int64_t vocab, int64_t k) { return tokens >= 0 && cols > 0 && vocab > 0 && k > 0; }
size_t snip_vocab_loss_workspace_bytes(int64_t tokens, int64_t cols, int64_t vocab, int64_t k)
{
    return vocab_extents(tokens, cols, vocab, k) ? vocab_loss_bytes(tokens, vocab, k) : 0;
}
size_t snip_vocab_loss_backward_workspace_bytes(int64_t tokens, int64_t cols, int64_t vocab, int64_t k)
{
    return vocab_extents(tokens, cols, vocab, k) ? vocab_loss_backward_bytes(tokens, cols, vocab, k) : 0;
}

static VocabLossArgs loss_args(const void* x, int64_t tokens, int64_t cols, int64_t ld_x, const void* w, int64_t vocab, int64_t ld_w, const void* indices,
                               int index_dtype, bool distill, const void* teacher, int teacher_dtype, int64_t k, float tau, void* workspace)
{
    VocabLossArgs a = {};
    a.x = (const uint16_t*)x; a.tokens = tokens; a.cols = cols; a.ldx = ld_x; a.w = (const uint16_t*)w; a.vocab = vocab; a.ldw = ld_w;
    a.indices = indices; a.index64 = index_dtype == SNIP_INDEX_I64; a.distill = distill; a.teacher = teacher; a.teacher_fp32 = teacher_dtype == SNIP_OUT_FP32;
    a.k = k; a.tau = tau; a.workspace = workspace;
    return a;
}
static void grad_args(VocabLossArgs& a, const float* lse, const float* dloss, void* dx, int64_t ld_dx, void* dw, int dw_dtype, int64_t ld_dw, int32_t accumulate)
{
    a.lse_in = lse; a.dloss = dloss; a.dx = (uint16_t*)dx; a.lddx = ld_dx; a.dw = dw; a.dw_fp32 = dw_dtype == SNIP_OUT_FP32; a.lddw = ld_dw; a.add = accumulate != 0;
}

snip_status snip_cross_entropy(const void* x, int64_t tokens, int64_t cols, int64_t ld_x, const void* w, int64_t vocab, int64_t ld_w,
                               const void* targets, snip_index_dtype index_dtype, float* loss, float* lse, void* workspace,
                               size_t workspace_bytes_, void* stream)
{
    VocabLossArgs a = loss_args(x, tokens, cols, ld_x, w, vocab, ld_w, targets, index_dtype, false, nullptr, SNIP_OUT_BF16, 1, 1.f, workspace);
    a.loss = loss; a.lse = lse;
    return vocab_loss(a, index_dtype, workspace_bytes_, stream);
}
snip_status snip_cross_entropy_backward(const void* x, int64_t tokens, int64_t cols, int64_t ld_x, const void* w, int64_t vocab,
                                        int64_t ld_w, const void* targets, snip_index_dtype index_dtype, const float* lse,
                                        const float* dloss, void* dx, int64_t ld_dx, void* dw, snip_out_dtype dw_dtype, int64_t ld_dw,
                                        int32_t accumulate, void* workspace, size_t workspace_bytes_, void* stream)
{
    VocabLossArgs a = loss_args(x, tokens, cols, ld_x, w, vocab, ld_w, targets, index_dtype, false, nullptr, SNIP_OUT_BF16, 1, 1.f, workspace);
    grad_args(a, lse, dloss, dx, ld_dx, dw, dw_dtype, ld_dw, accumulate);
    return vocab_loss_backward(a, index_dtype, dw_dtype, workspace_bytes_, stream);
}
snip_status snip_distill(const void* x, int64_t tokens, int64_t cols, int64_t ld_x, const void* w, int64_t vocab, int64_t ld_w,
                         const void* indices, snip_index_dtype index_dtype, const void* teacher, snip_out_dtype teacher_dtype, int64_t k,
                         float temperature, float* loss, float* lse, void* workspace, size_t workspace_bytes_, void* stream)
{
    const snip_status st = check_teacher(teacher, teacher_dtype, tokens);
    if (st != SNIP_OK) return st;
    VocabLossArgs a = loss_args(x, tokens, cols, ld_x, w, vocab, ld_w, indices, index_dtype, true, teacher, teacher_dtype, k, temperature, workspace);
    a.loss = loss; a.lse = lse;
    return vocab_loss(a, index_dtype, workspace_bytes_, stream);
}
snip_status snip_distill_backward(const void* x, int64_t tokens, int64_t cols, int64_t ld_x, const void* w, int64_t vocab, int64_t ld_w,
                                  const void* indices, snip_index_dtype index_dtype, const void* teacher, snip_out_dtype teacher_dtype,
                                  int64_t k, float temperature, const float* lse, const float* dloss, void* dx, int64_t ld_dx, void* dw,
                                  snip_out_dtype dw_dtype, int64_t ld_dw, int32_t accumulate, void* workspace, size_t workspace_bytes_,
                                  void* stream)
{
    const snip_status st = check_teacher(teacher, teacher_dtype, tokens);
    if (st != SNIP_OK) return st;
    VocabLossArgs a = loss_args(x, tokens, cols, ld_x, w, vocab, ld_w, indices, index_dtype, true, teacher, teacher_dtype, k, temperature, workspace);
    grad_args(a, lse, dloss, dx, ld_dx, dw, dw_dtype, ld_dw, accumulate);
    return vocab_loss_backward(a, index_dtype, dw_dtype, workspace_bytes_, stream);
}

size_t snip_noalloc_max_cols(void) { return (size_t)kNoallocMaxCols; }

snip_status snip_quant_error_stats_noalloc(const void* x, int64_t rows, int64_t cols, int64_t ld, snip_axis axis,
                                           snip_scale_rule rule, snip_stats* out, float* per_line, void* stream)
{
    snip_status st = check_source(x, rows, cols, ld, axis, rule);
    if (st != SNIP_OK) return st;
    if (!out) return SNIP_ERR_NULL;
    if (cols > kNoallocMaxCols) return SNIP_ERR_WORKSPACE;         // the resident scratch array is sized for this many columns
    // device address of this device's copy of the array, looked up once per device
    constexpr int kMaxDevices = 64;
    static void* g_scratch_ptr[kMaxDevices] = {};
    static std::mutex g_scratch_mutex;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return SNIP_ERR_HIP;
    void* ptr;
    {
        std::lock_guard<std::mutex> lock(g_scratch_mutex);
        if (!g_scratch_ptr[dev]) {
            void* p = nullptr;
            if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) return SNIP_ERR_HIP;
            g_scratch_ptr[dev] = p;
        }
        ptr = g_scratch_ptr[dev];
    }
    StatsArgs a;
    a.x = (const uint16_t*)x; a.rows = rows; a.cols = cols; a.ld = ld; a.axis = axis; a.rule = rule;
    a.stats = (double*)out; a.per_line = per_line; a.workspace = ptr;
    return launch_stats(a, (hipStream_t)stream) == hipSuccess ? SNIP_OK : SNIP_ERR_HIP;
}

const char* snip_status_string(snip_status s)
{
    switch (s) {
        case SNIP_OK: return "ok";
        case SNIP_ERR_NULL: return "null pointer";
        case SNIP_ERR_SHAPE: return "bad shape";
        case SNIP_ERR_FORMAT: return "bad format or enum";
        case SNIP_ERR_LAYOUT: return "bad alignment or mismatched operands";
        case SNIP_ERR_WORKSPACE: return "workspace missing or too small";
        case SNIP_ERR_HIP: return "kernel launch failed";
    }
    return "unknown status";
}

}  // extern "C"
