// The linear layer in 8-bit floating point: plans, checks and the calls of include/wq.h.
#include <new>

#include "wq_fp8_form.h"
#include "wq_fp8_quantize.h"
#include "wq_layer_norm_args.h"

namespace {

uint64_t up256(uint64_t v) { return (v + 255) / 256 * 256; }

bool good_buffer(const void *b) { return b && (uintptr_t)b % 16 == 0; }
bool good_type(int type) { return type == WQ_FP32 || type == WQ_BF16 || type == WQ_FP16; }
int type_size(int type) { return type == WQ_FP32 ? 4 : 2; }

// A tensor [rows][cols] of the type with a row stride: aligned to its elements, rows that do not overlap.
bool good_rows(const void *t, int64_t stride, int rows, int cols, int type) {
    return ((uintptr_t)t % type_size(type)) == 0 && (rows <= 1 || (stride >= cols && stride <= INT64_MAX / 16 / rows));
}

wq_status_t status(hipError_t e) { return e == hipSuccess ? WQ_OK : WQ_ERR_DEVICE; }

// An operand in planes of a piece of all R rows: codes in `groups` groups of 128, or values in twice as many of 64.
wq_fp8_operand planes(const void *data, const float *scales, int rows, int R, int groups, bool values) {
    const unsigned piece = 16u * (unsigned)R;
    return {(const uint8_t *)data, scales, (unsigned)groups * (values ? 16u : 8u) * piece, 256u, 8u * piece, piece, rows, R};
}
// Weights in 16-row blocks.
wq_fp8_operand blocks(const uint8_t *codes, const float *scales, int rows16, int groups, int scale_step) {
    return {codes, scales, (unsigned)rows16 * (unsigned)groups * 128u, 2048u * (unsigned)groups, 2048u, 256u, rows16, scale_step};
}

wq_status_t check_calls(const wq_fp8_plan *plan, int rows, int type, int activation, int gated) {
    if (!plan) return WQ_ERR_INVALID_ARG;
    if (rows < 0 || rows > plan->P || !good_type(type) || activation < WQ_ACT_NONE || activation > WQ_ACT_GELU_TANH || (gated != 0 && gated != 1))
        return WQ_ERR_INVALID_ARG;
    if (gated && plan->Cout % 64 != 0) return WQ_ERR_UNSUPPORTED;
    return WQ_OK;
}

// What wq_fp8_matmul and wq_fp8_forward check about the product.
wq_status_t check_product(const wq_fp8_plan *plan, int rows, const void *workspace, size_t workspace_bytes, const void *blob, size_t blob_bytes,
                          int activation, int gated, int type, const void *res, int64_t res_stride, const void *pre, int64_t pre_stride,
                          const void *y, int64_t y_stride) {
    if (!plan || !good_buffer(workspace) || !good_buffer(blob) || (rows != 0 && !y)) return WQ_ERR_INVALID_ARG;
    const wq_status_t st = check_calls(plan, rows, type, activation, gated);
    if (st != WQ_OK) return st;
    const int outs = gated ? plan->Cout / 2 : plan->Cout;
    if (!good_rows(y, y_stride, rows, outs, type) || (res && !good_rows(res, res_stride, rows, outs, type)) ||
        (pre && !good_rows(pre, pre_stride, rows, plan->Cout, type)))
        return WQ_ERR_INVALID_ARG;
    if (workspace_bytes < plan->lay.ws_bytes || blob_bytes < plan->lay.blob_bytes) return WQ_ERR_WORKSPACE;
    return plan->prepared.load() ? WQ_OK : WQ_ERR_NOT_PREPARED;
}

void set_wide(wq_fp8_product &p) {
    const int64_t piece = 4 * type_size(p.type);
    auto whole = [&](const void *t, int64_t stride) { return !t || ((uintptr_t)t % piece == 0 && (p.rows == 1 || stride % 4 == 0)); };
    p.wide = whole(p.y, p.ys) && whole(p.res, p.rs) && whole(p.pre, p.ps);
}

// exact: sums that keep 24 bits (a kernel for few rows, which reads weights all the while, has no others)
wq_status_t run_product(const wq_fp8_plan *plan, wq_fp8_product &p, bool exact, hipStream_t s) {
    set_wide(p);
    const wq_fp8_form form = wq_fp8_choose_form(p.rows, p.outs, p.gated, p.groups, exact);
    if (form.row_blocks) return status(wq_launch_fp8_rows(p, form.row_blocks, s));
    const int mode = exact ? plan->fp32_scales ? WQ_FP8_EXACT_FP32 : WQ_FP8_EXACT : plan->fp32_scales ? WQ_FP8_DIRECT_FP32 : WQ_FP8_DIRECT;
    return status(wq_launch_fp8_tile(p, mode, form.tile, s));
}

bool is_captured(hipStream_t s) {
    hipStreamCaptureStatus status;
    if (hipStreamIsCapturing(s, &status) == hipSuccess) return status != hipStreamCaptureStatusNone;
    (void)hipGetLastError();   // (the question's own: the launch that follows has its answer checked)
    return false;
}

// Whether the product takes the rows of x as they are: few of them, and apart from what some workgroups write while others still
// read x.
bool quantizes_itself(const wq_fp8_product &p, const void *x, int64_t xs, int Cin, hipStream_t s) {
    const wq_fp8_form form = wq_fp8_choose_form(p.rows, p.outs, p.gated, p.groups, true);
    if (!wq_fp8_takes_rows(form, p.rows, Cin, false) || (!wq_fp8_takes_rows(form, p.rows, Cin, true) && is_captured(s))) return false;
    const int64_t e = type_size(p.type), last = p.rows - 1;
    const char *x0 = (const char *)x, *x1 = x0 + (last * xs + Cin) * e;
    auto apart = [&](const void *t, int64_t stride, int cols) {
        const char *t0 = (const char *)t, *t1 = t0 + (last * stride + cols) * e;
        return !t || x1 <= t0 || t1 <= x0;
    };
    return apart(p.y, p.ys, p.outs) && apart(p.pre, p.ps, p.cols);
}

wq_fp8_product forward_product(const wq_fp8_plan *plan, int rows, const void *workspace, const void *blob, int activation, int gated, int type,
                               const void *res, int64_t res_stride, void *pre, int64_t pre_stride, void *y, int64_t y_stride) {
    const char *ws = (const char *)workspace, *b = (const char *)blob;
    const wq_fp8_layout_t &L = plan->lay;
    wq_fp8_product p = {};
    p.a = blocks((const uint8_t *)(b + L.blob_codes_off), (const float *)(b + L.blob_scales_off), plan->Cout16, plan->in_blocks, plan->in_blocks);
    p.b = planes((const uint8_t *)(ws + L.ws_codes_off), (const float *)(ws + L.ws_scales_off), rows, plan->P, plan->in_blocks, false);
    p.groups = plan->in_blocks;
    p.bias = (const float *)(b + L.blob_bias_off);
    p.res = res; p.y = y; p.pre = pre; p.rs = res_stride; p.ys = y_stride; p.ps = pre_stride;
    p.rows = rows; p.outs = gated ? plan->Cout / 2 : plan->Cout; p.cols = plan->Cout;
    p.type = type; p.act = activation; p.gated = gated;
    return p;
}

wq_status_t prepare_weights(wq_fp8_plan *plan, hipStream_t s, wq_fp8_weight_args &a, int type, bool load, void *blob) {
    char *b = (char *)blob;
    const wq_fp8_layout_t &L = plan->lay;
    a.codes = (uint8_t *)(b + L.blob_codes_off);
    a.codesT = plan->backward ? (uint8_t *)(b + L.blob_codes_t_off) : nullptr;
    a.scales = (float *)(b + L.blob_scales_off);
    a.scalesT = (float *)(b + L.blob_scales_t_off);
    a.bias_out = (float *)(b + L.blob_bias_off);
    a.Cin = plan->Cin; a.Cout = plan->Cout; a.Cin16 = plan->Cin16; a.Cout16 = plan->Cout16;
    a.in_blocks = plan->in_blocks; a.out_blocks = plan->out_blocks;
    if (wq_launch_fp8_weights(a, type, load, s) != hipSuccess) return WQ_ERR_DEVICE;
    plan->prepared.store(1);
    return WQ_OK;
}

}  // namespace

// ------------------------------------------------------------------ C ABI
extern "C" {

wq_status_t wq_fp8_plan_create(wq_fp8_plan_t **out, int rows, int Cin, int Cout, int backward, int fp32_scales) {
    if (!out) return WQ_ERR_INVALID_ARG;
    *out = nullptr;
    if (rows < 1 || Cin < 1 || Cout < 1 || (backward != 0 && backward != 1) || (fp32_scales != 0 && fp32_scales != 1)) return WQ_ERR_INVALID_ARG;
    // every buffer that a kernel addresses stays below 2 GiB: codes, and along the rows values of two bytes
    const uint64_t most = (1ull << 31) - 1, R = (uint64_t)rows;
    const uint64_t B = ((uint64_t)Cin + 127) / 128, O = ((uint64_t)Cout + 127) / 128, TB = (R + 127) / 128;
    const uint64_t Cin16 = ((uint64_t)Cin + 15) / 16 * 16, Cout16 = ((uint64_t)Cout + 15) / 16 * 16;
    if (B * 128 * R > most || B * 128 * Cout16 > most || O * B * 4 > most) return WQ_ERR_UNSUPPORTED;
    if (backward && (O * 128 * R > most || O * 128 * Cin16 > most || TB * 256 * Cin16 > most || TB * 256 * Cout16 > most))
        return WQ_ERR_UNSUPPORTED;
    wq_fp8_plan *p = new (std::nothrow) wq_fp8_plan();
    if (!p) return WQ_ERR_DEVICE;
    p->P = rows; p->Cin = Cin; p->Cout = Cout;
    p->in_blocks = (int)B; p->out_blocks = (int)O; p->Cin16 = (int)Cin16; p->Cout16 = (int)Cout16;
    p->backward = backward; p->fp32_scales = fp32_scales;
    wq_fp8_layout_t &L = p->lay;
    L = {};
    L.rows = rows; L.Cin = Cin; L.Cout = Cout; L.in_blocks = (int)B; L.out_blocks = (int)O; L.backward = backward; L.fp32_scales = fp32_scales;
    L.blob_codes_off = 0;
    L.blob_scales_off = up256(B * 128 * Cout16);
    L.blob_bias_off = L.blob_scales_off + up256(O * B * 4);
    L.blob_codes_t_off = L.blob_bias_off + up256(Cout16 * 4);
    L.blob_scales_t_off = L.blob_codes_t_off + (backward ? up256(O * 128 * Cin16) : 0);
    L.blob_bytes = L.blob_scales_t_off + (backward ? up256(O * B * 4) : 0);
    L.ws_codes_off = 0;
    L.ws_scales_off = up256(B * 128 * R);
    uint64_t at = L.ws_scales_off + up256(B * R * 4);
    auto take = [&](uint64_t &off, uint64_t bytes) {
        off = at;
        if (backward) at += up256(bytes);
    };
    take(L.ws_dz_codes_off, O * 128 * R);
    take(L.ws_dz_scales_off, O * R * 4);
    take(L.ws_xt_off, TB * 256 * Cin16);
    take(L.ws_xt_scales_off, TB * Cin16 * 4);
    take(L.ws_dzt_off, TB * 256 * Cout16);
    take(L.ws_dzt_scales_off, TB * Cout16 * 4);
    take(L.ws_db_off, TB * (uint64_t)Cout * 4);
    L.ws_bytes = at;
    p->prepared.store(0);
    *out = p;
    return WQ_OK;
}

wq_status_t wq_fp8_plan_destroy(wq_fp8_plan_t *plan) {
    if (!plan) return WQ_ERR_INVALID_ARG;
    delete plan;
    return WQ_OK;
}

wq_status_t wq_fp8_plan_layout(const wq_fp8_plan_t *plan, wq_fp8_layout_t *out) {
    if (!plan || !out) return WQ_ERR_INVALID_ARG;
    *out = plan->lay;
    return WQ_OK;
}

wq_status_t wq_fp8_weight_prepare(wq_fp8_plan_t *plan, void *stream, int type, const void *w_dev, int64_t w_stride,
                                  const float *bias_dev, void *weight_blob_dev, size_t blob_bytes) {
    if (!plan || !w_dev || !good_buffer(weight_blob_dev) || !good_type(type) || ((uintptr_t)bias_dev & 3) ||
        !good_rows(w_dev, w_stride, plan->Cout, plan->Cin, type))
        return WQ_ERR_INVALID_ARG;
    if (blob_bytes < plan->lay.blob_bytes) return WQ_ERR_WORKSPACE;
    wq_fp8_weight_args a = {};
    a.w = w_dev; a.ws = w_stride; a.bias = bias_dev;
    return prepare_weights(plan, (hipStream_t)stream, a, type, false, weight_blob_dev);
}

wq_status_t wq_fp8_weight_load(wq_fp8_plan_t *plan, void *stream, const void *codes_dev, int64_t codes_stride, int scale_type,
                               const void *scales_dev, const float *bias_dev, void *weight_blob_dev, size_t blob_bytes) {
    if (!plan || !codes_dev || !scales_dev || !good_buffer(weight_blob_dev) || ((uintptr_t)bias_dev & 3) ||
        (scale_type != WQ_SCALE_FP32 && scale_type != WQ_SCALE_E8M0) || (scale_type == WQ_SCALE_FP32 && ((uintptr_t)scales_dev & 3)) ||
        (plan->Cout > 1 && (codes_stride < plan->Cin || codes_stride > INT64_MAX / 16 / plan->Cout)))
        return WQ_ERR_INVALID_ARG;
    if (scale_type == WQ_SCALE_FP32 && !plan->fp32_scales) return WQ_ERR_UNSUPPORTED;
    if (blob_bytes < plan->lay.blob_bytes) return WQ_ERR_WORKSPACE;
    wq_fp8_weight_args a = {};
    a.w = codes_dev; a.ws = codes_stride; a.given = scales_dev; a.scale_type = scale_type; a.bias = bias_dev;
    return prepare_weights(plan, (hipStream_t)stream, a, WQ_BF16, true, weight_blob_dev);
}

wq_status_t wq_fp8_quantize(const wq_fp8_plan_t *plan, void *stream, int rows, int type, const void *x_dev, int64_t x_stride,
                            void *workspace_dev, size_t workspace_bytes) {
    if (!plan || (rows != 0 && !x_dev) || !good_buffer(workspace_dev)) return WQ_ERR_INVALID_ARG;
    if (rows < 0 || rows > plan->P || !good_type(type) || !good_rows(x_dev, x_stride, rows, plan->Cin, type)) return WQ_ERR_INVALID_ARG;
    if (workspace_bytes < plan->lay.ws_bytes) return WQ_ERR_WORKSPACE;
    if (rows == 0) return WQ_OK;
    char *ws = (char *)workspace_dev;
    wq_fp8_rows_args a = {};
    a.x = x_dev; a.xs = x_stride;
    a.codes = (uint8_t *)(ws + plan->lay.ws_codes_off);
    a.scales = (float *)(ws + plan->lay.ws_scales_off);
    a.rows = rows; a.P = plan->P; a.cols = plan->Cin; a.groups = plan->in_blocks;
    return status(wq_launch_fp8_quantize(a, type, (hipStream_t)stream));
}

wq_status_t wq_fp8_layer_norm_quantize(const wq_fp8_plan_t *plan, void *stream, int rows, int type, const void *x_dev,
                                       int64_t x_stride, const void *residual_dev, int64_t residual_stride,
                                       const float *gamma_dev, const float *beta_dev, double eps, void *sum_dev,
                                       int64_t sum_stride, void *workspace_dev, size_t workspace_bytes) {
    if (!plan || !good_buffer(workspace_dev) || rows > plan->P) return WQ_ERR_INVALID_ARG;
    char *ws = (char *)workspace_dev;
    wq_layer_norm_args a = {};
    a.x = x_dev; a.res = residual_dev; a.sum = sum_dev; a.gamma = gamma_dev; a.beta = beta_dev;
    a.xs = x_stride; a.rs = residual_stride; a.ss = sum_stride;
    a.rows = rows; a.C = plan->Cin; a.P = plan->P; a.padded = plan->in_blocks * kGroup; a.eps = eps;
    a.codes = (uint8_t *)(ws + plan->lay.ws_codes_off);
    a.scales = (float *)(ws + plan->lay.ws_scales_off);
    if (!wq_good_layer_norm(a, type)) return WQ_ERR_INVALID_ARG;
    if (workspace_bytes < plan->lay.ws_bytes) return WQ_ERR_WORKSPACE;
    if (rows == 0) return WQ_OK;
    return status(wq_launch_layer_norm(a, type, (hipStream_t)stream));
}

wq_status_t wq_fp8_matmul(const wq_fp8_plan_t *plan, void *stream, int rows, const void *workspace_dev, size_t workspace_bytes,
                          const void *weight_blob_dev, size_t blob_bytes, int activation, int gated, int type,
                          const void *residual_dev, int64_t residual_stride, void *pre_dev, int64_t pre_stride, void *y_dev,
                          int64_t y_stride) {
    const wq_status_t st = check_product(plan, rows, workspace_dev, workspace_bytes, weight_blob_dev, blob_bytes, activation, gated, type,
                                         residual_dev, residual_stride, pre_dev, pre_stride, y_dev, y_stride);
    if (st != WQ_OK || rows == 0) return st;
    wq_fp8_product p = forward_product(plan, rows, workspace_dev, weight_blob_dev, activation, gated, type, residual_dev, residual_stride,
                                       pre_dev, pre_stride, y_dev, y_stride);
    return run_product(plan, p, true, (hipStream_t)stream);
}

wq_status_t wq_fp8_forward(const wq_fp8_plan_t *plan, void *stream, int rows, int type, const void *x_dev, int64_t x_stride,
                           const void *weight_blob_dev, size_t blob_bytes, void *workspace_dev, size_t workspace_bytes,
                           int activation, int gated, const void *residual_dev, int64_t residual_stride, void *pre_dev,
                           int64_t pre_stride, void *y_dev, int64_t y_stride) {
    wq_status_t st = check_product(plan, rows, workspace_dev, workspace_bytes, weight_blob_dev, blob_bytes, activation, gated, type,
                                   residual_dev, residual_stride, pre_dev, pre_stride, y_dev, y_stride);
    if (st != WQ_OK) return st;
    if ((rows != 0 && !x_dev) || !good_rows(x_dev, x_stride, rows, plan->Cin, type)) return WQ_ERR_INVALID_ARG;
    if (rows == 0) return WQ_OK;
    wq_fp8_product p = forward_product(plan, rows, workspace_dev, weight_blob_dev, activation, gated, type, residual_dev, residual_stride,
                                       pre_dev, pre_stride, y_dev, y_stride);
    if (quantizes_itself(p, x_dev, x_stride, plan->Cin, (hipStream_t)stream)) {
        p.x = x_dev; p.xs = x_stride; p.xcols = plan->Cin;
    } else {
        st = wq_fp8_quantize(plan, stream, rows, type, x_dev, x_stride, workspace_dev, workspace_bytes);
        if (st != WQ_OK) return st;
    }
    return run_product(plan, p, true, (hipStream_t)stream);
}

wq_status_t wq_fp8_backward(const wq_fp8_plan_t *plan, void *stream, int rows, int type, const void *x_dev, int64_t x_stride,
                            const void *dy_dev, int64_t dy_stride, const void *pre_dev, int64_t pre_stride,
                            const void *weight_blob_dev, size_t blob_bytes, void *workspace_dev, size_t workspace_bytes,
                            int activation, int gated, void *dx_dev, int64_t dx_stride, int dw_type, void *dw_dev,
                            int64_t dw_stride, float *db_dev, int accumulate) {
    wq_status_t st = check_calls(plan, rows, type, activation, gated);
    if (st != WQ_OK) return st;
    if (!plan->backward) return WQ_ERR_UNSUPPORTED;
    const bool through = activation != WQ_ACT_NONE || gated;
    const int outs = gated ? plan->Cout / 2 : plan->Cout;
    if (!good_buffer(workspace_dev) || (accumulate != 0 && accumulate != 1) || ((uintptr_t)db_dev & 3) ||
        (dw_dev && ((dw_type != type && dw_type != WQ_FP32) || !good_rows(dw_dev, dw_stride, plan->Cout, plan->Cin, dw_type))) ||
        (dx_dev && (!good_buffer(weight_blob_dev) || !good_rows(dx_dev, dx_stride, rows, plan->Cin, type))))
        return WQ_ERR_INVALID_ARG;
    if (rows != 0 && (!dy_dev || (dw_dev && !x_dev) || (through && !pre_dev))) return WQ_ERR_INVALID_ARG;
    if (!good_rows(dy_dev, dy_stride, rows, outs, type) || (dw_dev && !good_rows(x_dev, x_stride, rows, plan->Cin, type)) ||
        (through && !good_rows(pre_dev, pre_stride, rows, plan->Cout, type)))
        return WQ_ERR_INVALID_ARG;
    if (workspace_bytes < plan->lay.ws_bytes || (dx_dev && blob_bytes < plan->lay.blob_bytes)) return WQ_ERR_WORKSPACE;
    if (dx_dev && !plan->prepared.load()) return WQ_ERR_NOT_PREPARED;
    hipStream_t s = (hipStream_t)stream;
    if (rows == 0) {
        if (accumulate || (!dw_dev && !db_dev)) return WQ_OK;
        return status(wq_launch_fp8_zero(dw_dev, plan->Cout, plan->Cin, dw_stride, dw_dev ? dw_type : WQ_FP32, db_dev, s));
    }
    if (!dx_dev && !dw_dev && !db_dev) return WQ_OK;
    const wq_fp8_layout_t &L = plan->lay;
    char *ws = (char *)workspace_dev;
    const int TB = (rows + kGroup - 1) / kGroup;
    const bool wide_values = dw_dev && dw_type == WQ_FP32;   // sums for an fp32 result are of bf16 values
    const int along = !dw_dev ? 0 : wide_values ? 2 : 1;
    hipError_t e;

    wq_fp8_both_args x = {}, q = {};
    x.rows = q.rows = rows; x.P = q.P = plan->P;
    if (dw_dev) {   // along the rows
        x.v = x_dev; x.vs = x_stride; x.cols = plan->Cin; x.colsT = plan->Cin16; x.groups = plan->in_blocks;
        x.codesT = (uint8_t *)(ws + L.ws_xt_off); x.scalesT = (float *)(ws + L.ws_xt_scales_off);
    }
    q.v = dy_dev; q.vs = dy_stride; q.pre = through ? pre_dev : nullptr; q.ps = pre_stride; q.act = activation; q.gated = gated;
    q.cols = plan->Cout; q.colsT = plan->Cout16; q.groups = plan->out_blocks;
    q.codesT = (uint8_t *)(ws + L.ws_dzt_off); q.scalesT = (float *)(ws + L.ws_dzt_scales_off);
    q.codes = dx_dev ? (uint8_t *)(ws + L.ws_dz_codes_off) : nullptr; q.scales = (float *)(ws + L.ws_dz_scales_off);
    q.db = db_dev ? (float *)(ws + L.ws_db_off) : nullptr;
    if ((e = wq_launch_fp8_both(x, q, type, along, s)) != hipSuccess) return status(e);
    if (db_dev && (e = wq_launch_fp8_db(q.db, TB, plan->Cout, db_dev, accumulate, s)) != hipSuccess) return status(e);

    if (dw_dev) {   // columns of dw are rows of `a`, x's columns
        const wq_fp8_form form = wq_fp8_choose_grad_form(plan->Cout, plan->Cin, TB);
        wq_fp8_product p = {};
        p.a = planes((const uint8_t *)(ws + L.ws_xt_off), (const float *)(ws + L.ws_xt_scales_off), plan->Cin16, plan->Cin16, TB, wide_values);
        p.b = planes((const uint8_t *)(ws + L.ws_dzt_off), (const float *)(ws + L.ws_dzt_scales_off), plan->Cout16, plan->Cout16, TB, wide_values);
        p.groups = TB;
        p.y = dw_dev; p.ys = dw_stride; p.rows = plan->Cout; p.outs = p.cols = plan->Cin; p.type = dw_type;
        if (accumulate) p.res = dw_dev, p.rs = dw_stride;
        set_wide(p);
        if ((e = wq_launch_fp8_tile(p, wide_values ? WQ_FP8_VALUES : WQ_FP8_DIRECT_ROWS, form.tile, s)) != hipSuccess) return status(e);
    }
    if (dx_dev) {
        const char *b = (const char *)weight_blob_dev;
        wq_fp8_product p = {};
        p.a = blocks((const uint8_t *)(b + L.blob_codes_t_off), (const float *)(b + L.blob_scales_t_off), plan->Cin16, plan->out_blocks, plan->out_blocks);
        p.b = planes((const uint8_t *)(ws + L.ws_dz_codes_off), (const float *)(ws + L.ws_dz_scales_off), rows, plan->P, plan->out_blocks, false);
        p.groups = plan->out_blocks;
        p.y = dx_dev; p.ys = dx_stride; p.rows = rows; p.outs = p.cols = plan->Cin; p.type = type;
        return run_product(plan, p, type == WQ_FP32, s);
    }
    return WQ_OK;
}

}  // extern "C"
