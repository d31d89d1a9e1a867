// layer_norm.hip -- layer norm with the residual's addition (tg_layer_norm) and its
// gradient (tg_layer_norm_grad); the kernels are norm.h's.
#include "norm.h"

using namespace tg;

extern "C" {

tg_status tg_layer_norm(const tg_layer_norm_args *q, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    TG_TRY(check_sizes(q->rows, q->cols));
    if (q->reserved) return call_failed(TG_EINVAL, "reserved must be 0");
    if (!norm_type(q->type)) return call_failed(TG_EINVAL, "type %d", q->type);
    if (q->out_type != q->type && q->out_type != TG_E4M3) return call_failed(TG_EINVAL, "out_type %d", q->out_type);
    if (!(std::isfinite(q->eps) && q->eps >= 0)) return call_failed(TG_EINVAL, "eps must be finite and not negative");
    if (q->out_type != TG_E4M3 && q->scale) return call_failed(TG_EINVAL, "a scale belongs to an 8-bit output");
    if (q->rows == 0) return TG_OK;
    if (q->cols > 0) {
        TG_TRY(check_rows(q->x, q->ldx, q->rows, q->cols, q->type, "x"));
        TG_TRY(check_rows(q->y, q->ldy, q->rows, q->cols, q->out_type, "y"));
        TG_TRY(check_rows(q->weight, 0, 1, q->cols, q->type, "weight"));
        if (q->bias) TG_TRY(check_rows(q->bias, 0, 1, q->cols, q->type, "bias"));
        if (q->residual) TG_TRY(check_rows(q->residual, q->ldr, q->rows, q->cols, q->type, "residual"));
        if (q->hidden) TG_TRY(check_rows(q->hidden, q->ldh, q->rows, q->cols, q->type, "hidden"));
    }
    if (q->out_type == TG_E4M3) TG_TRY(check_rows(q->scale, 0, 1, 1, TG_F32, "scale"));
    if (q->mean) TG_TRY(check_rows(q->mean, 0, 1, 1, TG_F32, "mean"));
    if (q->rstd) TG_TRY(check_rows(q->rstd, 0, 1, 1, TG_F32, "rstd"));
    const bool one = q->rows == 1;
    NormArgs a{q->x, q->residual, q->weight, q->bias, q->hidden, q->y, q->scale, q->mean, q->rstd, q->rows,
               one ? 0 : q->ldx, one ? 0 : q->ldr, one ? 0 : q->ldh, one ? 0 : q->ldy,
               0, (int)q->cols, q->eps, q->cols ? (float)(1.0 / (double)q->cols) : 0.0f};
    const hipStream_t s = (hipStream_t)stream;
    const bool eight = q->out_type == TG_E4M3;
    hipError_t e;
    if (q->type == TG_F32)
        e = eight ? launch_norm<float, true, true>(a, s) : launch_norm<float, false, true>(a, s);
    else if (q->type == TG_BF16)
        e = eight ? launch_norm<bf16, true, true>(a, s) : launch_norm<bf16, false, true>(a, s);
    else
        e = eight ? launch_norm<f16, true, true>(a, s) : launch_norm<f16, false, true>(a, s);
    return e == hipSuccess ? TG_OK : device_failed(e, "norm_kernel");
}

size_t tg_layer_norm_grad_workspace_bytes(const tg_layer_norm_grad_args *q) {
    if (!q || q->rows < 0 || q->cols < 0 || q->rows > 0x7fffffff || q->cols > 0x7fffffff - 64) return 0;
    return round256((size_t)grad_blocks(q->rows) * q->cols * (q->dbias ? 8 : 4));
}

tg_status tg_layer_norm_grad(const tg_layer_norm_grad_args *q, void *d_ws, size_t ws_bytes, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    TG_TRY(check_sizes(q->rows, q->cols));
    if (q->reserved) return call_failed(TG_EINVAL, "reserved must be 0");
    if (!norm_type(q->type)) return call_failed(TG_EINVAL, "type %d", q->type);
    if (q->cols == 0) return TG_OK;
    TG_TRY(check_rows(q->dweight, 0, 1, q->cols, q->type, "dweight"));
    if (q->dbias) TG_TRY(check_rows(q->dbias, 0, 1, q->cols, q->type, "dbias"));
    const hipStream_t s = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    if (q->rows > 0) {
        TG_TRY(check_rows(q->dy, q->lddy, q->rows, q->cols, q->type, "dy"));
        TG_TRY(check_rows(q->hidden, q->ldh, q->rows, q->cols, q->type, "hidden"));
        TG_TRY(check_rows(q->weight, 0, 1, q->cols, q->type, "weight"));
        TG_TRY(check_rows(q->dx, q->lddx, q->rows, q->cols, q->type, "dx"));
        TG_TRY(check_rows(q->mean, 0, 1, 1, TG_F32, "mean"));
        TG_TRY(check_rows(q->rstd, 0, 1, 1, TG_F32, "rstd"));
        if (q->dhidden) TG_TRY(check_rows(q->dhidden, q->lddh, q->rows, q->cols, q->type, "dhidden"));
        if ((uintptr_t)d_ws % 256) return call_failed(TG_EINVAL, "the workspace is not 256-byte aligned");
        const size_t need = tg_layer_norm_grad_workspace_bytes(q);
        if (ws_bytes < need || !d_ws) return call_failed(TG_ENOMEM, "workspace of %zu bytes, %zu needed", d_ws ? ws_bytes : 0, need);
        const bool one = q->rows == 1;
        float *const sums = (float *)d_ws;
        GradArgs a{q->dy, q->dhidden, q->hidden, q->weight, q->mean, q->rstd, q->dx, sums,
                   q->dbias ? sums + (int64_t)grad_blocks(q->rows) * q->cols : nullptr, q->rows,
                   one ? 0 : q->lddy, one ? 0 : q->lddh, one ? 0 : q->ldh, one ? 0 : q->lddx,
                   0, (int)q->cols, (float)(1.0 / (double)q->cols)};
        e = q->type == TG_F32    ? launch_grad<float, true>(a, s)
            : q->type == TG_BF16 ? launch_grad<bf16, true>(a, s)
                                 : launch_grad<f16, true>(a, s);
        if (e != hipSuccess) return device_failed(e, "norm_grad_kernel");
    }
    e = launch_column_sums_of_two((const float *)d_ws, grad_blocks(q->rows), q->cols, q->dweight, q->dbias, q->type, s);
    return e == hipSuccess ? TG_OK : device_failed(e, "column_sums");
}

}  // extern "C"
