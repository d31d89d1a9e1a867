// rms_norm.hip -- root-mean-square norm with the residual's addition
// (tg_rms_norm) and its gradient (tg_rms_norm_grad); the kernels are norm.h's.
#include "norm.h"

namespace tg {
namespace {

// A block takes rows blockIdx.x, + gridDim.x, ... and keeps its columns' share of
// dweight in registers over all of them; one row of sums a block leaves it.  The
// weight stays in registers too, except in blocks of 1024, whose threads have 128.
// 8192 x 8192 in bf16 with 768 or 1024 blocks took 24 and 11 us more than with 512, with
// the next row fetched ahead the same.  Short rows are bound by latency: the 512 blocks
// have a wave each up to 64 units a row, and 16384 x 512 in bf16 takes 47 us, 1.4 TB/s.
template <typename E, int T, int N>
__global__ __launch_bounds__(T) void norm_grad_kernel(GradArgs a) {
    constexpr int kUnit = kUnitOf<E>;
    using unit = vec<float, kUnit>;
    __shared__ float slots[2][T / 64];
    const int t = threadIdx.x;
    const int units = (a.cols + kUnit - 1) / kUnit;
    constexpr bool kKeep = T < 1024;
    unit kept[N], dw[N];
    const auto weight = [&](int n) {
        const int u = t + n * T;
        return u < units ? load_f32<E, kUnit>((const E *)a.weight + u * kUnit, left_of(a.cols, u * kUnit)) : unit(0.0f);
    };
#pragma unroll
    for (int n = 0; n < N; ++n) {
        dw[n] = unit(0.0f);
        if (kKeep) kept[n] = weight(n);
    }
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const E *const dy = (const E *)a.dy + row * a.lddy;
        const E *const hidden = (const E *)a.hidden + row * a.ldh;
        const E *const dh = a.dhidden ? (const E *)a.dhidden + row * a.lddh : nullptr;
        unit g[N], h[N], more[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int u = t + n * T, valid = u < units ? left_of(a.cols, u * kUnit) : 0;
            g[n] = h[n] = more[n] = unit(0.0f);
            if (u >= units) continue;
            g[n] = load_f32<E, kUnit>(dy + u * kUnit, valid);
            h[n] = load_f32<E, kUnit>(hidden + u * kUnit, valid);
            if (dh) more[n] = load_f32<E, kUnit>(dh + u * kUnit, valid);
        }
        const float rstd = a.rstd[row];
        float dot = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const unit w = kKeep ? kept[n] : weight(n);
#pragma unroll
            for (int e = 0; e < kUnit; ++e) {
                const float xhat = h[n][e] * rstd;
                dw[n][e] = fmaf(g[n][e], xhat, dw[n][e]);
                g[n][e] *= w[e];
                h[n][e] = xhat;
                dot = fmaf(g[n][e], xhat, dot);
            }
        }
        // the slots of the row before last are free: a barrier lies between
        const float mean = block_reduce<OpSum, T>(dot, slots[turn]) * a.inv_cols;
        E *const dx = (E *)a.dx + row * a.lddx;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int u = t + n * T;
            if (u >= units) continue;
            unit d;
#pragma unroll
            for (int e = 0; e < kUnit; ++e) d[e] = fmaf(rstd, fmaf(-h[n][e], mean, g[n][e]), more[n][e]);
            store_f32<E, kUnit>(dx + u * kUnit, d, left_of(a.cols, u * kUnit));
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int u = t + n * T;
        if (u < units)
            store_f32<float, kUnit>(a.partial + (int64_t)blockIdx.x * a.cols + u * kUnit, dw[n], left_of(a.cols, u * kUnit));
    }
}

// Blocks of the gradient: each leaves a row of sums, so no more than fill the
// chip a few times over.
int grad_blocks(int64_t rows) { return (int)(rows < 512 ? rows : 512); }

template <typename E>
hipError_t launch_grad(GradArgs a, hipStream_t s) {
    const int units = (a.cols + kUnitOf<E> - 1) / kUnitOf<E>;
    const dim3 grid((unsigned)grad_blocks(a.rows));
    const auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, a); };
    constexpr int kMost = kUnitOf<E> == 4 ? 4096 : 2048;  // units of a row that stays in registers
    if (units <= 64) {
        go(norm_grad_kernel<E, 64, 1>, 64);
    } else if (units <= 256) {
        go(norm_grad_kernel<E, 256, 1>, 256);
    } else if (units <= 512) {
        go(norm_grad_kernel<E, 256, 2>, 256);
    } else if (units <= 1024) {
        go(norm_grad_kernel<E, 512, 2>, 512);
    } else if (units <= 2048) {
        go(norm_grad_kernel<E, 1024, 2>, 1024);
    } else if (units <= kMost) {
        go(norm_grad_kernel<E, 1024, kMost / 1024>, 1024);
    } else {
        launch_grad_stream<E, false>(a, grid.x, s);
    }
    return hipGetLastError();
}

}  // namespace
}  // namespace tg

using namespace tg;

extern "C" {

tg_status tg_rms_norm(const tg_rms_norm_args *q, tg_stream stream) {
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
        if (q->residual) TG_TRY(check_rows(q->residual, q->ldr, q->rows, q->cols, q->type, "residual"));
        if (q->hidden) TG_TRY(check_rows(q->hidden, q->ldh, q->rows, q->cols, q->type, "hidden"));
    }
    if (q->out_type == TG_E4M3) TG_TRY(check_rows(q->scale, 0, 1, 1, TG_F32, "scale"));
    if (q->rstd) TG_TRY(check_rows(q->rstd, 0, 1, 1, TG_F32, "rstd"));
    const bool one = q->rows == 1;
    NormArgs a{q->x, q->residual, q->weight, nullptr, q->hidden, q->y, q->scale, nullptr, q->rstd, q->rows,
               one ? 0 : q->ldx, one ? 0 : q->ldr, one ? 0 : q->ldh, one ? 0 : q->ldy,
               0, (int)q->cols, q->eps, q->cols ? (float)(1.0 / (double)q->cols) : 0.0f};
    const hipStream_t s = (hipStream_t)stream;
    const bool eight = q->out_type == TG_E4M3;
    hipError_t e;
    if (q->type == TG_F32)
        e = eight ? launch_norm<float, true, false>(a, s) : launch_norm<float, false, false>(a, s);
    else if (q->type == TG_BF16)
        e = eight ? launch_norm<bf16, true, false>(a, s) : launch_norm<bf16, false, false>(a, s);
    else
        e = eight ? launch_norm<f16, true, false>(a, s) : launch_norm<f16, false, false>(a, s);
    return e == hipSuccess ? TG_OK : device_failed(e, "norm_kernel");
}

size_t tg_rms_norm_grad_workspace_bytes(const tg_rms_norm_grad_args *q) {
    if (!q || q->rows < 0 || q->cols < 0 || q->rows > 0x7fffffff || q->cols > 0x7fffffff - 64) return 0;
    return round256((size_t)grad_blocks(q->rows) * q->cols * 4);
}

tg_status tg_rms_norm_grad(const tg_rms_norm_grad_args *q, void *d_ws, size_t ws_bytes, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    TG_TRY(check_sizes(q->rows, q->cols));
    if (q->reserved) return call_failed(TG_EINVAL, "reserved must be 0");
    if (!norm_type(q->type)) return call_failed(TG_EINVAL, "type %d", q->type);
    if (q->cols == 0) return TG_OK;
    TG_TRY(check_rows(q->dweight, 0, 1, q->cols, q->type, "dweight"));
    const hipStream_t s = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    if (q->rows > 0) {
        TG_TRY(check_rows(q->dy, q->lddy, q->rows, q->cols, q->type, "dy"));
        TG_TRY(check_rows(q->hidden, q->ldh, q->rows, q->cols, q->type, "hidden"));
        TG_TRY(check_rows(q->weight, 0, 1, q->cols, q->type, "weight"));
        TG_TRY(check_rows(q->dx, q->lddx, q->rows, q->cols, q->type, "dx"));
        TG_TRY(check_rows(q->rstd, 0, 1, 1, TG_F32, "rstd"));
        if (q->dhidden) TG_TRY(check_rows(q->dhidden, q->lddh, q->rows, q->cols, q->type, "dhidden"));
        if ((uintptr_t)d_ws % 256) return call_failed(TG_EINVAL, "the workspace is not 256-byte aligned");
        const size_t need = tg_rms_norm_grad_workspace_bytes(q);
        if (ws_bytes < need || !d_ws) return call_failed(TG_ENOMEM, "workspace of %zu bytes, %zu needed", d_ws ? ws_bytes : 0, need);
        const bool one = q->rows == 1;
        GradArgs a{q->dy, q->dhidden, q->hidden, q->weight, nullptr, q->rstd, q->dx, (float *)d_ws, nullptr, q->rows,
                   one ? 0 : q->lddy, one ? 0 : q->lddh, one ? 0 : q->ldh, one ? 0 : q->lddx,
                   0, (int)q->cols, (float)(1.0 / (double)q->cols)};
        e = q->type == TG_F32 ? launch_grad<float>(a, s) : q->type == TG_BF16 ? launch_grad<bf16>(a, s) : launch_grad<f16>(a, s);
        if (e != hipSuccess) return device_failed(e, "norm_grad_kernel");
    }
    e = launch_column_sums((const float *)d_ws, grad_blocks(q->rows), q->cols, q->dweight, q->type, s);
    return e == hipSuccess ? TG_OK : device_failed(e, "column_sums");
}

}  // extern "C"
