// layer_norm.hip -- layer norm with the residual's addition (tg_layer_norm) and its
// gradient (tg_layer_norm_grad); the forward kernels are norm.h's.
//
// Both are bound by memory as the root-mean-square norm's are.  8192 x 12288 in bf16
// with a residual takes 136 to 149 us forward (5.4 to 5.9 TB/s) and 156 to 164 backward
// (5 TB/s), where a large copy reaches 4.8.
#include <type_traits>

#include "norm.h"

namespace tg {
namespace {

// The compiler does not know from here on what the bits became before.
__device__ inline void forget(i32x4 &bits) { asm volatile("" : "+v"(bits)); }

// dx, and a row of sums for dweight and dbias from each block; one block alone writes
// dweight and dbias themselves.  T threads have a row; with T = 64 a block has kRows of
// them at a time, else one.  A row stays in 16-byte units as it was read, converted in
// both passes over it, so that there is room for the next row, on its way meanwhile
// (kAhead); the sums of a thread's columns stay in registers over all rows.
template <typename E, int T, int N, int kRows, bool kAhead>
__global__ __launch_bounds__(T *kRows) void layer_norm_grad_kernel(GradArgs a, E *dweight, E *dbias) {  // NULL: sums to a.partial
    constexpr int kUnit = kUnitOf<E>;
    // 768 threads have no registers left for it: 3001 x 12289 in f16 takes 90 us, so 104
    constexpr bool kOneLoad = T < 768;
    using unit = vec<float, kUnit>;
    static_assert(T == 64 || kRows == 1, "rows that meet at barriers have a block of their own");
    __shared__ unit sums[2][T == 64 ? N * 64 : 1];
    __shared__ Two pairs[2][T / 64];
    const int t = threadIdx.x % T, units = (a.cols + kUnit - 1) / kUnit;
    i32x4 weight[N];
    unit dw[N], db[N];
    const auto valid = [&](int n) { return t + n * T < units ? left_of(a.cols, (t + n * T) * kUnit) : 0; };
#pragma unroll
    for (int n = 0; n < N; ++n) {
        weight[n] = load_bits<E>((const E *)a.weight + (t + n * T) * kUnit, valid(n));
        dw[n] = db[n] = unit(0.0f);
    }
    struct Row {
        i32x4 g[N], h[N], more[N];
        float mean, rstd;
    };
    const auto fetch = [&](Row &r, int64_t row) {
        const E *const dy = (const E *)a.dy + row * a.lddy, *const hidden = (const E *)a.hidden + row * a.ldh;
        const E *const dh = a.dhidden ? (const E *)a.dhidden + row * a.lddh : nullptr;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int col = (t + n * T) * kUnit, left = valid(n);
            const auto load = [&](const E *p) { return kOneLoad ? load_unit<E>(p, col, left) : load_bits<E>(p + col, left); };
            r.g[n] = load(dy);
            r.h[n] = load(hidden);
            r.more[n] = dh ? load(dh) : i32x4(0);
        }
        r.mean = a.mean[row], r.rstd = a.rstd[row];
    };
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / T;
    Row now;
    if (kAhead && row < a.rows) fetch(now, row);
    for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
        Row next;
        if (!kAhead)
            fetch(now, row);
        else if (row + step < a.rows)
            fetch(next, row + step);
        Two two{0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int col = (t + n * T) * kUnit, left = valid(n);
            if constexpr (kOneLoad) in_place<E>(now.g[n], col, left), in_place<E>(now.h[n], col, left), in_place<E>(now.more[n], col, left);
            // past the row's end g is 0, and mean rstd may be an infinity
            const auto add = [&](auto whole) {
                const unit g = floats<E>(now.g[n]), h = floats<E>(now.h[n]), w = floats<E>(weight[n]);
#pragma unroll
                for (int e = 0; e < kUnit; ++e) {
                    const float xhat = whole || e < left ? (h[e] - now.mean) * now.rstd : 0.0f, gw = g[e] * w[e];
                    dw[n][e] = fmaf(g[e], xhat, dw[n][e]);
                    db[n][e] += g[e];
                    two.a += gw;
                    two.b = fmaf(gw, xhat, two.b);
                }
            };
            if (left >= kUnit)
                add(std::true_type{});
            else if (left > 0)
                add(std::false_type{});
            forget(now.g[n]), forget(now.h[n]), forget(weight[n]);
            __builtin_amdgcn_sched_barrier(0);  // a unit's floats at a time
        }
        // the pairs of the row before last are free: a barrier lies between
        two = block_sums<T>(two, pairs[turn]);
        const float lift = two.a * a.inv_cols, mean = two.b * a.inv_cols;
        E *const dx = (E *)a.dx + row * a.lddx;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int left = valid(n);
            if (left <= 0) continue;
            const unit g = floats<E>(now.g[n]), h = floats<E>(now.h[n]), w = floats<E>(weight[n]), more = floats<E>(now.more[n]);
            unit d;
#pragma unroll
            for (int e = 0; e < kUnit; ++e) {
                const float xhat = (h[e] - now.mean) * now.rstd;
                d[e] = fmaf(now.rstd, fmaf(-xhat, mean, fmaf(g[e], w[e], -lift)), more[e]);
            }
            store_f32<E, kUnit>(dx + (t + n * T) * kUnit, d, left);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (kAhead) now = next;
    }
    if constexpr (T == 64) {  // the rows of a block, in order
        for (int r = 0; r < kRows; ++r) {
            if ((int)threadIdx.x / T == r) {
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    if (r) dw[n] = sums[0][n * 64 + t] + dw[n], db[n] = sums[1][n * 64 + t] + db[n];
                    sums[0][n * 64 + t] = dw[n], sums[1][n * 64 + t] = db[n];
                }
            }
            __syncthreads();
        }
        if ((int)threadIdx.x / T != kRows - 1) return;
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int64_t at = (int64_t)blockIdx.x * a.cols + (t + n * T) * kUnit;
        if (valid(n) <= 0) continue;
        if (dweight) {
            store_f32<E, kUnit>(dweight + at, dw[n], valid(n));
            if (dbias) store_f32<E, kUnit>(dbias + at, db[n], valid(n));
            continue;
        }
        store_f32<float, kUnit>(a.partial + at, dw[n], valid(n));
        if (a.partial2) store_f32<float, kUnit>(a.partial2 + at, db[n], valid(n));
    }
}

int64_t units_of(int64_t cols, int type) { return ceil_div(cols * (type == TG_F32 ? 4 : 2), 16); }
constexpr int64_t kMostUnits = 2048;  // of a row that stays in registers

// A wave has a row, eight of them a block, where its units leave room in registers for
// the next row's: three a lane, of floats four.
bool wave_has_a_row(int64_t units, int type) { return units <= (type == TG_F32 ? 256 : 192); }

// Few rows are left to one block, which writes the gradients itself and takes less than
// the launch that adds up several (eight waves with a row each; 2 us a row of many).
bool one_block(int64_t rows, int64_t cols, int type) {
    const int64_t units = units_of(cols, type);
    return rows > 0 && (units <= 128 ? rows <= 64 : units <= kMostUnits && rows <= 2);
}

// Blocks of the gradient: but for a single one, each leaves a row of sums for the weight
// and one for the bias, and as many as run at once are enough.  In bf16 with 256, 512
// and 768 blocks: 16384 x 512 takes 18.3, 19.1 and 22 us, 16384 x 2048 96, 59 and 56,
// 8192 x 4096 68, 57 and 61, 8192 x 8192 110, 119 and 125, 8192 x 12288 158, 158 (256
// run at once) and 185.
int layer_grad_blocks(int64_t rows, int64_t cols, int type) {
    const int64_t units = units_of(cols, type);
    if (one_block(rows, cols, type)) return 1;
    const bool waves = wave_has_a_row(units, type);
    return (int)std::min<int64_t>(waves ? ceil_div(rows, 8) : rows, waves ? 256 : units <= 256 ? 768 : units <= 512 || units > kMostUnits ? 512 : 256);
}

template <typename E>
hipError_t launch_layer_grad(GradArgs a, int blocks, void *dweight, void *dbias, hipStream_t s) {
    const int units = (a.cols + kUnitOf<E> - 1) / kUnitOf<E>;
    const auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, s, a, (E *)dweight, (E *)dbias); };
    // 16384 x 512 in bf16 takes 18 us, where blocks of one wave took 47; 16384 x 1304 42
    // and 50 by 256 threads a row, 16384 x 2048 58 and 103 by a wave, whose registers do
    // not hold four units and the next; 16384 x 520 of floats 33 and 40.  Longer rows
    // get threads for two units, in steps of 256, so that few have none: 8192 x 12288
    // takes 162 us by 768 threads and 213 by 1024 (without the row ahead).
    if (units <= 64)
        go(layer_norm_grad_kernel<E, 64, 1, 8, true>, 512);
    else if (units <= 128)
        go(layer_norm_grad_kernel<E, 64, 2, 8, true>, 512);
    else if (units <= 192)
        go(layer_norm_grad_kernel<E, 64, 3, 8, true>, 512);
    else if (units <= 256) {
        if constexpr (sizeof(E) == 4)
            go(layer_norm_grad_kernel<E, 64, 4, 8, true>, 512);
        else
            go(layer_norm_grad_kernel<E, 256, 1, 1, true>, 256);
    } else if (units <= 512)
        go(layer_norm_grad_kernel<E, 256, 2, 1, true>, 256);
    else if (units <= 1024)
        go(layer_norm_grad_kernel<E, 512, 2, 1, true>, 512);
    else if (units <= 1536)
        go(layer_norm_grad_kernel<E, 768, 2, 1, true>, 768);
    else if (units <= kMostUnits)
        go(layer_norm_grad_kernel<E, 1024, 2, 1, false>, 1024);
    else
        launch_grad_stream<E, true>(a, blocks, s);
    return hipGetLastError();
}

}  // namespace
}  // namespace tg

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
    if (one_block(q->rows, q->cols, q->type)) return 0;
    return round256((size_t)layer_grad_blocks(q->rows, q->cols, q->type) * q->cols * (q->dbias ? 8 : 4));
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
        if (need && (ws_bytes < need || !d_ws)) return call_failed(TG_ENOMEM, "workspace of %zu bytes, %zu needed", d_ws ? ws_bytes : 0, need);
        const bool one = q->rows == 1;
        float *const sums = (float *)d_ws;
        const int blocks = layer_grad_blocks(q->rows, q->cols, q->type);
        const bool alone = one_block(q->rows, q->cols, q->type);
        void *const dweight = alone ? q->dweight : nullptr, *const dbias = alone ? q->dbias : nullptr;
        GradArgs a{q->dy, q->dhidden, q->hidden, q->weight, q->mean, q->rstd, q->dx, sums,
                   q->dbias ? sums + (int64_t)blocks * q->cols : nullptr, q->rows,
                   one ? 0 : q->lddy, one ? 0 : q->lddh, one ? 0 : q->ldh, one ? 0 : q->lddx,
                   0, (int)q->cols, (float)(1.0 / (double)q->cols)};
        e = q->type == TG_F32    ? launch_layer_grad<float>(a, blocks, dweight, dbias, s)
            : q->type == TG_BF16 ? launch_layer_grad<bf16>(a, blocks, dweight, dbias, s)
                                 : launch_layer_grad<f16>(a, blocks, dweight, dbias, s);
        if (e != hipSuccess) return device_failed(e, "norm_grad_kernel");
        if (alone) return TG_OK;
    }
    e = launch_column_sums_of_two((const float *)d_ws, layer_grad_blocks(q->rows, q->cols, q->type), q->cols, q->dweight, q->dbias, q->type, s);
    return e == hipSuccess ? TG_OK : device_failed(e, "column_sums");
}

}  // extern "C"
