// rms_norm.hip -- root-mean-square norm with the residual's addition
// (tg_rms_norm) and its gradient (tg_rms_norm_grad).
//
// Both are bound by memory: forward reads x and residual and writes hidden and
// y, backward reads dy, hidden and dhidden and writes dx, each once, so a row
// stays in registers between its statistic and its output.  A row is cut into
// units of 16 bytes; thread t of the row's T threads holds units t, t + T, ...
// (N of them), every load of the row in flight before the reduction.  8192 x 8192
// in bf16 takes 89 us forward (6.0 TB/s), as much with 8 bits out, and 117
// backward (4.6 TB/s), where a large copy reaches 4.8 to 4.9; forward with 256
// threads a row took 96, backward with 768 or 1024 blocks 24 and 11 more in all,
// with the next row fetched ahead the same.  The gradient of short rows is bound
// by latency instead: its 512 blocks have a wave each up to 64 units a row, and
// 16384 x 512 in bf16 takes 47 us, 1.4 TB/s.
//
// hidden is h rounded once to the inputs' type, which is what the next operator
// and the gradient read; y is of the h before that rounding.  In 16 bits with a
// residual the gradients so carry the error of one rounding beside their own.
#include <algorithm>
#include <cmath>

#include "layer_device.h"

namespace tg {
namespace {

template <typename E>
constexpr int kUnitOf = 16 / sizeof(E);

constexpr float kLeastScale = 0x1p-126f;  // of an 8-bit output: the least normal number

struct NormArgs {
    const void *x, *residual, *weight;
    void *hidden, *y;
    float *scale, *rstd;
    int64_t rows, ldx, ldr, ldh, ldy;
    int64_t first;  // row of block 0
    int cols;
    float eps, inv_cols;
};

__device__ inline int left_of(int cols, int col) { return cols - col; }  // <= 0: none

template <int kUnit>
__device__ inline void store_e4m3(unsigned char *p, vec<float, kUnit> q, int valid) {
    vec<unsigned, kUnit / 4> w;
#pragma unroll
    for (int h = 0; h < kUnit / 4; ++h) {
        int t = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h], q[4 * h + 1], 0, false);
        w[h] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h + 2], q[4 * h + 3], t, true);
    }
    if (valid >= kUnit) {
        reinterpret_cast<Loose<vec<unsigned, kUnit / 4>, 1> *>(p)->v = w;
    } else {
#pragma unroll
        for (int e = 0; e < kUnit; ++e)
            if (e < valid) p[e] = (unsigned char)(w[e / 4] >> (8 * (e % 4)));
    }
}

// One row per T threads, N units a thread (T N units or fewer), 256 / T rows a block
// where T is 64.  kStream: rows of any length, read again for each pass (x and
// residual add up to the same h every time), one row a block.
template <typename E, bool kEight, int T, int N, bool kStream>
__global__ __launch_bounds__(T == 64 ? 256 : T) void norm_kernel(NormArgs a) {
    constexpr int kUnit = kUnitOf<E>;
    using unit = vec<float, kUnit>;
    constexpr int kRows = T == 64 ? 4 : 1;
    __shared__ float slots[2][T / 64];
    const int t = threadIdx.x % T;
    const int64_t row = a.first + (int64_t)blockIdx.x * kRows + threadIdx.x / T;
    if (kRows > 1 && row >= a.rows) return;  // whole waves, which meet no barrier
    const E *const x = (const E *)a.x + row * a.ldx;
    const E *const r = a.residual ? (const E *)a.residual + row * a.ldr : nullptr;
    E *const hidden = a.hidden ? (E *)a.hidden + row * a.ldh : nullptr;
    const E *const weight = (const E *)a.weight;

    const auto read = [&](int col) {
        const int valid = left_of(a.cols, col);
        unit h = load_f32<E, kUnit>(x + col, valid);
        if (r) h += load_f32<E, kUnit>(r + col, valid);
        return h;
    };
    const auto write = [&](int col, unit y, float scale) {
        const int valid = left_of(a.cols, col);
        if (kEight) {
#pragma unroll
            for (int e = 0; e < kUnit; ++e) y[e] /= scale;
            store_e4m3<kUnit>((unsigned char *)a.y + row * a.ldy + col, y, valid);
        } else {
            store_f32<E, kUnit>((E *)a.y + row * a.ldy + col, y, valid);
        }
    };

    unit h[N];
    float squares = 0.0f;
    const int units = (a.cols + kUnit - 1) / kUnit;
    if (kStream) {
        for (int u = t; u < units; u += T) {
            h[0] = read(u * kUnit);
#pragma unroll
            for (int e = 0; e < kUnit; ++e) squares = fmaf(h[0][e], h[0][e], squares);
        }
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) h[n] = t + n * T < units ? read((t + n * T) * kUnit) : unit(0.0f);
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int e = 0; e < kUnit; ++e) squares = fmaf(h[n][e], h[n][e], squares);
        }
    }
    squares = block_reduce<OpSum, T>(squares, slots[0]);
    const float rstd = 1.0f / sqrtf(fmaf(squares, a.inv_cols, a.eps));
    if (a.rstd && t == 0) a.rstd[row] = rstd;

    const auto normed = [&](unit v, int col) {
        const unit w = load_f32<E, kUnit>(weight + col, left_of(a.cols, col));
        unit y;
#pragma unroll
        for (int e = 0; e < kUnit; ++e) y[e] = (v[e] * rstd) * w[e];
        return y;
    };
    float scale = 1.0f;
    if (kEight) {
        float most = 0.0f;
        if (kStream) {
            for (int u = t; u < units; u += T) {
                const unit y = normed(read(u * kUnit), u * kUnit);
#pragma unroll
                for (int e = 0; e < kUnit; ++e) most = fmaxf(most, finite_abs(y[e]));
            }
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int u = t + n * T;
                if (u >= units) continue;
                if (hidden) store_f32<E, kUnit>(hidden + u * kUnit, h[n], left_of(a.cols, u * kUnit));
                h[n] = normed(h[n], u * kUnit);
#pragma unroll
                for (int e = 0; e < kUnit; ++e) most = fmaxf(most, finite_abs(h[n][e]));
            }
        }
        most = block_reduce<OpMax, T>(most, slots[1]);
        // a subnormal scale has few bits, and a row's largest over it could pass 448
        scale = most > 0.0f ? fmaxf(most / kE4M3Max, kLeastScale) : 1.0f;
        if (t == 0) a.scale[row] = scale;
    }
    if (kStream) {
        for (int u = t; u < units; u += T) {
            const unit v = read(u * kUnit);
            // hidden may be x or residual: this unit was just read for the last time
            if (hidden) store_f32<E, kUnit>(hidden + u * kUnit, v, left_of(a.cols, u * kUnit));
            write(u * kUnit, normed(v, u * kUnit), scale);
        }
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int u = t + n * T;
            if (u >= units) continue;
            if (!kEight && hidden) store_f32<E, kUnit>(hidden + u * kUnit, h[n], left_of(a.cols, u * kUnit));
            write(u * kUnit, kEight ? h[n] : normed(h[n], u * kUnit), scale);
        }
    }
}

struct GradArgs {
    const void *dy, *dhidden, *hidden, *weight;
    const float *rstd;
    void *dx;
    float *partial;  // [gridDim.x, cols] sums of dy h rstd
    int64_t rows, lddy, lddh, ldh, lddx;
    int64_t first;  // of block 0: its unit of columns (norm_grad_weight_stream), its row (norm_grad_stream)
    int cols;
    float inv_cols;
};

// A block takes rows blockIdx.x, + gridDim.x, ... and keeps its columns' share of
// dweight in registers over all of them; one row of sums a block leaves it.  The
// weight stays in registers too, except in blocks of 1024, whose threads have 128.
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

// Rows too long for registers: dweight's sums first, while dy is whole (dx may
// be dy), a thread a unit of columns and a block a share of the rows ...
template <typename E>
__global__ __launch_bounds__(256) void norm_grad_weight_stream(GradArgs a) {
    constexpr int kUnit = kUnitOf<E>;
    using unit = vec<float, kUnit>;
    const int64_t u = a.first + (int64_t)blockIdx.y * 256 + threadIdx.x;
    if (u * kUnit >= a.cols) return;
    const int col = (int)u * kUnit, valid = left_of(a.cols, col);
    unit dw(0.0f);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const unit g = load_f32<E, kUnit>((const E *)a.dy + row * a.lddy + col, valid);
        const unit h = load_f32<E, kUnit>((const E *)a.hidden + row * a.ldh + col, valid);
        const float rstd = a.rstd[row];
#pragma unroll
        for (int e = 0; e < kUnit; ++e) dw[e] = fmaf(g[e], h[e] * rstd, dw[e]);
    }
    store_f32<float, kUnit>(a.partial + (int64_t)blockIdx.x * a.cols + col, dw, valid);
}
// ... then dx, a row a block, read twice.
template <typename E>
__global__ __launch_bounds__(1024) void norm_grad_stream(GradArgs a) {
    constexpr int kUnit = kUnitOf<E>;
    using unit = vec<float, kUnit>;
    __shared__ float slots[16];
    const int64_t row = a.first + blockIdx.x;
    const int units = (a.cols + kUnit - 1) / kUnit;
    const E *const dy = (const E *)a.dy + row * a.lddy;
    const E *const hidden = (const E *)a.hidden + row * a.ldh;
    const E *const dh = a.dhidden ? (const E *)a.dhidden + row * a.lddh : nullptr;
    E *const dx = (E *)a.dx + row * a.lddx;
    const float rstd = a.rstd[row];
    float dot = 0.0f;
    for (int u = threadIdx.x; u < units; u += 1024) {
        const int col = u * kUnit, valid = left_of(a.cols, col);
        const unit g = load_f32<E, kUnit>(dy + col, valid), h = load_f32<E, kUnit>(hidden + col, valid);
        const unit w = load_f32<E, kUnit>((const E *)a.weight + col, valid);
#pragma unroll
        for (int e = 0; e < kUnit; ++e) dot = fmaf(g[e] * w[e], h[e] * rstd, dot);
    }
    const float mean = block_reduce<OpSum, 1024>(dot, slots) * a.inv_cols;
    for (int u = threadIdx.x; u < units; u += 1024) {
        const int col = u * kUnit, valid = left_of(a.cols, col);
        const unit g = load_f32<E, kUnit>(dy + col, valid), h = load_f32<E, kUnit>(hidden + col, valid);
        const unit w = load_f32<E, kUnit>((const E *)a.weight + col, valid);
        unit d(0.0f);
        if (dh) d = load_f32<E, kUnit>(dh + col, valid);
#pragma unroll
        for (int e = 0; e < kUnit; ++e) d[e] = fmaf(rstd, fmaf(-(h[e] * rstd), mean, g[e] * w[e]), d[e]);
        store_f32<E, kUnit>(dx + col, d, valid);
    }
}

constexpr int64_t kMostBlocks = 1 << 20;  // of a launch: a grid holds fewer than 2^32 threads

template <typename E, bool kEight>
hipError_t launch_norm(NormArgs a, hipStream_t s) {
    const int units = (a.cols + kUnitOf<E> - 1) / kUnitOf<E>;
    const auto go = [&](auto kernel, int threads, int rows_per_block) {
        for (a.first = 0; a.first < a.rows; a.first += kMostBlocks * rows_per_block) {
            const int64_t blocks = std::min(kMostBlocks, ceil_div(a.rows - a.first, rows_per_block));
            hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, s, a);
        }
    };
    // A wave a row while a row is at most two units a lane; beyond that 256 to
    // 1024 threads with one or two units each, and four only in rows of more than
    // 2048 units.  Few rows leave most of the chip idle whatever is done, so
    // they take more threads a row.
    if (units <= 64)
        go(norm_kernel<E, kEight, 64, 1, false>, 256, 4);
    else if (units <= 128)
        go(norm_kernel<E, kEight, 64, 2, false>, 256, 4);
    else if (units <= 256)
        go(norm_kernel<E, kEight, 256, 1, false>, 256, 1);
    else if (units <= 512 && a.rows >= 256)
        go(norm_kernel<E, kEight, 256, 2, false>, 256, 1);
    else if (units <= 1024 && a.rows >= 256)
        go(norm_kernel<E, kEight, 512, 2, false>, 512, 1);
    else if (units <= 1024)
        go(norm_kernel<E, kEight, 1024, 1, false>, 1024, 1);
    else if (units <= 2048)
        go(norm_kernel<E, kEight, 1024, 2, false>, 1024, 1);
    else if (units <= 4096)
        go(norm_kernel<E, kEight, 1024, 4, false>, 1024, 1);
    else
        go(norm_kernel<E, kEight, 1024, 1, true>, 1024, 1);
    return hipGetLastError();
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
        constexpr int64_t kMostUnits = 1 << 20;  // of a launch: 2^12 blocks across the columns by 512 down the rows
        for (; a.first < units; a.first += kMostUnits) {
            const dim3 blocks(grid.x, (unsigned)ceil_div(std::min(kMostUnits, units - a.first), 256));
            hipLaunchKernelGGL(norm_grad_weight_stream<E>, blocks, dim3(256), 0, s, a);
        }
        for (a.first = 0; a.first < a.rows; a.first += kMostBlocks)
            hipLaunchKernelGGL(norm_grad_stream<E>, dim3((unsigned)std::min(kMostBlocks, a.rows - a.first)), dim3(1024), 0, s, a);
    }
    return hipGetLastError();
}

size_t size_of(int type) { return type == TG_F32 ? 4 : type == TG_E4M3 ? 1 : 2; }
bool norm_type(int type) { return type == TG_F32 || type == TG_BF16 || type == TG_F16; }

tg_status check_rows(const void *p, int64_t ld, int64_t rows, int64_t cols, int type, const char *what) {
    if (!p) return call_failed(TG_EINVAL, "%s is NULL", what);
    if ((uintptr_t)p % size_of(type)) return call_failed(TG_EINVAL, "%s is not aligned to its elements", what);
    if (rows > 1 && ld < cols) return call_failed(TG_EINVAL, "%s: row stride %lld below the row length %lld", what, (long long)ld, (long long)cols);
    return TG_OK;
}

tg_status check_sizes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || rows > 0x7fffffff || cols > 0x7fffffff - 64)
        return call_failed(TG_EINVAL, "rows %lld, cols %lld", (long long)rows, (long long)cols);
    return TG_OK;
}

}  // namespace
}  // namespace tg

using namespace tg;

#define TG_TRY(call)                  \
    do {                              \
        const tg_status st_ = (call); \
        if (st_ != TG_OK) return st_; \
    } while (0)

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
    NormArgs a{q->x, q->residual, q->weight, q->hidden, q->y, q->scale, q->rstd, q->rows,
               one ? 0 : q->ldx, one ? 0 : q->ldr, one ? 0 : q->ldh, one ? 0 : q->ldy,
               0, (int)q->cols, q->eps, q->cols ? (float)(1.0 / (double)q->cols) : 0.0f};
    const hipStream_t s = (hipStream_t)stream;
    const bool eight = q->out_type == TG_E4M3;
    hipError_t e;
    if (q->type == TG_F32)
        e = eight ? launch_norm<float, true>(a, s) : launch_norm<float, false>(a, s);
    else if (q->type == TG_BF16)
        e = eight ? launch_norm<bf16, true>(a, s) : launch_norm<bf16, false>(a, s);
    else
        e = eight ? launch_norm<f16, true>(a, s) : launch_norm<f16, false>(a, s);
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
        GradArgs a{q->dy, q->dhidden, q->hidden, q->weight, q->rstd, q->dx, (float *)d_ws, q->rows,
                   one ? 0 : q->lddy, one ? 0 : q->lddh, one ? 0 : q->ldh, one ? 0 : q->lddx,
                   0, (int)q->cols, (float)(1.0 / (double)q->cols)};
        e = q->type == TG_F32 ? launch_grad<float>(a, s) : q->type == TG_BF16 ? launch_grad<bf16>(a, s) : launch_grad<f16>(a, s);
        if (e != hipSuccess) return device_failed(e, "norm_grad_kernel");
    }
    e = launch_column_sums((const float *)d_ws, grad_blocks(q->rows), q->cols, q->dweight, q->type, s);
    return e == hipSuccess ? TG_OK : device_failed(e, "column_sums");
}

}  // extern "C"
