// norm.h -- norms over rows with the residual's addition, and their gradients: the
// kernels of rms_norm.hip (kCentre false) and layer_norm.hip (kCentre true).
//
// Both are bound by memory: forward reads x and residual and writes hidden and
// y, backward reads dy, hidden and dhidden and writes dx, each once, so a row
// stays in registers between its statistic and its output.  A row is cut into
// units of 16 bytes; thread t of the row's T threads holds units t, t + T, ...
// (N of them), every load of the row in flight before the reduction.  8192 x 8192
// in bf16 takes 89 us forward (6.0 TB/s), as much with 8 bits out, and 117
// backward (4.6 TB/s), where a large copy reaches 4.8 to 4.9; forward with 256
// threads a row took 96.
//
// hidden is h rounded once to the inputs' type, which is what the next operator
// and the gradient read; y is of the h before that rounding.  In 16 bits with a
// residual the gradients so carry the error of one rounding beside their own.
#pragma once

#include <algorithm>
#include <cmath>

#include "layer_device.h"

namespace tg {
namespace {

struct NormArgs {
    const void *x, *residual, *weight, *bias;
    void *hidden, *y;
    float *scale, *mean, *rstd;
    int64_t rows, ldx, ldr, ldh, ldy;
    int64_t first;  // row of block 0
    int cols;
    float eps, inv_cols;
};

__device__ inline int left_of(int cols, int col) { return cols - col; }  // <= 0: none

// Both reductions at once, in the order of block_reduce.
struct Two {
    float a, b;
};
template <int T>
__device__ inline Two block_sums(Two x, Two *slots) {
    x.a = wave_reduce<OpSum>(x.a), x.b = wave_reduce<OpSum>(x.b);
    if (T == 64) return x;
    if (threadIdx.x % 64 == 0) slots[threadIdx.x / 64] = x;
    __syncthreads();
    x = slots[0];
#pragma unroll
    for (int w = 1; w < T / 64; ++w) x.a += slots[w].a, x.b += slots[w].b;
    return x;
}

// kCentre: the row's mean is taken off first, and the bias added at the end.  The
// second pass over the registers corrects the first one's mean by what is left of
// the row around it, so a row far from 0 keeps its deviations.
// One row per T threads, N units a thread (T N units or fewer), 256 / T rows a block
// where T is 64.  kStream: rows of any length, read again for each pass (x and
// residual add up to the same h every time), one row a block.
template <typename E, bool kEight, int T, int N, bool kStream, bool kCentre>
__global__ __launch_bounds__(T == 64 ? 256 : T) void norm_kernel(NormArgs a) {
    constexpr int kUnit = kUnitOf<E>;
    using unit = vec<float, kUnit>;
    constexpr int kRows = T == 64 ? 4 : 1;
    constexpr bool kOneLoad = kCentre && !kStream;
    __shared__ float slots[2][T / 64];
    __shared__ Two pairs[T / 64];
    const int t = threadIdx.x % T;
    const int64_t row = a.first + (int64_t)blockIdx.x * kRows + threadIdx.x / T;
    if (kRows > 1 && row >= a.rows) return;  // whole waves, which meet no barrier
    const E *const x = (const E *)a.x + row * a.ldx;
    const E *const r = a.residual ? (const E *)a.residual + row * a.ldr : nullptr;
    E *const hidden = a.hidden ? (E *)a.hidden + row * a.ldh : nullptr;
    const E *const weight = (const E *)a.weight, *const bias = (const E *)a.bias;

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
    const int units = (a.cols + kUnit - 1) / kUnit;
    // f(h, valid elements of it) over the thread's units
    const auto over = [&](auto f) {
        if (kStream) {
            for (int u = t; u < units; u += T) f(read(u * kUnit), left_of(a.cols, u * kUnit));
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) f(h[n], t + n * T < units ? left_of(a.cols, (t + n * T) * kUnit) : 0);
        }
    };
    if constexpr (kOneLoad) {
        i32x4 from[N], more[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int col = (t + n * T) * kUnit, left = t + n * T < units ? left_of(a.cols, col) : 0;
            from[n] = load_unit<E>(x, col, left);
            more[n] = r ? load_unit<E>(r, col, left) : i32x4(0);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int col = (t + n * T) * kUnit, left = t + n * T < units ? left_of(a.cols, col) : 0;
            in_place<E>(from[n], col, left), in_place<E>(more[n], col, left);
            h[n] = floats<E>(from[n]);
            if (r) h[n] += floats<E>(more[n]);
        }
    } else if (!kStream) {
#pragma unroll
        for (int n = 0; n < N; ++n) h[n] = t + n * T < units ? read((t + n * T) * kUnit) : unit(0.0f);
    }
    float squares = 0.0f, mean = 0.0f;
    if constexpr (kCentre) {
        float sum = 0.0f;
        over([&](unit v, int) {
#pragma unroll
            for (int e = 0; e < kUnit; ++e) sum += v[e];
        });
        mean = block_reduce<OpSum, T>(sum, slots[0]) * a.inv_cols;
        Two two{0.0f, 0.0f};
        over([&](unit v, int valid) {
#pragma unroll
            for (int e = 0; e < kUnit; ++e) {
                const float d = e < valid ? v[e] - mean : 0.0f;
                two.a += d, two.b = fmaf(d, d, two.b);
            }
        });
        two = block_sums<T>(two, pairs);
        const float off = two.a * a.inv_cols;
        squares = fmaxf(fmaf(-two.a, off, two.b), two.b * 0.0f);  // not below 0; NaN stays
        mean += off;
        if (a.mean && t == 0) a.mean[row] = mean;
    } else {
        over([&](unit v, int) {
#pragma unroll
            for (int e = 0; e < kUnit; ++e) squares = fmaf(v[e], v[e], squares);
        });
        squares = block_reduce<OpSum, T>(squares, slots[0]);
    }
    const float rstd = 1.0f / sqrtf(fmaf(squares, a.inv_cols, a.eps));
    if (a.rstd && t == 0) a.rstd[row] = rstd;

    const auto normed = [&](unit v, int col) {
        const int left = left_of(a.cols, col);
        unit w, b(0.0f), y;
        if constexpr (kOneLoad) {
            i32x4 from = load_unit<E>(weight, col, left), more = bias ? load_unit<E>(bias, col, left) : i32x4(0);
            in_place<E>(from, col, left), in_place<E>(more, col, left);
            w = floats<E>(from), b = floats<E>(more);
        } else {
            w = load_f32<E, kUnit>(weight + col, left);
            if (kCentre && bias) b = load_f32<E, kUnit>(bias + col, left);
        }
        if constexpr (kCentre) {
#pragma unroll
            for (int e = 0; e < kUnit; ++e) y[e] = fmaf((v[e] - mean) * rstd, w[e], b[e]);
        } else {
#pragma unroll
            for (int e = 0; e < kUnit; ++e) y[e] = (v[e] * rstd) * w[e];
        }
        return y;
    };
    float scale = 1.0f;
    if (kEight) {
        float most = 0.0f;
        if (kStream) {
            for (int u = t; u < units; u += T) {
                const unit y = normed(read(u * kUnit), u * kUnit);
#pragma unroll
                for (int e = 0; e < kUnit; ++e) most = fmaxf(most, finite_abs(y[e]));  // past the row's end weight and bias are 0
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
    const float *mean, *rstd;
    void *dx;
    float *partial;   // [gridDim.x, cols] sums of dy h rstd
    float *partial2;  // those of dy, or NULL
    int64_t rows, lddy, lddh, ldh, lddx;
    int64_t first;  // of block 0: its unit of columns (norm_grad_weight_stream), its row (norm_grad_stream)
    int cols;
    float inv_cols;
};

// Rows too long for registers: dweight's sums first, while dy is whole (dx may
// be dy), a thread a unit of columns and a block a share of the rows ...
template <typename E, bool kCentre>
__global__ __launch_bounds__(256) void norm_grad_weight_stream(GradArgs a) {
    constexpr int kUnit = kUnitOf<E>;
    using unit = vec<float, kUnit>;
    const int64_t u = a.first + (int64_t)blockIdx.y * 256 + threadIdx.x;
    if (u * kUnit >= a.cols) return;
    const int col = (int)u * kUnit, valid = left_of(a.cols, col);
    unit dw(0.0f), db(0.0f);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const unit g = load_f32<E, kUnit>((const E *)a.dy + row * a.lddy + col, valid);
        const unit h = load_f32<E, kUnit>((const E *)a.hidden + row * a.ldh + col, valid);
        const float rstd = a.rstd[row], centre = kCentre ? a.mean[row] : 0.0f;
#pragma unroll
        for (int e = 0; e < kUnit; ++e) dw[e] = fmaf(g[e], (kCentre ? h[e] - centre : h[e]) * rstd, dw[e]);
        if (kCentre) db += g;
    }
    store_f32<float, kUnit>(a.partial + (int64_t)blockIdx.x * a.cols + col, dw, valid);
    if (kCentre && a.partial2) store_f32<float, kUnit>(a.partial2 + (int64_t)blockIdx.x * a.cols + col, db, valid);
}
// ... then dx, a row a block, read twice.
template <typename E, bool kCentre>
__global__ __launch_bounds__(1024) void norm_grad_stream(GradArgs a) {
    constexpr int kUnit = kUnitOf<E>;
    using unit = vec<float, kUnit>;
    __shared__ float slots[16];
    __shared__ Two pairs[16];
    const int64_t row = a.first + blockIdx.x;
    const int units = (a.cols + kUnit - 1) / kUnit;
    const E *const dy = (const E *)a.dy + row * a.lddy;
    const E *const hidden = (const E *)a.hidden + row * a.ldh;
    const E *const dh = a.dhidden ? (const E *)a.dhidden + row * a.lddh : nullptr;
    E *const dx = (E *)a.dx + row * a.lddx;
    const float rstd = a.rstd[row], centre = kCentre ? a.mean[row] : 0.0f;
    float dot = 0.0f, sum = 0.0f;
    for (int u = threadIdx.x; u < units; u += 1024) {
        const int col = u * kUnit, valid = left_of(a.cols, col);
        const unit g = load_f32<E, kUnit>(dy + col, valid), h = load_f32<E, kUnit>(hidden + col, valid);
        const unit w = load_f32<E, kUnit>((const E *)a.weight + col, valid);
#pragma unroll
        for (int e = 0; e < kUnit; ++e) {
            // past the row's end g is 0 and centre rstd may be an infinity
            dot = fmaf(g[e] * w[e], kCentre ? (e < valid ? (h[e] - centre) * rstd : 0.0f) : h[e] * rstd, dot);
            if (kCentre) sum = fmaf(g[e], w[e], sum);
        }
    }
    float mean, lift = 0.0f;
    if constexpr (kCentre) {
        const Two two = block_sums<1024>(Two{dot, sum}, pairs);
        mean = two.a * a.inv_cols, lift = two.b * a.inv_cols;
    } else {
        mean = block_reduce<OpSum, 1024>(dot, slots) * a.inv_cols;
    }
    for (int u = threadIdx.x; u < units; u += 1024) {
        const int col = u * kUnit, valid = left_of(a.cols, col);
        const unit g = load_f32<E, kUnit>(dy + col, valid), h = load_f32<E, kUnit>(hidden + col, valid);
        const unit w = load_f32<E, kUnit>((const E *)a.weight + col, valid);
        unit d(0.0f);
        if (dh) d = load_f32<E, kUnit>(dh + col, valid);
#pragma unroll
        for (int e = 0; e < kUnit; ++e) {
            const float xhat = (kCentre ? h[e] - centre : h[e]) * rstd;
            d[e] = fmaf(rstd, fmaf(-xhat, mean, kCentre ? g[e] * w[e] - lift : g[e] * w[e]), d[e]);
        }
        store_f32<E, kUnit>(dx + col, d, valid);
    }
}

constexpr int64_t kMostBlocks = 1 << 20;  // of a launch: a grid holds fewer than 2^32 threads

template <typename E, bool kEight, bool kCentre>
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
        go(norm_kernel<E, kEight, 64, 1, false, kCentre>, 256, 4);
    else if (units <= 128)
        go(norm_kernel<E, kEight, 64, 2, false, kCentre>, 256, 4);
    else if (units <= 256)
        go(norm_kernel<E, kEight, 256, 1, false, kCentre>, 256, 1);
    else if (units <= 512 && a.rows >= 256)
        go(norm_kernel<E, kEight, 256, 2, false, kCentre>, 256, 1);
    else if (units <= 1024 && a.rows >= 256)
        go(norm_kernel<E, kEight, 512, 2, false, kCentre>, 512, 1);
    else if (units <= 1024)
        go(norm_kernel<E, kEight, 1024, 1, false, kCentre>, 1024, 1);
    else if (kCentre && units <= 1536 && a.rows >= 256 && sizeof(E) == 2)  // 8192 x 12288: 149 us, by 768 threads 152
        go(norm_kernel<E, kEight, 512, 3, false, kCentre>, 512, 1);
    else if (kCentre && units <= 1536)  // 8192 x 6000 of floats: 144 us, by 512 threads 153
        go(norm_kernel<E, kEight, 768, 2, false, kCentre>, 768, 1);
    else if (units <= 2048)
        go(norm_kernel<E, kEight, 1024, 2, false, kCentre>, 1024, 1);
    else if (units <= 4096)
        go(norm_kernel<E, kEight, 1024, 4, false, kCentre>, 1024, 1);
    else
        go(norm_kernel<E, kEight, 1024, 1, true, kCentre>, 1024, 1);
    return hipGetLastError();
}

// Rows too long for registers: `blocks` down the rows leave a row of sums each.
template <typename E, bool kCentre>
void launch_grad_stream(GradArgs a, int blocks, hipStream_t s) {
    const int units = (a.cols + kUnitOf<E> - 1) / kUnitOf<E>;
    constexpr int64_t kMostUnits = 1 << 20;  // of a launch: 2^12 blocks across the columns by 512 down the rows
    for (; a.first < units; a.first += kMostUnits) {
        const dim3 grid(blocks, (unsigned)ceil_div(std::min(kMostUnits, units - a.first), 256));
        hipLaunchKernelGGL((norm_grad_weight_stream<E, kCentre>), grid, dim3(256), 0, s, a);
    }
    for (a.first = 0; a.first < a.rows; a.first += kMostBlocks)
        hipLaunchKernelGGL((norm_grad_stream<E, kCentre>), dim3((unsigned)std::min(kMostBlocks, a.rows - a.first)), dim3(1024), 0, s, a);
}

inline bool norm_type(int type) { return type == TG_F32 || type == TG_BF16 || type == TG_F16; }

inline tg_status check_rows(const void *p, int64_t ld, int64_t rows, int64_t cols, int type, const char *what) {
    if (!p) return call_failed(TG_EINVAL, "%s is NULL", what);
    if ((uintptr_t)p % size_of(type)) return call_failed(TG_EINVAL, "%s is not aligned to its elements", what);
    if (rows > 1 && ld < cols) return call_failed(TG_EINVAL, "%s: row stride %lld below the row length %lld", what, (long long)ld, (long long)cols);
    return TG_OK;
}

inline tg_status check_sizes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || rows > 0x7fffffff || cols > 0x7fffffff - 64)
        return call_failed(TG_EINVAL, "rows %lld, cols %lld", (long long)rows, (long long)cols);
    return TG_OK;
}

}  // namespace
}  // namespace tg
