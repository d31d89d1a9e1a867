// quantize.hip -- 8-bit values with a scale for every block of 128 columns of one
// row or of 128 rows (tg_quantize).
//
// Bound by memory: x is read once and stays in registers while its block's largest
// value is found.  8192 x 28672 in bf16 takes 121 to 128 us by rows (5.5 to 5.8 TB/s)
// and 131 by squares, where a large copy reaches 4.8.
#include <algorithm>

#include "layer_device.h"

namespace tg {
namespace {

constexpr int kBlock = 128;

struct QuantizeArgs {
    const void *x;
    unsigned char *y;
    void *scale;
    int64_t rows, ldx, ldy, lds;
    int64_t first;  // of block 0
    int cols;
    int across;  // blocks of threads (quantize_rows), blocks of values (quantize_squares) across the columns
    int lanes;   // quantize_rows: threads that share a row, a power of two
};

// A block's scale and what x is multiplied by first.
struct Scale {
    float scale, inverse;
    unsigned code;
};
template <bool kPowers>
__device__ inline Scale scale_of(float most) {
    Scale s;
    s.scale = most > 0.0f ? fmaxf(most / kE4M3Max, kLeastScale) : 1.0f;
    s.code = 0;
    if (kPowers) {
        const unsigned bits = __float_as_uint(s.scale);
        s.code = (bits >> 23) + ((bits & 0x7fffffu) != 0);
        s.scale = __uint_as_float(s.code << 23);
        s.inverse = __uint_as_float((254u - s.code) << 23);
    } else {
        s.inverse = 1.0f / s.scale;
    }
    return s;
}
// v / scale, rounded once: the quotient by the inverse, corrected by what is left of
// v.  (Where an infinity has no remainder, NaN.)
template <bool kPowers, int N>
__device__ inline vec<float, N> divided(vec<float, N> v, const Scale &s) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float q = v[e] * s.inverse;
        v[e] = kPowers ? q : fmaf(fmaf(-q, s.scale, v[e]), s.inverse, q);
    }
    return v;
}
template <bool kPowers>
__device__ inline void store_scale(void *row, int64_t b, const Scale &s) {
    if (kPowers)
        ((Global<unsigned char> *)row)[b] = (unsigned char)s.code;
    else
        ((Global<float> *)row)[b] = s.scale;
}

// The largest over 16 neighbouring lanes, or 32.
template <int kLanes>
__device__ inline float lanes_max(float x) {
    x = OpMax::of(x, moved<0xB1>(x));
    x = OpMax::of(x, moved<0x4E>(x));
    x = OpMax::of(x, moved<0x141>(x));
    x = OpMax::of(x, moved<0x140>(x));
    if (kLanes == 32) {
        const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = OpMax::of(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
    }
    return x;
}

// Blocks of one row: 16 lanes (32 of floats) have a block, a unit of 16 bytes each,
// and a thread N units, `lanes` apart.
template <typename E, bool kPowers, int N>
__global__ __launch_bounds__(256) void quantize_rows(QuantizeArgs a) {
    constexpr int kUnit = kUnitOf<E>, kLanes = kBlock / kUnit;
    const int64_t block = a.first + blockIdx.x;
    const int t = threadIdx.x & (a.lanes - 1);
    const int64_t row = block / a.across * (256 / a.lanes) + threadIdx.x / a.lanes;
    const int64_t unit0 = block % a.across * (int64_t)(N * a.lanes) + t;
    if (row >= a.rows) return;  // groups of lanes that have a block as a whole
    const E *const x = (const E *)a.x + row * a.ldx;
    unsigned char *const y = a.y + row * a.ldy;
    char *const scales = (char *)a.scale + row * a.lds * (kPowers ? 1 : 4);
    i32x4 from[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int64_t col = (unit0 + n * a.lanes) * kUnit;
        from[n] = col < a.cols ? load_unit<E>(x, (int)col, (int)(a.cols - col)) : i32x4(0);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int64_t col = (unit0 + n * a.lanes) * kUnit;
        if (col < a.cols) in_place<E>(from[n], (int)col, (int)(a.cols - col));
        const vec<float, kUnit> v = floats<E>(from[n]);
        float most = 0.0f;
#pragma unroll
        for (int e = 0; e < kUnit; ++e) most = fmaxf(most, finite_abs(v[e]));
        const Scale s = scale_of<kPowers>(lanes_max<kLanes>(most));
        if (col >= a.cols) continue;
        store_e4m3<kUnit>(y + col, divided<kPowers, kUnit>(v, s), (int)(a.cols - col));
        if (t % kLanes == 0) store_scale<kPowers>(scales, col / kBlock, s);
    }
}

// Blocks of 128 rows: a block of threads each.
template <typename E, bool kPowers>
__global__ __launch_bounds__(256) void quantize_squares(QuantizeArgs a) {
    constexpr int kUnit = kUnitOf<E>, kLanes = kBlock / kUnit, kRows = 256 / kLanes, kN = kBlock / kRows;
    __shared__ float slots[4];
    const int64_t block = a.first + blockIdx.x;
    const int64_t row0 = block / a.across * kBlock + threadIdx.x / kLanes;
    const int64_t b = block % a.across, col = b * kBlock + threadIdx.x % kLanes * kUnit;
    const int valid = (int)(a.cols - col);
    i32x4 from[kN];
    vec<float, kUnit> v[kN];
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        const int64_t row = row0 + n * kRows;
        from[n] = row < a.rows && valid > 0 ? load_unit<E>((const E *)a.x + row * a.ldx, (int)col, valid) : i32x4(0);
    }
    float most = 0.0f;
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        if (valid > 0) in_place<E>(from[n], (int)col, valid);
        v[n] = floats<E>(from[n]);
#pragma unroll
        for (int e = 0; e < kUnit; ++e) most = fmaxf(most, finite_abs(v[n][e]));
    }
    const Scale s = scale_of<kPowers>(block_reduce<OpMax, 256>(most, slots));
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        const int64_t row = row0 + n * kRows;
        if (row < a.rows && valid > 0) store_e4m3<kUnit>(a.y + row * a.ldy + col, divided<kPowers, kUnit>(v[n], s), valid);
    }
    if (threadIdx.x == 0) store_scale<kPowers>((char *)a.scale + block / a.across * a.lds * (kPowers ? 1 : 4), b, s);
}

constexpr int64_t kMostBlocks = 1 << 20;  // of a launch: a grid holds fewer than 2^32 threads

template <typename E, bool kPowers>
hipError_t launch_quantize(QuantizeArgs a, bool square, hipStream_t s) {
    const auto go = [&](auto kernel, int64_t blocks) {
        for (a.first = 0; a.first < blocks; a.first += kMostBlocks)
            hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(kMostBlocks, blocks - a.first)), dim3(256), 0, s, a);
    };
    if (square) {
        a.across = (int)ceil_div(a.cols, kBlock);
        go(quantize_squares<E, kPowers>, ceil_div(a.rows, kBlock) * a.across);
        return hipGetLastError();
    }
    const int64_t units = ceil_div(a.cols, kUnitOf<E>);
    for (a.lanes = kBlock / kUnitOf<E>; a.lanes < 256 && a.lanes < units;) a.lanes *= 2;
    const int64_t rows = ceil_div(a.rows, 256 / a.lanes);
    // Two units a thread (four of floats, which are half as long) where that leaves
    // 1024 blocks: 8192 x 28672 in bf16 takes 128 us with two, 137 with four and 147 with
    // one, 512 x 28672 10.6, 11.5 and 11.6, 8192^2 of floats 68, 66 and 77.
    constexpr int kMany = sizeof(E) == 4 ? 4 : 2;
    const int n = units >= kMany * a.lanes && rows * ceil_div(units, kMany * a.lanes) >= 1024 ? kMany : 1;
    a.across = (int)ceil_div(units, n * a.lanes);
    if (n == kMany)
        go(quantize_rows<E, kPowers, kMany>, rows * a.across);
    else
        go(quantize_rows<E, kPowers, 1>, rows * a.across);
    return hipGetLastError();
}

}  // namespace
}  // namespace tg

using namespace tg;

extern "C" tg_status tg_quantize(const tg_quantize_args *q, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    if (q->reserved) return call_failed(TG_EINVAL, "reserved must be 0");
    if (q->type != TG_F32 && q->type != TG_BF16 && q->type != TG_F16) return call_failed(TG_EINVAL, "type %d", q->type);
    if (q->scale_type != TG_F32 && q->scale_type != TG_E8M0) return call_failed(TG_EINVAL, "scale_type %d", q->scale_type);
    if (q->block_rows != 1 && q->block_rows != kBlock) return call_failed(TG_EINVAL, "block_rows %d, 1 or 128 expected", q->block_rows);
    if (q->rows < 0 || q->cols < 0 || q->rows > 0x7fffffff || q->cols > 0x7fffffff - kBlock)
        return call_failed(TG_EINVAL, "rows %lld, cols %lld", (long long)q->rows, (long long)q->cols);
    if (q->rows == 0 || q->cols == 0) return TG_OK;
    if (!q->x || !q->y || !q->scale) return call_failed(TG_EINVAL, "%s is NULL", !q->x ? "x" : !q->y ? "y" : "scale");
    if ((uintptr_t)q->x % (q->type == TG_F32 ? 4 : 2)) return call_failed(TG_EINVAL, "x is not aligned to its elements");
    if (q->scale_type == TG_F32 && (uintptr_t)q->scale % 4) return call_failed(TG_EINVAL, "scale is not aligned to its elements");
    const int64_t scale_rows = ceil_div(q->rows, q->block_rows), scale_cols = ceil_div(q->cols, kBlock);
    if (q->rows > 1 && (q->ldx < q->cols || q->ldy < q->cols))
        return call_failed(TG_EINVAL, "%s: row stride below the row length %lld", q->ldx < q->cols ? "x" : "y", (long long)q->cols);
    if (scale_rows > 1 && q->lds < scale_cols) return call_failed(TG_EINVAL, "scale: row stride below the row length %lld", (long long)scale_cols);
    QuantizeArgs a{};
    a.x = q->x, a.y = (unsigned char *)q->y, a.scale = q->scale, a.rows = q->rows, a.cols = (int)q->cols;
    a.ldx = q->rows > 1 ? q->ldx : 0, a.ldy = q->rows > 1 ? q->ldy : 0, a.lds = scale_rows > 1 ? q->lds : 0;
    const hipStream_t s = (hipStream_t)stream;
    const bool powers = q->scale_type == TG_E8M0, square = q->block_rows == kBlock;
    hipError_t e;
    if (q->type == TG_F32)
        e = powers ? launch_quantize<float, true>(a, square, s) : launch_quantize<float, false>(a, square, s);
    else if (q->type == TG_BF16)
        e = powers ? launch_quantize<bf16, true>(a, square, s) : launch_quantize<bf16, false>(a, square, s);
    else
        e = powers ? launch_quantize<f16, true>(a, square, s) : launch_quantize<f16, false>(a, square, s);
    return e == hipSuccess ? TG_OK : device_failed(e, "quantize");
}
