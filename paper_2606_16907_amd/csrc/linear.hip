// linear.hip -- matrix product with bias, activation and residual in its
// epilogue (tg_linear), and its gradients (tg_linear_grad).
//
// All three products are C[i][j] = sum over r of P(i, r) Q(j, r), written row by
// row:   y  = x w^T    P = x, Q = w, both with r along their rows
//        dx = dz w     P = dz,       Q = w with r down its columns
//        dw = dz^T x   P = dz and Q = x with r down their columns
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "layer_device.h"

namespace tg {
namespace {

// ---------------------------------------------------------------------------
// tiles of an operand in LDS and the fragments of the matrix instructions
// ---------------------------------------------------------------------------
// A tile holds kStepBytes of r for each of its rows (or columns).  With r along
// the rows ("along") it is [rows][128 bytes], and the 16-byte units of a row are
// permuted by the row, unit ^ (row & 7), so that the 16 rows of a fragment meet
// different banks.  With r down the columns ("down", 16-bit types) it is
// [64 r][columns], read through the transposing LDS load, and the 32-byte units
// of a row are permuted by the row's bits 0, 1 and 3, the ones in which the rows
// of one load differ.
constexpr int kStepBytes = 128;

__device__ inline int along_at(int row, int unit) { return row * kStepBytes + ((unit ^ (row & 7)) << 4); }
__device__ inline int down_bits(int r) { return (r & 3) | ((r >> 1) & 4); }

template <typename T>
struct Matrix;
template <>
struct Matrix<bf16> {
    static constexpr int kSub = 2;  // matrix instructions along a step's r
    using frag = vec<bf16, 8>;
    static __device__ f32x4 mma(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Matrix<f16> {
    static constexpr int kSub = 2;
    using frag = vec<f16, 8>;
    static __device__ f32x4 mma(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
// Lane l's part of rows row0 .. row0 + 15: 16 bytes of row l % 16.
// Which r a lane holds does not matter as long as P and Q agree.
template <typename T>
__device__ inline typename Matrix<T>::frag read_along(const char *tile, int row0, int sub) {
    const int lane = threadIdx.x % 64, row = row0 + lane % 16;
    return *(const typename Matrix<T>::frag *)(tile + along_at(row, sub * 4 + lane / 16));
}
// The same from a "down" tile of `width` columns: the transposing load hands each
// lane of 16 one column of the 4 x 16 block whose rows the lanes point at.
template <typename T>
__device__ inline typename Matrix<T>::frag read_down(const char *tile, int col0, int sub, int width) {
    using s16x4 = vec<short, 4>;
    const int lane = threadIdx.x % 64, r = sub * 32 + (lane / 16) * 8 + (lane % 16) / 4;
    s16x4 half[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = (r + 4 * h) * width * 2 + (((col0 / 16) ^ down_bits(r + 4 * h)) << 5) + (lane % 4) * 8;
        half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(tile + at));
    }
    using s16x8 = vec<short, 8>;
    return __builtin_bit_cast(typename Matrix<T>::frag, (s16x8)__builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
}
template <typename T, bool kDown>
__device__ inline typename Matrix<T>::frag read_frag(const char *tile, int at, int sub, int width) {
    if constexpr (kDown)
        return read_down<T>(tile, at, sub, width);
    else
        return read_along<T>(tile, at, sub);
}

// ---------------------------------------------------------------------------
// epilogue
// ---------------------------------------------------------------------------
struct Epilogue {
    const float *x_scale, *w_scale;
    const void *bias, *residual;
    void *out, *pre;
    int64_t ldr, ldo, ldp;
    int act;
};

__device__ inline float normal_cdf(float z) { return 0.5f * erfcf(z * -0.70710678f); }

__device__ inline float activate(float z, int act) {
    switch (act) {
        case TG_ACT_RELU: return z < 0.0f ? 0.0f : z;  // NaN stays
        case TG_ACT_SILU: return z / (1.0f + expf(-z));
        case TG_ACT_GELU: return z * normal_cdf(z);
        default: return z;
    }
}
__device__ inline float slope(float z, int act) {
    switch (act) {
        case TG_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
        case TG_ACT_SILU: {
            const float t = 1.0f / (1.0f + expf(-z));
            return t * fmaf(z, 1.0f - t, 1.0f);
        }
        case TG_ACT_GELU: return fmaf(z * 0.39894228f, expf(-0.5f * z * z), normal_cdf(z));
        default: return 1.0f;
    }
}

// Four columns j .. j + 3 of row i.
template <typename O>
__device__ inline void finish(f32x4 z, int64_t i, int64_t j, int valid, const Epilogue &e) {
    if (e.x_scale) {
        const float sx = e.x_scale[i];
        z *= sx;
        z *= load_f32<float, 4>(e.w_scale + j, valid);
    }
    if (e.bias) z += load_f32<O, 4>((const O *)e.bias + j, valid);
    if (e.pre) store_f32<O, 4>((O *)e.pre + i * e.ldp + j, z, valid);
    if (e.act != TG_ACT_NONE) {
#pragma unroll
        for (int c = 0; c < 4; ++c) z[c] = activate(z[c], e.act);
    }
    if (e.residual) z += load_f32<O, 4>((const O *)e.residual + i * e.ldr + j, valid);
    store_f32<O, 4>((O *)e.out + i * e.ldo + j, z, valid);
}

// ---------------------------------------------------------------------------
// the product for operands at any alignment
// ---------------------------------------------------------------------------
struct Product {
    const void *p, *q;
    int64_t ldp, ldq;     // elements
    int64_t ni, nj, nr;   // rows and columns of C, length of the sums
};

// Units of 8 elements: 16 bytes in the matrix instruction's type, read as 8 bytes
// where the operand is e4m3.  Those at or past `valid` are 0 and not read.
template <typename T>
struct Unit {
    using raw = vec<int, sizeof(T) * 2>;
    static __device__ raw load(const T *p, int64_t valid) {
        if (valid >= 8) return reinterpret_cast<const Loose<raw, alignof(T)> *>(p)->v;
        raw r = raw(0);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e < valid) {
                const unsigned b = sizeof(T) == 1 ? ((const unsigned char *)p)[e] : ((const unsigned short *)p)[e];
                r[e * (int)sizeof(T) / 4] |= (int)(b << (8 * (e * sizeof(T) % 4)));
            }
        }
        return r;
    }
};
__device__ inline i32x4 widened(i32x4 u) { return u; }
// e4m3 values are bf16 values too.
__device__ inline i32x4 widened(vec<int, 2> u) {
    using bf16x2 = vec<bf16, 2>;
    i32x4 r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        r[2 * h] = __builtin_bit_cast(int, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[h], 1.0f, false));
        r[2 * h + 1] = __builtin_bit_cast(int, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[h], 1.0f, true));
    }
    return r;
}

constexpr int kAnyTile = 128;
constexpr int kAnyUnits = kAnyTile * kStepBytes / 16 / 256;  // units of a tile each thread moves

template <typename T, bool kDown>
__device__ inline void fetch(typename Unit<T>::raw (&u)[kAnyUnits], const T *base, int64_t ld, int64_t at0, int64_t n_at, int64_t r0,
                             int64_t nr) {
#pragma unroll
    for (int n = 0; n < kAnyUnits; ++n) {
        const int c = threadIdx.x + n * 256;
        if constexpr (kDown) {  // 16 units a row of r
            const int64_t r = r0 + c / 16, at = at0 + (c % 16) * 8;
            u[n] = Unit<T>::load(base + r * ld + at, r < nr ? n_at - at : 0);
        } else {  // 8 units a row
            const int64_t at = at0 + c / 8, r = r0 + (c % 8) * 8;
            u[n] = Unit<T>::load(base + at * ld + r, at < n_at ? nr - r : 0);
        }
    }
}
template <typename T, bool kDown>
__device__ inline void place(const typename Unit<T>::raw (&u)[kAnyUnits], char *tile) {
#pragma unroll
    for (int n = 0; n < kAnyUnits; ++n) {
        const int c = threadIdx.x + n * 256;
        if constexpr (kDown) {
            const int r = c / 16, unit = c % 16;
            *(i32x4 *)(tile + r * kAnyTile * 2 + ((((unit >> 1) ^ down_bits(r)) << 5) | ((unit & 1) << 4))) = widened(u[n]);
        } else {
            *(i32x4 *)(tile + along_at(c / 8, c % 8)) = widened(u[n]);
        }
    }
}

// 128 x 128 of C by four waves of 64 x 64.  Units pass through registers, so
// rows may start anywhere and end inside a unit; the next step's are on their
// way while this step's are multiplied.  8-bit operands become bf16 on the way,
// which is exact: the 8-bit matrix instruction's own sums are not (see there).
template <typename T, typename O, bool kDownP, bool kDownQ>
__global__ __launch_bounds__(256) void product_any(Product a, Epilogue e, int64_t tiles_j) {
    __shared__ __attribute__((aligned(16))) char tile_p[2][kAnyTile * kStepBytes], tile_q[2][kAnyTile * kStepBytes];
    using C = std::conditional_t<sizeof(T) == 1, bf16, T>;
    constexpr int kStep = kStepBytes / 2;
    const int64_t i0 = blockIdx.x / tiles_j * kAnyTile, j0 = blockIdx.x % tiles_j * kAnyTile;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const int wi = (wave / 2) * 64, wj = (wave % 2) * 64;
    f32x4 acc[4][4] = {};
    typename Unit<T>::raw up[kAnyUnits], uq[kAnyUnits];
    const int64_t steps = (a.nr + kStep - 1) / kStep;
    if (steps > 0) {
        fetch<T, kDownP>(up, (const T *)a.p, a.ldp, i0, a.ni, 0, a.nr);
        fetch<T, kDownQ>(uq, (const T *)a.q, a.ldq, j0, a.nj, 0, a.nr);
        place<T, kDownP>(up, tile_p[0]);
        place<T, kDownQ>(uq, tile_q[0]);
        __syncthreads();
    }
    for (int64_t t = 0; t < steps; ++t) {
        const bool more = t + 1 < steps;
        if (more) {
            fetch<T, kDownP>(up, (const T *)a.p, a.ldp, i0, a.ni, (t + 1) * kStep, a.nr);
            fetch<T, kDownQ>(uq, (const T *)a.q, a.ldq, j0, a.nj, (t + 1) * kStep, a.nr);
        }
        const char *const tp = tile_p[t & 1], *const tq = tile_q[t & 1];
#pragma unroll
        for (int sub = 0; sub < Matrix<C>::kSub; ++sub) {
            typename Matrix<C>::frag p[4], q[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                p[n] = read_frag<C, kDownP>(tp, wi + n * 16, sub, kAnyTile);
                q[n] = read_frag<C, kDownQ>(tq, wj + n * 16, sub, kAnyTile);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) acc[x][y] = Matrix<C>::mma(q[y], p[x], acc[x][y]);
        }
        if (more) {
            place<T, kDownP>(up, tile_p[(t + 1) & 1]);
            place<T, kDownQ>(uq, tile_q[(t + 1) & 1]);
        }
        __syncthreads();
    }
    // a lane has columns 4 (lane / 16) .. + 3 of row lane % 16 of each 16 x 16 part
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int64_t i = i0 + wi + x * 16 + lane % 16;
        if (i >= a.ni) continue;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int64_t j = j0 + wj + y * 16 + (lane / 16) * 4;
            if (j < a.nj) finish<O>(acc[x][y], i, j, (int)std::min<int64_t>(4, a.nj - j), e);
        }
    }
}

template <typename T, typename O, bool kDownP, bool kDownQ>
hipError_t launch_product(const Product &a, const Epilogue &e, hipStream_t s) {
    if (a.ni == 0 || a.nj == 0) return hipSuccess;
    const int64_t ti = ceil_div(a.ni, kAnyTile), tj = ceil_div(a.nj, kAnyTile);
    hipLaunchKernelGGL((product_any<T, O, kDownP, kDownQ>), dim3((unsigned)(ti * tj)), dim3(256), 0, s, a, e, tj);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// dz = dy act'(z) and the bias's gradient
// ---------------------------------------------------------------------------
struct SlopeArgs {
    const void *dy, *pre;
    void *dz;        // NULL: only the sums
    float *partial;  // [gridDim.y, n] sums of dz's rows, or NULL
    int64_t m, n, lddy, ldp, ldz;
    int act;
};

// 256 columns by 8 rows at a time; a block goes down its share of the rows and
// leaves one row of sums.  dz's rows are padded with zeros to ldz.
template <typename E>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a) {
    using f32x8 = vec<float, 8>;
    __shared__ float strand[8][256 + 8];
    const int64_t col = (int64_t)blockIdx.x * 256 + (threadIdx.x % 32) * 8;
    const int g = threadIdx.x / 32;
    const int valid = (int)std::max<int64_t>(0, std::min<int64_t>(8, a.n - col));
    const int64_t width = a.dz ? a.ldz : a.n;
    f32x8 sum(0.0f);
    if (col < width) {
        for (int64_t row = (int64_t)blockIdx.y * 8 + g; row < a.m; row += (int64_t)gridDim.y * 8) {
            f32x8 d = load_f32<E, 8>((const E *)a.dy + row * a.lddy + col, valid);
            if (a.act != TG_ACT_NONE) {
                const f32x8 z = load_f32<E, 8>((const E *)a.pre + row * a.ldp + col, valid);
#pragma unroll
                for (int c = 0; c < 8; ++c) d[c] *= slope(z[c], a.act);
            }
            if (a.dz) {
#pragma unroll
                for (int c = 0; c < 8; ++c) d[c] = c < valid ? d[c] : 0.0f;
                store_f32<E, 8>((E *)a.dz + row * a.ldz + col, d, 8);
            }
            sum += d;
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int c = 0; c < 8; ++c) strand[g][(threadIdx.x % 32) * 8 + c] = sum[c];
    __syncthreads();
    const int64_t out = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (out >= a.n) return;
    float total = strand[0][threadIdx.x];
#pragma unroll
    for (int h = 1; h < 8; ++h) total += strand[h][threadIdx.x];
    a.partial[blockIdx.y * a.n + out] = total;
}

int slope_rows(int64_t m, int64_t n) {  // blocks down the rows: about 2048 blocks in all, 8 rows at least in each
    const int64_t want = std::max<int64_t>(1, 2048 / std::max<int64_t>(1, ceil_div(n, 256)));
    return (int)std::min<int64_t>(want, std::max<int64_t>(1, ceil_div(m, 8)));
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
size_t size_of(int type) { return type == TG_F32 ? 4 : type == TG_E4M3 ? 1 : 2; }

tg_status check_matrix(const void *p, int64_t ld, int64_t rows, int64_t cols, int type, const char *what) {
    if (rows == 0 || cols == 0) return TG_OK;
    if (!p) return call_failed(TG_EINVAL, "%s is NULL", what);
    if ((uintptr_t)p % size_of(type)) return call_failed(TG_EINVAL, "%s is not aligned to its elements", what);
    if (rows > 1 && ld < cols)
        return call_failed(TG_EINVAL, "%s: row stride %lld below the row length %lld", what, (long long)ld, (long long)cols);
    return TG_OK;
}

bool sizes_fit(int64_t m, int64_t n, int64_t k) {
    const int64_t most = 0x7fffffff - 256;
    return m >= 0 && n >= 0 && k >= 0 && m <= most && n <= most && k <= most &&
           ceil_div(m, kAnyTile) * ceil_div(std::max(n, k), kAnyTile) < (1 << 24) &&
           ceil_div(n, kAnyTile) * ceil_div(k, kAnyTile) < (1 << 24);
}

bool valid_types(int type, int out_type) {
    if (type == TG_E4M3) return out_type == TG_BF16 || out_type == TG_F16;
    return (type == TG_BF16 || type == TG_F16) && out_type == type;
}

struct GradPlan {
    bool slope, sums;  // dz differs from dy; a bias's gradient is wanted
    int64_t ldz;
    int rows;
    size_t dz_bytes, sum_bytes;
};

GradPlan plan_grad(const tg_linear_grad_args &q) {
    GradPlan p;
    p.slope = q.act != TG_ACT_NONE && (q.dx || q.dw);
    p.sums = q.dbias != nullptr;
    p.ldz = ceil_div(q.n, 8) * 8;
    p.rows = slope_rows(q.m, q.n);
    p.dz_bytes = p.slope ? round256((size_t)q.m * p.ldz * 2) : 0;
    p.sum_bytes = p.sums ? round256((size_t)p.rows * q.n * 4) : 0;
    return p;
}

template <typename E>
tg_status run_grad(const tg_linear_grad_args &q, const GradPlan &p, char *ws, hipStream_t s) {
    const void *dz = q.dy;
    int64_t ldz = q.lddy;
    if ((p.slope || p.sums) && q.m > 0 && q.n > 0) {
        SlopeArgs a{q.dy, q.pre, p.slope ? ws : nullptr, p.sums ? (float *)(ws + p.dz_bytes) : nullptr,
                    q.m, q.n, q.lddy, q.ldp, p.ldz, q.act};
        hipLaunchKernelGGL(slope_kernel<E>, dim3((unsigned)ceil_div(q.n, 256), p.rows), dim3(256), 0, s, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return device_failed(e, "slope_kernel");
        if (p.slope) dz = ws, ldz = p.ldz;
    }
    if (p.sums) {
        const hipError_t e = launch_column_sums((const float *)(ws + p.dz_bytes), q.m > 0 ? p.rows : 0, q.n, q.dbias, q.type, s);
        if (e != hipSuccess) return device_failed(e, "column_sums");
    }
    if (q.dx) {
        Epilogue e{};
        e.out = q.dx, e.ldo = q.lddx;
        const hipError_t r = launch_product<E, E, false, true>(Product{dz, q.w, ldz, q.ldw, q.m, q.k, q.n}, e, s);
        if (r != hipSuccess) return device_failed(r, "the product dz w");
    }
    if (q.dw) {
        Epilogue e{};
        e.out = q.dw, e.ldo = q.lddw;
        const hipError_t r = launch_product<E, E, true, true>(Product{dz, q.x, ldz, q.ldx, q.n, q.k, q.m}, e, s);
        if (r != hipSuccess) return device_failed(r, "the product dz^T x");
    }
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

size_t tg_linear_workspace_bytes(const tg_linear_args *q) {
    (void)q;
    return 0;
}

tg_status tg_linear(const tg_linear_args *q, void *d_ws, size_t ws_bytes, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    if (q->reserved) return call_failed(TG_EINVAL, "reserved must be 0");
    if (!valid_types(q->type, q->out_type)) return call_failed(TG_EINVAL, "type %d with out_type %d", q->type, q->out_type);
    if (q->act < TG_ACT_NONE || q->act > TG_ACT_GELU) return call_failed(TG_EINVAL, "act %d", q->act);
    if (!sizes_fit(q->m, q->n, q->k))
        return call_failed(TG_EINVAL, "m %lld, n %lld, k %lld", (long long)q->m, (long long)q->n, (long long)q->k);
    if ((q->x_scale != nullptr) != (q->w_scale != nullptr) || (q->x_scale && q->type != TG_E4M3))
        return call_failed(TG_EINVAL, "x_scale and w_scale come together, with 8-bit inputs");
    TG_TRY(check_matrix(q->x, q->ldx, q->m, q->k, q->type, "x"));
    TG_TRY(check_matrix(q->w, q->ldw, q->n, q->k, q->type, "w"));
    TG_TRY(check_matrix(q->y, q->ldy, q->m, q->n, q->out_type, "y"));
    if (q->pre) TG_TRY(check_matrix(q->pre, q->ldp, q->m, q->n, q->out_type, "pre"));
    if (q->residual) TG_TRY(check_matrix(q->residual, q->ldr, q->m, q->n, q->out_type, "residual"));
    if (q->bias) TG_TRY(check_matrix(q->bias, 0, 1, q->n, q->out_type, "bias"));
    if (q->x_scale) TG_TRY(check_matrix(q->x_scale, 0, 1, q->m, TG_F32, "x_scale"));
    if (q->w_scale) TG_TRY(check_matrix(q->w_scale, 0, 1, q->n, TG_F32, "w_scale"));
    const Product a{q->x, q->w, q->ldx, q->ldw, q->m, q->n, q->k};
    const Epilogue e{q->x_scale, q->w_scale, q->bias, q->residual, q->y, q->pre, q->ldr, q->ldy, q->ldp, q->act};
    const hipStream_t s = (hipStream_t)stream;
    hipError_t r;
    if (q->type == TG_BF16)
        r = launch_product<bf16, bf16, false, false>(a, e, s);
    else if (q->type == TG_F16)
        r = launch_product<f16, f16, false, false>(a, e, s);
    else if (q->out_type == TG_BF16)
        r = launch_product<e4m3, bf16, false, false>(a, e, s);
    else
        r = launch_product<e4m3, f16, false, false>(a, e, s);
    return r == hipSuccess ? TG_OK : device_failed(r, "the product x w^T");
}

size_t tg_linear_grad_workspace_bytes(const tg_linear_grad_args *q) {
    if (!q || !sizes_fit(q->m, q->n, q->k)) return 0;
    const GradPlan p = plan_grad(*q);
    return p.dz_bytes + p.sum_bytes;
}

tg_status tg_linear_grad(const tg_linear_grad_args *q, void *d_ws, size_t ws_bytes, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    if (q->type != TG_BF16 && q->type != TG_F16) return call_failed(TG_EINVAL, "type %d", q->type);
    if (q->act < TG_ACT_NONE || q->act > TG_ACT_GELU) return call_failed(TG_EINVAL, "act %d", q->act);
    if (!sizes_fit(q->m, q->n, q->k))
        return call_failed(TG_EINVAL, "m %lld, n %lld, k %lld", (long long)q->m, (long long)q->n, (long long)q->k);
    TG_TRY(check_matrix(q->dy, q->lddy, q->m, q->n, q->type, "dy"));
    if (q->act != TG_ACT_NONE) TG_TRY(check_matrix(q->pre, q->ldp, q->m, q->n, q->type, "pre"));
    if (q->dw) {
        TG_TRY(check_matrix(q->x, q->ldx, q->m, q->k, q->type, "x"));
        TG_TRY(check_matrix(q->dw, q->lddw, q->n, q->k, q->type, "dw"));
    }
    if (q->dx) {
        TG_TRY(check_matrix(q->w, q->ldw, q->n, q->k, q->type, "w"));
        TG_TRY(check_matrix(q->dx, q->lddx, q->m, q->k, q->type, "dx"));
    }
    if (q->dbias) TG_TRY(check_matrix(q->dbias, 0, 1, q->n, q->type, "dbias"));
    const GradPlan p = plan_grad(*q);
    const size_t need = p.dz_bytes + p.sum_bytes;
    if ((uintptr_t)d_ws % 256) return call_failed(TG_EINVAL, "the workspace is not 256-byte aligned");
    if (need && (!d_ws || ws_bytes < need)) return call_failed(TG_ENOMEM, "workspace of %zu bytes, %zu needed", d_ws ? ws_bytes : 0, need);
    return q->type == TG_BF16 ? run_grad<bf16>(*q, p, (char *)d_ws, (hipStream_t)stream)
                              : run_grad<f16>(*q, p, (char *)d_ws, (hipStream_t)stream);
}

}  // extern "C"
