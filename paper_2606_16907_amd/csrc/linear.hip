// linear.hip -- matrix product with bias, activation and residual in its
// epilogue (tg_linear), and its gradients (tg_linear_grad).
//
// The three products as product.h has them:
//        y  = x w^T    P = x, Q = w, both with r along their rows
//        dx = dz w     P = dz,       Q = w with r down its columns
//        dw = dz^T x   P = dz and Q = x with r down their columns
#include "product.h"

namespace tg {
namespace {

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
// leaves one row of sums.  dz's rows are padded with zeros to ldz.  z is what the
// forward pass kept of it in 16 bits, and dz is rounded to 16 bits because the
// matrix instructions of the two products read no more; the bias's sums take it
// before that.  Bound by memory: 8192 x 6144 in bf16 takes 59 us, 5.1 TB/s.
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
                d *= slope<8>(load_f32<E, 8>((const E *)a.pre + row * a.ldp + col, valid), a.act);
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

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// What tg_linear_grad does, and what lies where in its workspace: dz, sums, and
// the place of the two products, which run one after the other.
struct GradPlan {
    bool slope, sums;  // dz is not dy where it lies; a bias's gradient is wanted
    int64_t ldz;
    int rows;
    size_t dz_bytes, sum_bytes, product_bytes;
    Product dx, dw;
    size_t bytes() const { return dz_bytes + sum_bytes + product_bytes; }
};

GradPlan plan_grad(const tg_linear_grad_args &q, char *ws) {
    GradPlan p{};
    const int64_t lddy = ld_of(q.lddy, q.m, q.n, q.type);
    // dy is read as it lies where there is no activation and its rows are aligned
    p.slope = (q.dx || q.dw) && (q.act != TG_ACT_NONE || !streams(q.dy, lddy, 2, q.n * 2, false));
    p.sums = q.dbias != nullptr;
    p.ldz = p.slope ? whole_ld(q.n, 2) : lddy;
    p.rows = slope_rows(q.m, q.n);
    p.dz_bytes = p.slope ? round256((size_t)q.m * p.ldz * 2) : 0;
    p.sum_bytes = p.sums ? round256((size_t)p.rows * q.n * 4) : 0;
    const void *const dz = p.slope ? ws : q.dy;
    p.dx = Product{dz, q.w, p.ldz, ld_of(q.ldw, q.n, q.k, q.type), q.m, q.k, q.n};
    p.dw = Product{dz, q.x, p.ldz, ld_of(q.ldx, q.m, q.k, q.type), q.n, q.k, q.m};
    if (q.dx) p.product_bytes = plan_product(p.dx, 2, (p.slope ? p.ldz * 2 : q.n * 2), false, true).bytes;
    if (q.dw) p.product_bytes = std::max(p.product_bytes, plan_product(p.dw, 2, 0, true, true).bytes);
    return p;
}

template <typename E>
tg_status run_grad(const tg_linear_grad_args &q, const GradPlan &p, char *ws, hipStream_t s) {
    char *const place = ws + p.dz_bytes + p.sum_bytes;
    float *const sums = (float *)(ws + p.dz_bytes);
    if ((p.slope || p.sums) && q.m > 0 && q.n > 0) {
        SlopeArgs a{q.dy, q.pre, p.slope ? ws : nullptr, p.sums ? sums : nullptr, q.m, q.n, q.lddy, q.ldp, p.ldz, q.act};
        hipLaunchKernelGGL(slope_kernel<E>, dim3((unsigned)ceil_div(q.n, 256), p.rows), dim3(256), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return device_failed(e, "slope_kernel");
    }
    if (p.sums) {
        const hipError_t e = launch_column_sums(sums, q.m > 0 ? p.rows : 0, q.n, q.dbias, q.type, s);
        if (e != hipSuccess) return device_failed(e, "column_sums");
    }
    if (q.dx) {
        Epilogue e{};
        e.out = q.dx, e.ldo = q.lddx;
        const hipError_t r = launch_product<E, E, false, true>(p.dx, e, (p.slope ? p.ldz * 2 : q.n * 2), place, s);
        if (r != hipSuccess) return device_failed(r, "the product dz w");
    }
    if (q.dw) {
        Epilogue e{};
        e.out = q.dw, e.ldo = q.lddw;
        const hipError_t r = launch_product<E, E, true, true>(p.dw, e, 0, place, s);
        if (r != hipSuccess) return device_failed(r, "the product dz^T x");
    }
    return TG_OK;
}

Product forward_product(const tg_linear_args &q) {
    return Product{q.x, q.w, ld_of(q.ldx, q.m, q.k, q.type), ld_of(q.ldw, q.n, q.k, q.type), q.m, q.n, q.k};
}

}  // namespace
}  // namespace tg

using namespace tg;

extern "C" {

size_t tg_linear_workspace_bytes(const tg_linear_args *q) {
    if (!q || !sizes_fit(q->m, q->n, q->k) || !valid_types(q->type, q->out_type)) return 0;
    const int size = (int)size_of(q->type);
    return plan_product(forward_product(*q), size, q->k * size, false, false).bytes;
}

tg_status tg_linear(const tg_linear_args *q, void *d_ws, size_t ws_bytes, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    if (q->reserved) return call_failed(TG_EINVAL, "reserved must be 0");
    if (!valid_types(q->type, q->out_type)) return call_failed(TG_EINVAL, "type %d with out_type %d", q->type, q->out_type);
    if (q->act < TG_ACT_NONE || q->act > TG_ACT_GELU) return call_failed(TG_EINVAL, "act %d", q->act);
    if (!sizes_fit(q->m, q->n, q->k))
        return call_failed(TG_EINVAL, "m %lld, n %lld, k %lld", (long long)q->m, (long long)q->n, (long long)q->k);
    // those of no rows or columns may be NULL
    if ((q->x_scale || q->w_scale) && (q->type != TG_E4M3 || (!q->x_scale && q->m > 0) || (!q->w_scale && q->n > 0)))
        return call_failed(TG_EINVAL, "x_scale and w_scale come together, with 8-bit inputs");
    TG_TRY(check_matrix(q->x, q->ldx, q->m, q->k, q->type, "x"));
    TG_TRY(check_matrix(q->w, q->ldw, q->n, q->k, q->type, "w"));
    TG_TRY(check_matrix(q->y, q->ldy, q->m, q->n, q->out_type, "y"));
    if (q->pre) TG_TRY(check_matrix(q->pre, q->ldp, q->m, q->n, q->out_type, "pre"));
    if (q->residual) TG_TRY(check_matrix(q->residual, q->ldr, q->m, q->n, q->out_type, "residual"));
    if (q->bias) TG_TRY(check_matrix(q->bias, 0, 1, q->n, q->out_type, "bias"));
    if (q->x_scale) TG_TRY(check_matrix(q->x_scale, 0, 1, q->m, TG_F32, "x_scale"));
    if (q->w_scale) TG_TRY(check_matrix(q->w_scale, 0, 1, q->n, TG_F32, "w_scale"));
    TG_TRY(check_workspace(d_ws, ws_bytes, tg_linear_workspace_bytes(q)));
    const Product a = forward_product(*q);
    const Epilogue e{q->x_scale, q->w_scale, q->bias, q->residual, q->y, q->pre, q->ldr, q->ldy, q->ldp, q->act, nullptr};
    const hipStream_t s = (hipStream_t)stream;
    char *const ws = (char *)d_ws;
    hipError_t r;
    if (q->type == TG_BF16)
        r = launch_product<bf16, bf16, false, false>(a, e, q->k * 2, ws, s);
    else if (q->type == TG_F16)
        r = launch_product<f16, f16, false, false>(a, e, q->k * 2, ws, s);
    else if (q->out_type == TG_BF16)
        r = launch_product<e4m3, bf16, false, false>(a, e, q->k, ws, s);
    else
        r = launch_product<e4m3, f16, false, false>(a, e, q->k, ws, s);
    return r == hipSuccess ? TG_OK : device_failed(r, "the product x w^T");
}

size_t tg_linear_grad_workspace_bytes(const tg_linear_grad_args *q) {
    if (!q || !sizes_fit(q->m, q->n, q->k)) return 0;
    return plan_grad(*q, nullptr).bytes();
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
    const GradPlan p = plan_grad(*q, (char *)d_ws);
    TG_TRY(check_workspace(d_ws, ws_bytes, p.bytes()));
    return q->type == TG_BF16 ? run_grad<bf16>(*q, p, (char *)d_ws, (hipStream_t)stream)
                              : run_grad<f16>(*q, p, (char *)d_ws, (hipStream_t)stream);
}

}  // extern "C"
