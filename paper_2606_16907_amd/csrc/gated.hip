// gated.hip -- the gated projections of a feed-forward half: gate and up, the
// activation and their product in one kernel (tg_gated), and their gradients
// (tg_gated_grad).
//
// The products as product.h has them:
//        y        = act(x wg^T) (x wu^T)    P = x, Q = wg and wu side by side (kGated)
//        dx       = dg wg + du wu           P = [dg | du], Q = wg, then wu, with r down
//                                           their columns (kSeam)
//        dwg, dwu = dg^T x, du^T x          P = [dg | du], Q = x, with r down their
//                                           columns, C's rows to two outputs (kHalves)
// Gate and up are never read again for y, and each gradient is one product of twice
// the size: more tiles at once, and the sums of dx meet in registers.  Bound by the
// matrix units and by power as the plain products: 4096 x 4096 x 14336 in bf16 takes
// 760 to 820 us forward with gate and up kept (1170 to 1270 TFLOP/s; the library's
// product alone 728), 690 to 720 for dx (714) and 750 to 820 for the weights (946).
// One row through two weights of 4096 x 14336 takes 41 us, 5.7 TB/s.
#include "product.h"

namespace tg {
namespace {

// ---------------------------------------------------------------------------
// dg = dy up act'(gate), du = dy act(gate), and the biases' gradients
// ---------------------------------------------------------------------------
struct GatedSlopeArgs {
    const void *dy, *gate, *up;
    void *dz;        // [m, 2 half]: dg and du, each padded with zeros to `half` columns; NULL: only the sums
    float *partial;  // [2][rows, n] sums of dg's and du's rows, or NULL
    int64_t m, n, lddy, ldg, ldu, half;
    int act;
};

// act(z), and its slope, which share the exponential and the distribution function.
// z comes in 16 bits, where one that was finite may be an infinity: beyond |z| = 128
// the slope is its limit as in slope(), and so is the value, 0 below and z above.
template <int N>
__device__ inline vec<float, N> value_and_slope(vec<float, N> z, int act, vec<float, N> *value) {
    vec<float, N> s(1.0f);
    *value = z;
    if (act == TG_ACT_RELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            s[c] = z[c] > 0.0f ? 1.0f : 0.0f;
            (*value)[c] = z[c] < 0.0f ? 0.0f : z[c];
        }
    } else if (act == TG_ACT_SILU) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const float h = held(z[c]), t = __builtin_amdgcn_rcpf(1.0f + exp_f32(-h));
            s[c] = t * fmaf(h, 1.0f - t, 1.0f);
            (*value)[c] = (z[c] > 128.0f ? z[c] : h) * t;
        }
    } else if (act == TG_ACT_GELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const float h = held(z[c]), bell = exp_f32(-0.5f * h * h), cdf = normal_cdf(h, bell);
            s[c] = fmaf(h * 0.39894228f, bell, cdf);
            (*value)[c] = (z[c] > 128.0f ? z[c] : h) * cdf;
        }
    }
    return s;
}

// 256 columns by 8 rows at a time; a block goes down its share of the rows.  dg and
// du are rounded to the inputs' 16 bits because the matrix instructions of the
// products read no more; the biases' sums take them before that.  Bound by memory:
// three matrices read, two written (4096 x 14336 in bf16 takes 117 us, 5.0 TB/s).
// Rows of blocks from `rows` on pack what the products cannot stream.
template <typename E>
__global__ __launch_bounds__(256) void gated_slope_kernel(GatedSlopeArgs a, Packing k, int rows) {
    if ((int)blockIdx.y >= rows) {
        const int64_t blocks = (int64_t)(gridDim.y - rows) * gridDim.x, block = (int64_t)(blockIdx.y - rows) * gridDim.x + blockIdx.x;
#pragma unroll
        for (int o = 0; o < 3; ++o) pack_body<E>(k, o, block, blocks);
        return;
    }
    using f32x8 = vec<float, 8>;
    __shared__ float strand[2][8][256 + 8];
    const int64_t col = (int64_t)blockIdx.x * 256 + (threadIdx.x % 32) * 8;
    const int g = threadIdx.x / 32;
    const int valid = (int)std::max<int64_t>(0, std::min<int64_t>(8, a.n - col));
    const int64_t width = a.dz ? a.half : a.n;
    f32x8 sum[2] = {f32x8(0.0f), f32x8(0.0f)};
    if (col < width) {
        for (int64_t row = (int64_t)blockIdx.y * 8 + g; row < a.m; row += (int64_t)rows * 8) {
            const f32x8 dy = load_f32<E, 8>((const E *)a.dy + row * a.lddy + col, valid);
            const f32x8 gate = load_f32<E, 8>((const E *)a.gate + row * a.ldg + col, valid);
            const f32x8 up = load_f32<E, 8>((const E *)a.up + row * a.ldu + col, valid);
            f32x8 d[2], value;
            d[0] = dy * up * value_and_slope<8>(gate, a.act, &value);
            d[1] = dy * value;
#pragma unroll
            for (int o = 0; o < 2; ++o) {
#pragma unroll
                for (int c = 0; c < 8; ++c) d[o][c] = c < valid ? d[o][c] : 0.0f;
                if (a.dz) store_f32<E, 8>((E *)a.dz + row * 2 * a.half + o * a.half + col, d[o], 8);
                sum[o] += d[o];
            }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int o = 0; o < 2; ++o) {
#pragma unroll
        for (int c = 0; c < 8; ++c) strand[o][g][(threadIdx.x % 32) * 8 + c] = sum[o][c];
    }
    __syncthreads();
    const int64_t out = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (out >= a.n) return;
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        float total = strand[o][0][threadIdx.x];
#pragma unroll
        for (int h = 1; h < 8; ++h) total += strand[o][h][threadIdx.x];
        a.partial[((int64_t)o * rows + blockIdx.y) * a.n + out] = total;
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// Columns of dg and of du in their common matrix: whole steps of dx's product.
int64_t half_of(int64_t n) { return ceil_div(n, 64) * 64; }

bool gated_fits(int64_t m, int64_t n, int64_t k) { return n >= 0 && n <= kMostLd && sizes_fit(m, 2 * half_of(n), k); }

Product forward_product(const tg_gated_args &q) {
    Product a{q.x, q.w_gate, ld_of(q.ldx, q.m, q.k, q.type), ld_of(q.ldwg, q.n, q.k, q.type), q.m, q.n, q.k};
    a.q2 = q.w_up, a.ldq2 = ld_of(q.ldwu, q.n, q.k, q.type);
    return a;
}

// Both gradients' products in one launch, in tiles of 128, a place on each CU for
// either: small ones leave half of the GPU idle by themselves.  1531 x 1001 x 1367 in
// f16 takes 29 us, and what comes after it 5, where two launches took 19 and 18 and
// theirs 8.  cut_gradients chooses.
struct OneOfTwo {
    Product a;
    Epilogue e;
    int64_t r_bytes_p, r_bytes_q;
    int tiles_i, tiles_j, share, whole, splits;
    unsigned blocks, join_blocks;
};
template <Form kForm>
OneOfTwo one_of_two(const Product &a, Epilogue e, int64_t r_bytes_p, int64_t r_bytes_q, const TailCut &c, float *sums) {
    e.seam = a.seam, e.half = a.half, e.partial = sums;
    return {a, e, r_bytes_p, r_bytes_q, (int)ceil_div(a.ni, 128), (int)ceil_div(a.nj, 128), c.share, c.whole, c.splits,
            (unsigned)(c.whole + c.tail * c.splits), join_blocks<kForm>(c)};
}
template <typename E>
__global__ __launch_bounds__(256, 2) void product_two(OneOfTwo dx, OneOfTwo dw) {
    __shared__ __attribute__((aligned(1024))) char tiles[kPlace<2, 2>];
    const auto run = [&](auto form, auto down_p, const OneOfTwo &p, int64_t b) {
        const TailBlock block = tail_block(b, p.whole, (int64_t)p.tiles_i * p.tiles_j, p.splits);
        product_body<E, E, down_p, true, 2, 2, form>(tiles, block, p.a, p.e, p.tiles_i, p.tiles_j, p.r_bytes_p, p.r_bytes_q, p.share);
    };
    if (blockIdx.x < dx.blocks)
        run(std::integral_constant<Form, kSeam>{}, std::false_type{}, dx, blockIdx.x);
    else
        run(std::integral_constant<Form, kHalves>{}, std::true_type{}, dw, blockIdx.x - dx.blocks);
}
// What is left after them: the shares of both, and the biases' sums (32 columns of one bias a block).
template <typename E>
__global__ __launch_bounds__(256) void finish_two(OneOfTwo dx, OneOfTwo dw, const float *partial, int rows, int64_t n, E *bias, E *bias2) {
    unsigned b = blockIdx.x;
    if (b < dx.join_blocks) {
        join_body<E, kSeam, 128>(b, dx.e, dx.whole, dx.splits, dx.tiles_i, dx.tiles_j, dx.a.ni, dx.a.nj);
    } else if ((b -= dx.join_blocks) < dw.join_blocks) {
        join_body<E, kHalves, 128>(b, dw.e, dw.whole, dw.splits, dw.tiles_i, dw.tiles_j, dw.a.ni, dw.a.nj);
    } else {
        b -= dw.join_blocks;
        E *const out = b % 2 ? bias2 : bias;
        if (out) column_sums_block(partial + (b % 2 ? rows * n : 0), rows, n, (int64_t)(b / 2) * 32, out);
    }
}

// What tg_gated_grad does, and what lies where in its workspace: dg and du, the
// biases' sums, packed weights, packed x, shares of dx and of the weights' gradients.
struct GatedGradPlan {
    bool dz, sums, weights, two, pack_w, pack_x;
    int64_t half;
    int rows;
    size_t dz_bytes, sum_bytes, w_bytes, x_bytes, dx_bytes, dw_bytes;
    Product dx, dw;
    TailCut cut_dx, cut_dw;
    size_t bytes() const { return dz_bytes + sum_bytes + 2 * w_bytes + x_bytes + dx_bytes + dw_bytes; }
};

GatedGradPlan plan_grad(const tg_gated_grad_args &q, char *ws) {
    GatedGradPlan p{};
    p.weights = q.dw_gate || q.dw_up;
    p.dz = q.dx || p.weights;
    p.sums = q.dgate_bias || q.dup_bias;
    p.half = half_of(q.n);
    p.rows = slope_rows(q.m, q.n);
    p.dz_bytes = p.dz ? round256((size_t)q.m * 2 * p.half * 2) : 0;
    p.sum_bytes = p.sums ? round256((size_t)2 * p.rows * q.n * 4) : 0;
    const int64_t ldz = 2 * p.half;
    p.dx = Product{ws, q.w_gate, ldz, ld_of(q.ldwg, q.n, q.k, q.type), q.m, q.k, ldz};
    p.dx.q2 = q.w_up, p.dx.ldq2 = ld_of(q.ldwu, q.n, q.k, q.type), p.dx.seam = p.half, p.dx.half = q.n;
    // one weight's gradient alone: the first half of the rows, from its columns of dg and du on
    const bool both = q.dw_gate && q.dw_up;
    p.dw = Product{ws + (both || q.dw_gate ? 0 : p.half * 2), q.x, ldz, ld_of(q.ldx, q.m, q.k, q.type), both ? ldz : p.half, q.k, q.m};
    p.dw.seam = p.half, p.dw.half = q.n;
    if (q.m == 0 || q.n == 0 || q.k == 0) {  // empty sums or empty outputs: nothing is read
        if (q.dx) p.cut_dx = cut_tail(p.dx.ni, p.dx.nj, 0, 2);
        if (p.weights) p.cut_dw = cut_tail(p.dw.ni, p.dw.nj, 0, 2);
        return p;
    }
    const int64_t packed_k = whole_ld(q.k, 2) * 2;
    p.pack_w = q.dx && (!streams(p.dx.q, p.dx.ldq, 2, 0, true) || !streams(p.dx.q2, p.dx.ldq2, 2, 0, true) || p.dx.ldq != p.dx.ldq2);
    p.pack_x = p.weights && !streams(p.dw.q, p.dw.ldq, 2, 0, true);
    p.w_bytes = p.pack_w ? round256(q.n * packed_k) : 0;
    p.x_bytes = p.pack_x ? round256(q.m * packed_k) : 0;
    const GradCut c = cut_gradients(q.m, q.k, ldz, p.dw.ni, q.dx, p.weights);
    p.cut_dx = c.dx, p.cut_dw = c.dw, p.two = c.two;
    p.dx_bytes = round256(p.cut_dx.bytes());
    p.dw_bytes = round256(p.cut_dw.bytes());
    if (!p.two && p.dx_bytes && p.dw_bytes) p.dx_bytes = std::max(p.dx_bytes, p.dw_bytes), p.dw_bytes = 0;  // one after the other
    return p;
}

template <typename E>
tg_status run_grad(const tg_gated_grad_args &q, GatedGradPlan &p, char *ws, hipStream_t s) {
    float *const sums = (float *)(ws + p.dz_bytes);
    char *const packed = ws + p.dz_bytes + p.sum_bytes;
    float *const dx_sums = (float *)(packed + 2 * p.w_bytes + p.x_bytes);
    float *const dw_sums = p.dw_bytes ? (float *)((char *)dx_sums + p.dx_bytes) : dx_sums;
    Packing k{};
    if (p.pack_w) {
        pack_operand(k, 0, p.dx.q, p.dx.ldq, q.n, q.k, 2, packed);
        pack_operand(k, 1, p.dx.q2, p.dx.ldq2, q.n, q.k, 2, packed + p.w_bytes);
    }
    if (p.pack_x) pack_operand(k, 2, p.dw.q, p.dw.ldq, q.m, q.k, 2, packed + 2 * p.w_bytes);
    if (q.m > 0 && q.n > 0) {
        const GatedSlopeArgs a{q.dy, q.gate, q.up, p.dz ? ws : nullptr, p.sums ? sums : nullptr, q.m, q.n, q.lddy, q.ldg, q.ldu, p.half, q.act};
        const int64_t across = ceil_div(p.half, 256);
        const int64_t units = std::max({k.rows[0] * k.ld_to[0], k.rows[1] * k.ld_to[1], k.rows[2] * k.ld_to[2]}) / 8;
        const unsigned more = (unsigned)ceil_div(std::min<int64_t>(2048, ceil_div(units, 256)), across);
        hipLaunchKernelGGL(gated_slope_kernel<E>, dim3((unsigned)across, p.rows + more), dim3(256), 0, s, a, k, p.rows);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return device_failed(e, "gated_slope_kernel");
    }
    Epilogue ex{}, ew{};
    ex.out = q.dx, ex.ldo = q.lddx;
    ew.out = q.dw_gate ? q.dw_gate : q.dw_up, ew.ldo = q.dw_gate ? q.lddwg : q.lddwu;
    ew.out2 = q.dw_up, ew.ldo2 = q.lddwu;
    if (p.two) {
        const OneOfTwo dx = one_of_two<kSeam>(p.dx, ex, p.dx.ldp * 2, 0, p.cut_dx, dx_sums), dw = one_of_two<kHalves>(p.dw, ew, 0, 0, p.cut_dw, dw_sums);
        hipLaunchKernelGGL(product_two<E>, dim3(dx.blocks + dw.blocks), dim3(256), 0, s, dx, dw);
        const unsigned rest = dx.join_blocks + dw.join_blocks + (p.sums ? 2 * (unsigned)ceil_div(q.n, 32) : 0);
        if (rest) hipLaunchKernelGGL(finish_two<E>, dim3(rest), dim3(256), 0, s, dx, dw, sums, p.rows, q.n, (E *)q.dgate_bias, (E *)q.dup_bias);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? TG_OK : device_failed(e, "the gradients' products");
    }
    if (p.sums) {
        const hipError_t e = launch_column_sums_of_two(sums, q.m > 0 ? p.rows : 0, q.n, q.dgate_bias, q.dup_bias, q.type, s);
        if (e != hipSuccess) return device_failed(e, "column_sums");
    }
    if (q.dx) {
        const hipError_t r = launch_tiles<E, E, false, true, kSeam>(p.dx, ex, p.dx.ldp * 2, 0, p.cut_dx, dx_sums, s);
        if (r != hipSuccess) return device_failed(r, "the product dg wg + du wu");
    }
    if (p.weights) {
        const hipError_t r = launch_tiles<E, E, true, true, kHalves>(p.dw, ew, 0, 0, p.cut_dw, dw_sums, s);
        if (r != hipSuccess) return device_failed(r, "the products dg^T x and du^T x");
    }
    return TG_OK;
}

}  // namespace
}  // namespace tg

using namespace tg;

extern "C" {

size_t tg_gated_workspace_bytes(const tg_gated_args *q) {
    if (!q || !valid_types(q->type, q->out_type) || !gated_fits(q->m, q->n, q->k)) return 0;
    const int size = (int)size_of(q->type);
    return plan_product<kGated>(forward_product(*q), size, q->k * size, false, false).bytes;
}

tg_status tg_gated(const tg_gated_args *q, void *d_ws, size_t ws_bytes, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    if (q->reserved) return call_failed(TG_EINVAL, "reserved must be 0");
    if (!valid_types(q->type, q->out_type)) return call_failed(TG_EINVAL, "type %d with out_type %d", q->type, q->out_type);
    if (q->act < TG_ACT_NONE || q->act > TG_ACT_GELU) return call_failed(TG_EINVAL, "act %d", q->act);
    if (!gated_fits(q->m, q->n, q->k))
        return call_failed(TG_EINVAL, "m %lld, n %lld, k %lld", (long long)q->m, (long long)q->n, (long long)q->k);
    const bool scaled = q->x_scale || q->gate_scale || q->up_scale;
    // those of no rows or columns may be NULL
    if (scaled && (q->type != TG_E4M3 || (!q->x_scale && q->m > 0) || ((!q->gate_scale || !q->up_scale) && q->n > 0)))
        return call_failed(TG_EINVAL, "x_scale, gate_scale and up_scale come together, with 8-bit inputs");
    if ((q->gate != nullptr) != (q->up != nullptr)) return call_failed(TG_EINVAL, "gate and up are kept together");
    TG_TRY(check_matrix(q->x, q->ldx, q->m, q->k, q->type, "x"));
    TG_TRY(check_matrix(q->w_gate, q->ldwg, q->n, q->k, q->type, "w_gate"));
    TG_TRY(check_matrix(q->w_up, q->ldwu, q->n, q->k, q->type, "w_up"));
    TG_TRY(check_matrix(q->y, q->ldy, q->m, q->n, q->out_type, "y"));
    if (q->gate) TG_TRY(check_matrix(q->gate, q->ldg, q->m, q->n, q->out_type, "gate"));
    if (q->up) TG_TRY(check_matrix(q->up, q->ldu, q->m, q->n, q->out_type, "up"));
    if (q->gate_bias) TG_TRY(check_matrix(q->gate_bias, 0, 1, q->n, q->out_type, "gate_bias"));
    if (q->up_bias) TG_TRY(check_matrix(q->up_bias, 0, 1, q->n, q->out_type, "up_bias"));
    if (scaled) {
        TG_TRY(check_matrix(q->x_scale, 0, 1, q->m, TG_F32, "x_scale"));
        TG_TRY(check_matrix(q->gate_scale, 0, 1, q->n, TG_F32, "gate_scale"));
        TG_TRY(check_matrix(q->up_scale, 0, 1, q->n, TG_F32, "up_scale"));
    }
    TG_TRY(check_workspace(d_ws, ws_bytes, tg_gated_workspace_bytes(q)));
    const Product a = forward_product(*q);
    Epilogue e{};
    e.x_scale = q->x_scale, e.w_scale = q->gate_scale, e.w_scale2 = q->up_scale;
    e.bias = q->gate_bias, e.bias2 = q->up_bias;
    e.out = q->y, e.pre = q->gate, e.pre2 = q->up;
    e.ldo = q->ldy, e.ldp = q->ldg, e.ldp2 = q->ldu, e.act = q->act;
    const hipStream_t s = (hipStream_t)stream;
    char *const ws = (char *)d_ws;
    hipError_t r;
    if (q->type == TG_BF16)
        r = launch_product<bf16, bf16, false, false, kGated>(a, e, q->k * 2, ws, s);
    else if (q->type == TG_F16)
        r = launch_product<f16, f16, false, false, kGated>(a, e, q->k * 2, ws, s);
    else if (q->out_type == TG_BF16)
        r = launch_product<e4m3, bf16, false, false, kGated>(a, e, q->k, ws, s);
    else
        r = launch_product<e4m3, f16, false, false, kGated>(a, e, q->k, ws, s);
    return r == hipSuccess ? TG_OK : device_failed(r, "the gated products");
}

size_t tg_gated_grad_workspace_bytes(const tg_gated_grad_args *q) {
    if (!q || !gated_fits(q->m, q->n, q->k)) return 0;
    return plan_grad(*q, nullptr).bytes();
}

tg_status tg_gated_grad(const tg_gated_grad_args *q, void *d_ws, size_t ws_bytes, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    if (q->type != TG_BF16 && q->type != TG_F16) return call_failed(TG_EINVAL, "type %d", q->type);
    if (q->act < TG_ACT_NONE || q->act > TG_ACT_GELU) return call_failed(TG_EINVAL, "act %d", q->act);
    if (!gated_fits(q->m, q->n, q->k))
        return call_failed(TG_EINVAL, "m %lld, n %lld, k %lld", (long long)q->m, (long long)q->n, (long long)q->k);
    TG_TRY(check_matrix(q->dy, q->lddy, q->m, q->n, q->type, "dy"));
    TG_TRY(check_matrix(q->gate, q->ldg, q->m, q->n, q->type, "gate"));
    TG_TRY(check_matrix(q->up, q->ldu, q->m, q->n, q->type, "up"));
    if (q->dw_gate || q->dw_up) TG_TRY(check_matrix(q->x, q->ldx, q->m, q->k, q->type, "x"));
    if (q->dw_gate) TG_TRY(check_matrix(q->dw_gate, q->lddwg, q->n, q->k, q->type, "dw_gate"));
    if (q->dw_up) TG_TRY(check_matrix(q->dw_up, q->lddwu, q->n, q->k, q->type, "dw_up"));
    if (q->dx) {
        TG_TRY(check_matrix(q->w_gate, q->ldwg, q->n, q->k, q->type, "w_gate"));
        TG_TRY(check_matrix(q->w_up, q->ldwu, q->n, q->k, q->type, "w_up"));
        TG_TRY(check_matrix(q->dx, q->lddx, q->m, q->k, q->type, "dx"));
    }
    if (q->dgate_bias) TG_TRY(check_matrix(q->dgate_bias, 0, 1, q->n, q->type, "dgate_bias"));
    if (q->dup_bias) TG_TRY(check_matrix(q->dup_bias, 0, 1, q->n, q->type, "dup_bias"));
    GatedGradPlan p = plan_grad(*q, (char *)d_ws);
    TG_TRY(check_workspace(d_ws, ws_bytes, p.bytes()));
    return q->type == TG_BF16 ? run_grad<bf16>(*q, p, (char *)d_ws, (hipStream_t)stream)
                              : run_grad<f16>(*q, p, (char *)d_ws, (hipStream_t)stream);
}

}  // extern "C"
