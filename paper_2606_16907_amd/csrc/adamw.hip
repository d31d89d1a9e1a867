// adamw.hip -- AdamW over many tensors in one launch (tg_adamw_*).
//
// Bound by memory: with 16-bit weights and gradients and a master copy a step
// moves 28 bytes a parameter with 32-bit moments and 16.06 with 8-bit ones, for
// about 20 operations.  A block takes 4096 elements of one tensor, found
// in a list that create() lays out, so short and long tensors mix in one grid;
// a wave has all loads of its 1024 elements in flight before it computes.  A
// 256-element block of an 8-bit state is four elements a lane of one wave, so
// its scale is a reduction over the wave and nothing is stored in between.
// 100.7 M parameters with 32-bit moments take 475 us (5.9 TB/s; 537 where what is
// read and written once stayed in the caches), 436 M with 8-bit ones 1284 (5.5
// TB/s; 1372 with the reductions through LDS), where a large copy reaches 4.8.
#include <cmath>
#include <cstddef>
#include <memory>
#include <new>
#include <vector>

#include "layer_device.h"

namespace tg {
namespace {

constexpr int kChunk = 4096;      // elements of a block of threads
constexpr int kScaleBlock = 256;  // elements that share a scale
constexpr int kSub = 4;           // scale blocks of a wave
constexpr int64_t kMostChunks = (1 << 24) - 1;  // a grid holds fewer than 2^32 threads

struct ChunkOf {
    int tensor, chunk;
};

struct Rates {
    float beta1, beta2, one_minus_beta1, one_minus_beta2;
    float lr_over_c1, rsqrt_c2, eps, decay, grad_scale;  // decay = lr weight_decay
    unsigned key;                                       // seed + step 0x9E3779B1
};

__device__ inline unsigned mix(unsigned x) {
    x ^= x >> 16;
    x *= 0x85A308D3u;
    x ^= x >> 15;
    x *= 0xA4093823u;
    return x ^ (x >> 16);
}

// a (|a| <= 448 but for rounding, or not finite) to e4m3, up or down by 16
// random bits.  From 2^-6 on the type keeps the float's upper mantissa bits:
// the random bits are added to the upper 16 of the 20 that go, and the carry
// rounds.  Below, its values are the multiples of 2^-9.
__device__ inline float round_random(float a, unsigned bits16) {
    const float mag = fabsf(a);
    const float high = __uint_as_float((__float_as_uint(mag) + (bits16 << 4)) & ~0xFFFFFu);
    const float low = floorf(mag * 512.0f + (float)bits16 * (1.0f / 65536.0f)) * (1.0f / 512.0f);
    const float q = fminf(mag >= 0.015625f ? high : low, kE4M3Max);
    return finite_f32(a) ? copysignf(q, a) : __uint_as_float(0x7fc00000u);
}

__device__ inline unsigned pack_e4m3(const float (&q)[4]) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
}
__device__ inline f32x4 unpack_e4m3(unsigned w) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

__device__ inline unsigned load_codes(const unsigned char *p, int valid) {
    if (valid >= 4) return __builtin_nontemporal_load(&((const Global<Loose<unsigned, 1>> *)p)->v);
    unsigned w = 0;
    for (int e = 0; e < valid; ++e) w |= (unsigned)((const Global<unsigned char> *)p)[e] << (8 * e);
    return w;
}
__device__ inline void store_codes(unsigned char *p, unsigned w, int valid) {
    if (valid >= 4) {
        __builtin_nontemporal_store(w, &((Global<Loose<unsigned, 1>> *)p)->v);
        return;
    }
    for (int e = 0; e < valid; ++e) ((Global<unsigned char> *)p)[e] = (unsigned char)(w >> (8 * e));
}

// The block's values over their scale, rounded at random; lane 0 has the scale.
template <bool kKeepPositive>
__device__ inline unsigned quantise(f32x4 x, const unsigned (&bits16)[4], float *scale) {
    float most = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) most = fmaxf(most, finite_abs(x[e]));
    most = wave_reduce<OpMax>(most);
    const bool fine = most > 1e-30f;
    const float up = fine ? (1.0f / most) * kE4M3Max : 0.0f;
    *scale = fine ? most * (1.0f / kE4M3Max) : 0.0f;
    float q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float a = x[e] * up;
        q[e] = round_random(a, bits16[e]);
        if (kKeepPositive && a > 0.0f && q[e] == 0.0f) q[e] = 0.001953125f;
    }
    return pack_e4m3(q);
}

template <typename P, typename G, bool kMaster, bool kEight>
__global__ __launch_bounds__(256) void adamw_kernel(const tg_adamw_tensor *__restrict__ tensors,
                                                    const ChunkOf *__restrict__ chunks, Rates r) {
    const ChunkOf c = chunks[blockIdx.x];
    const tg_adamw_tensor t = tensors[c.tensor];
    const int lane = threadIdx.x % 64;
    const int64_t base = (int64_t)c.chunk * kChunk + (threadIdx.x / 64) * (kSub * kScaleBlock);
    P *const param = (P *)t.param;
    const G *const grad = (const G *)t.grad;

    f32x4 g[kSub], w[kSub], m[kSub], v[kSub];
    unsigned mc[kSub], vc[kSub];
    float ms[kSub], vs[kSub];
    int valid[kSub];
#pragma unroll
    for (int s = 0; s < kSub; ++s) {
        const int64_t at = base + s * kScaleBlock + lane * 4;
        const int64_t left = t.n - at;
        valid[s] = left >= 4 ? 4 : left > 0 ? (int)left : 0;
        g[s] = load_f32<G, 4, true>(grad + at, valid[s]);
        w[s] = kMaster ? load_f32<float, 4, true>(t.master + at, valid[s]) : load_f32<P, 4, true>(param + at, valid[s]);
        if (kEight) {
            mc[s] = load_codes((const unsigned char *)t.m + at, valid[s]);
            vc[s] = load_codes((const unsigned char *)t.v + at, valid[s]);
            const bool any = base + s * kScaleBlock < t.n;
            const int64_t block = base / kScaleBlock + s;
            ms[s] = any ? ((const Global<float> *)t.m_scale)[block] : 0.0f;
            vs[s] = any ? ((const Global<float> *)t.v_scale)[block] : 0.0f;
        } else {
            m[s] = load_f32<float, 4, true>((const float *)t.m + at, valid[s]);
            v[s] = load_f32<float, 4, true>((const float *)t.v + at, valid[s]);
        }
    }
    const unsigned key = kEight ? mix(r.key + (unsigned)c.tensor * 0x13198A2Fu) : 0u;
#pragma unroll
    for (int s = 0; s < kSub; ++s) {
        const int64_t at = base + s * kScaleBlock + lane * 4;
        if (base + s * kScaleBlock >= t.n) return;  // whole wave
        if (kEight) {
            const f32x4 mq = unpack_e4m3(mc[s]), vq = unpack_e4m3(vc[s]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[s][e] = mq[e] * ms[s];
                const float root = vq[e] * vs[s];
                v[s][e] = root * root;
            }
        }
        f32x4 root;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float ge = g[s][e] * r.grad_scale;
            // one rounding an operation, in the formulas' order: what the random
            // bits then do to an 8-bit moment can be recomputed anywhere
            m[s][e] = r.beta1 * m[s][e] + r.one_minus_beta1 * ge;
            v[s][e] = r.beta2 * v[s][e] + r.one_minus_beta2 * ge * ge;
            root[e] = kEight ? sqrtf(v[s][e]) : __builtin_amdgcn_sqrtf(v[s][e]);
            const float step = r.lr_over_c1 * m[s][e] * __builtin_amdgcn_rcpf(fmaf(root[e], r.rsqrt_c2, r.eps));
            w[s][e] -= fmaf(r.decay, w[s][e], step);
        }
        if (kMaster) store_f32<float, 4, true>(t.master + at, w[s], valid[s]);
        store_f32<P, 4, true>(param + at, w[s], valid[s]);
        if (kEight) {
            unsigned bm[4], bv[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned bits = mix((unsigned)(at + e) + key);
                bm[e] = bits >> 16;
                bv[e] = bits & 0xFFFFu;
            }
            float m_scale, v_scale;
            const unsigned qm = quantise<false>(m[s], bm, &m_scale);
            const unsigned qv = quantise<true>(root, bv, &v_scale);
            store_codes((unsigned char *)t.m + at, qm, valid[s]);
            store_codes((unsigned char *)t.v + at, qv, valid[s]);
            if (lane == 0) {
                ((Global<float> *)t.m_scale)[base / kScaleBlock + s] = m_scale;
                ((Global<float> *)t.v_scale)[base / kScaleBlock + s] = v_scale;
            }
        } else {
            store_f32<float, 4, true>((float *)t.m + at, m[s], valid[s]);
            store_f32<float, 4, true>((float *)t.v + at, v[s], valid[s]);
        }
    }
}

using Kernel = void (*)(const tg_adamw_tensor *, const ChunkOf *, Rates);

template <typename P, typename G>
Kernel pick_state(bool master, bool eight) {
    if (master) return eight ? adamw_kernel<P, G, true, true> : adamw_kernel<P, G, true, false>;
    return eight ? adamw_kernel<P, G, false, true> : adamw_kernel<P, G, false, false>;
}
Kernel pick(int param, int grad, bool master, bool eight) {
    if (param == TG_F32)  // its own master copy
        return eight ? adamw_kernel<float, float, false, true> : adamw_kernel<float, float, false, false>;
    if (param == TG_BF16)
        return grad == TG_F32 ? pick_state<bf16, float>(master, eight) : pick_state<bf16, bf16>(master, eight);
    return grad == TG_F32 ? pick_state<f16, float>(master, eight) : pick_state<f16, f16>(master, eight);
}

}  // namespace
}  // namespace tg

struct tg_adamw {
    int device;
    void *block;  // tensors, then chunks
    const tg_adamw_tensor *tensors;
    const tg::ChunkOf *chunks;
    int64_t n_chunks;
    tg::Kernel kernel;
};

using namespace tg;

namespace {

bool aligned_to(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

tg_status check_tensor(const tg_adamw_tensor &t, int i, size_t param_size, size_t grad_size, int bits, bool master) {
    if (t.n < 0) return call_failed(TG_EINVAL, "tensor %d: n = %lld", i, (long long)t.n);
    if ((t.master != nullptr) != master && t.n > 0)
        return call_failed(TG_EINVAL, "tensor %d: master copies are for all tensors or for none", i);
    if (t.n == 0) return TG_OK;
    if (!t.param || !t.grad || !t.m || !t.v) return call_failed(TG_EINVAL, "tensor %d: a buffer is NULL", i);
    if (bits == 8 && (!t.m_scale || !t.v_scale)) return call_failed(TG_EINVAL, "tensor %d: a scale buffer is NULL", i);
    const size_t state = bits == 8 ? 1 : 4;
    if (!aligned_to(t.param, param_size) || !aligned_to(t.grad, grad_size) || !aligned_to(t.master, 4) ||
        !aligned_to(t.m, state) || !aligned_to(t.v, state) || !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4))
        return call_failed(TG_EINVAL, "tensor %d: a buffer is not aligned to its elements", i);
    return TG_OK;
}

tg_status create(const tg_adamw_tensor *tensors, int32_t n, int param_type, int grad_type, int bits, tg_adamw **out) {
    if (n < 0 || (n > 0 && !tensors)) return call_failed(TG_EINVAL, "n_tensors = %d or tensors is NULL", n);
    if (param_type != TG_F32 && param_type != TG_BF16 && param_type != TG_F16)
        return call_failed(TG_EINVAL, "param_type %d", param_type);
    if (grad_type != param_type && grad_type != TG_F32) return call_failed(TG_EINVAL, "grad_type %d", grad_type);
    if (bits != 8 && bits != 32) return call_failed(TG_EINVAL, "state_bits %d: 8 or 32", bits);
    bool master = false;
    int64_t chunks = 0;
    for (int i = 0; i < n; ++i)
        if (tensors[i].n > 0) master = master || tensors[i].master;
    if (master && param_type == TG_F32) return call_failed(TG_EINVAL, "32-bit parameters take no master copies");
    for (int i = 0; i < n; ++i) {
        const tg_status st = check_tensor(tensors[i], i, param_type == TG_F32 ? 4 : 2, grad_type == TG_F32 ? 4 : 2, bits, master);
        if (st != TG_OK) return st;
        const int64_t c = ceil_div(tensors[i].n, kChunk);
        if (c > kMostChunks - chunks) return call_failed(TG_EINVAL, "too many elements for one handle");
        chunks += c;
    }
    std::unique_ptr<tg_adamw> a(new tg_adamw());
    std::vector<ChunkOf> list;
    list.reserve(chunks);
    for (int i = 0; i < n; ++i)
        for (int64_t c = 0; c < ceil_div(tensors[i].n, kChunk); ++c) list.push_back({i, (int)c});
    hipError_t e = hipGetDevice(&a->device);
    if (e != hipSuccess) return device_failed(e, "hipGetDevice");
    a->n_chunks = chunks;
    a->kernel = pick(param_type, grad_type, master, bits == 8);
    a->block = nullptr;
    if (chunks > 0) {
        const size_t head = round256(sizeof(tg_adamw_tensor) * n), tail = sizeof(ChunkOf) * list.size();
        e = hipMalloc(&a->block, head + tail);
        if (e != hipSuccess) return device_failed(e, "the table of tensors");
        e = hipMemcpy(a->block, tensors, sizeof(tg_adamw_tensor) * n, hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipMemcpy((char *)a->block + head, list.data(), tail, hipMemcpyHostToDevice);
        if (e != hipSuccess) {
            (void)hipFree(a->block);
            return device_failed(e, "the table of tensors");
        }
        a->tensors = (const tg_adamw_tensor *)a->block;
        a->chunks = (const ChunkOf *)((const char *)a->block + head);
    }
    *out = a.release();
    return TG_OK;
}

}  // namespace

extern "C" {

tg_status tg_adamw_create(const tg_adamw_tensor *tensors, int32_t n_tensors, int32_t param_type, int32_t grad_type,
                          int32_t state_bits, tg_adamw **out) {
    if (!out) return call_failed(TG_EINVAL, "out is NULL");
    *out = nullptr;
    try {
        return create(tensors, n_tensors, param_type, grad_type, state_bits, out);
    } catch (const std::bad_alloc &) {
        return call_failed(TG_ENOMEM, "host allocation failed");
    }
}

tg_status tg_adamw_step(const tg_adamw *a, const tg_adamw_rates *rates, tg_stream stream) {
    if (!a || !rates) return call_failed(TG_EINVAL, "handle or rates is NULL");
    const tg_adamw_rates &q = *rates;
    if (q.step < 1) return call_failed(TG_EINVAL, "step %lld: steps count from 1", (long long)q.step);
    if (q.reserved) return call_failed(TG_EINVAL, "reserved must be 0");
    if (!std::isfinite(q.lr) || !std::isfinite(q.eps) || !std::isfinite(q.weight_decay) || !std::isfinite(q.grad_scale))
        return call_failed(TG_EINVAL, "a rate is not finite");
    if (!(q.beta1 >= 0 && q.beta1 < 1 && q.beta2 >= 0 && q.beta2 < 1)) return call_failed(TG_EINVAL, "a beta is outside [0, 1)");
    int cur = -1;
    hipError_t e = hipGetDevice(&cur);
    if (e != hipSuccess) return device_failed(e, "hipGetDevice");
    if (cur != a->device) return call_failed(TG_EINVAL, "device %d is current; the tensors live on device %d", cur, a->device);
    if (a->n_chunks == 0) return TG_OK;
    Rates r;
    r.beta1 = (float)q.beta1;
    r.beta2 = (float)q.beta2;
    r.one_minus_beta1 = (float)(1.0 - q.beta1);
    r.one_minus_beta2 = (float)(1.0 - q.beta2);
    r.lr_over_c1 = (float)(q.lr / (1.0 - std::pow(q.beta1, (double)q.step)));
    r.rsqrt_c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(q.beta2, (double)q.step)));
    r.eps = (float)q.eps;
    r.decay = (float)(q.lr * q.weight_decay);
    r.grad_scale = (float)q.grad_scale;
    r.key = q.seed + (uint32_t)q.step * 0x9E3779B1u;
    hipLaunchKernelGGL(a->kernel, dim3((unsigned)a->n_chunks), dim3(256), 0, (hipStream_t)stream, a->tensors, a->chunks, r);
    e = hipGetLastError();
    return e == hipSuccess ? TG_OK : device_failed(e, "adamw_kernel");
}

void tg_adamw_destroy(tg_adamw *a) {
    if (!a) return;
    int cur = 0;
    (void)hipGetDevice(&cur);
    (void)hipSetDevice(a->device);
    if (a->block) (void)hipFree(a->block);  // waits for the device
    (void)hipSetDevice(cur);
    delete a;
}

}  // extern "C"
