// layer_device.h -- what the layer operators' kernels share: element types,
// vector access at any alignment, reductions, and the error exit of api.hip.
#pragma once

#include <hip/hip_runtime.h>

#include "tangram_layer.h"

namespace tg {

// The thread's error message and the status to return (api.hip).
tg_status call_failed(tg_status st, const char *fmt, ...);
tg_status device_failed(hipError_t e, const char *what);

using bf16 = __bf16;
using f16 = _Float16;
struct e4m3 {
    unsigned char bits;
};

template <typename T, int N>
using vec = T __attribute__((ext_vector_type(N)));
using f32x4 = vec<float, 4>;
using f32x16 = vec<float, 16>;
using i32x4 = vec<int, 4>;

// Rows may start at any element, so wide accesses are made at the element's
// own alignment: gfx950 takes them in one instruction wherever they start.
template <typename V, int A>
struct __attribute__((packed, aligned(A))) Loose {
    V v;
};
template <typename T, int N>
__device__ inline vec<T, N> load_loose(const T *p) {
    return reinterpret_cast<const Loose<vec<T, N>, alignof(T)> *>(p)->v;
}
template <typename T, int N>
__device__ inline void store_loose(T *p, vec<T, N> v) {
    reinterpret_cast<Loose<vec<T, N>, alignof(T)> *>(p)->v = v;
}

// N elements of p as floats; those at or past `valid` are 0 and not read.
template <typename T, int N>
__device__ inline vec<float, N> load_f32(const T *p, int valid) {
    vec<float, N> r;
    if (valid >= N) {
        const vec<T, N> v = load_loose<T, N>(p);
#pragma unroll
        for (int e = 0; e < N; ++e) r[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) r[e] = e < valid ? (float)p[e] : 0.0f;
    }
    return r;
}
template <typename T, int N>
__device__ inline void store_f32(T *p, vec<float, N> r, int valid) {
    if (valid >= N) {
        vec<T, N> v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)r[e];
        store_loose<T, N>(p, v);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < valid) p[e] = (T)r[e];
    }
}

constexpr float kE4M3Max = 448.0f;

__device__ inline bool finite_f32(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
// |x| where x is a number below infinity, else 0.
__device__ inline float finite_abs(float x) { return finite_f32(x) ? fabsf(x) : 0.0f; }

struct OpSum {
    static __device__ float of(float a, float b) { return a + b; }
};
struct OpMax {
    static __device__ float of(float a, float b) { return fmaxf(a, b); }
};

// All lanes get the reduction over the wave, in a fixed order.
template <typename Op>
__device__ inline float wave_reduce(float x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x = Op::of(x, __shfl_xor(x, d));
    return x;
}
// All threads of a block of T get the reduction; T = 64 is the wave alone.
// `slots` holds T / 64 floats and is free again when the next use begins after
// a barrier, which the alternating halves of the callers' arrays provide.
template <typename Op, int T>
__device__ inline float block_reduce(float x, float *slots) {
    x = wave_reduce<Op>(x);
    if (T == 64) return x;
    const int wave = threadIdx.x / 64;
    if (threadIdx.x % 64 == 0) slots[wave] = x;
    __syncthreads();
    x = slots[0];
#pragma unroll
    for (int w = 1; w < T / 64; ++w) x = Op::of(x, slots[w]);
    return x;
}

// out[c] = the sum of partial[r][c] over rows r (reduce.hip: ascending r within
// eight interleaved strands, then the strands in order).
hipError_t launch_column_sums(const float *partial, int rows, int64_t cols, void *out, int type, hipStream_t s);

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace tg
