// layer_device.h -- what the layer operators' kernels share: element types,
// vector access at any alignment, reductions, and the error exit of api.hip.
#pragma once

#include <hip/hip_runtime.h>

#include "sizes.h"
#include "tangram_layer.h"

namespace tg {

// The thread's error message and the status to return (api.hip).
tg_status call_failed(tg_status st, const char *fmt, ...);
tg_status device_failed(hipError_t e, const char *what);

#define TG_TRY(call)                  \
    do {                              \
        const tg_status st_ = (call); \
        if (st_ != TG_OK) return st_; \
    } while (0)

inline size_t size_of(int type) { return type == TG_F32 ? 4 : type == TG_E4M3 ? 1 : 2; }

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
// Operands lie in device memory, which the compiler does not know of addresses
// that come out of a table.
template <typename T>
using Global = __attribute__((address_space(1))) T;

// kOnce: what is read or written once in a pass much larger than the caches need
// not stay in them.
template <typename T, int N, bool kOnce = false>
__device__ inline vec<T, N> load_loose(const T *p) {
    const auto *const at = &((const Global<Loose<vec<T, N>, alignof(T)>> *)p)->v;
    return kOnce ? __builtin_nontemporal_load(at) : *at;
}
template <typename T, int N, bool kOnce = false>
__device__ inline void store_loose(T *p, vec<T, N> v) {
    auto *const at = &((Global<Loose<vec<T, N>, alignof(T)>> *)p)->v;
    if (kOnce)
        __builtin_nontemporal_store(v, at);
    else
        *at = v;
}

// N elements of p; those at or past `valid` are 0 and not read.
template <typename T, int N>
__device__ inline vec<T, N> load_part(const T *p, int valid) {
    if (valid >= N) return load_loose<T, N>(p);
    vec<T, N> r;
    const Global<T> *const g = (const Global<T> *)p;
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = e < valid ? g[e] : (T)0.0f;
    return r;
}
// The same as floats.
template <typename T, int N, bool kOnce = false>
__device__ inline vec<float, N> load_f32(const T *p, int valid) {
    vec<float, N> r;
    if (valid >= N) {
        const vec<T, N> v = load_loose<T, N, kOnce>(p);
#pragma unroll
        for (int e = 0; e < N; ++e) r[e] = (float)v[e];
    } else {
        const Global<T> *const g = (const Global<T> *)p;
#pragma unroll
        for (int e = 0; e < N; ++e) r[e] = e < valid ? (float)g[e] : 0.0f;
    }
    return r;
}
template <typename T, int N, bool kOnce = false>
__device__ inline void store_f32(T *p, vec<float, N> r, int valid) {
    if (valid >= N) {
        vec<T, N> v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)r[e];
        store_loose<T, N, kOnce>(p, v);
    } else {
        Global<T> *const g = (Global<T> *)p;
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < valid) g[e] = (T)r[e];
    }
}

constexpr float kE4M3Max = 448.0f;
constexpr float kLeastScale = 0x1p-126f;  // of an 8-bit output: the least normal number

template <typename E>
constexpr int kUnitOf = 16 / sizeof(E);  // elements in 16 bytes

// 16 bytes of a row as they lie; elements at or past `valid` are 0 and not read.
template <typename E>
__device__ inline i32x4 load_bits(const E *p, int valid) {
    if (valid >= kUnitOf<E>) return ((const Global<Loose<i32x4, alignof(E)>> *)p)->v;
    i32x4 r(0);
#pragma unroll
    for (int e = 0; e < kUnitOf<E>; ++e) {
        if (e >= valid) continue;
        if constexpr (sizeof(E) == 4)
            r[e] = ((const Global<int> *)p)[e];
        else
            r[e / 2] |= (int)((unsigned)((const Global<unsigned short> *)p)[e] << (16 * (e % 2)));
    }
    return r;
}
// The same of a row's unit at `col` in one load: of a last unit that is not whole the
// row's last 16 bytes, for in_place to move down when they are used.  With a load and
// a branch for each element of it the layer norm of 16384 x 1605 in f16 took 81 us
// forward and 119 backward, so 41 and 57.
template <typename E>
__device__ inline i32x4 load_unit(const E *row, int col, int valid) {
    constexpr int kUnit = kUnitOf<E>;
    if (valid <= 0) return i32x4(0);
    if (col == 0 && valid < kUnit) return load_bits<E>(row, valid);
    return ((const Global<Loose<i32x4, alignof(E)>> *)(row + col + std::min(valid, kUnit) - kUnit))->v;
}
template <typename E>
__device__ inline void in_place(i32x4 &r, int col, int valid) {
    if (valid <= 0 || valid >= kUnitOf<E> || col == 0) return;
    const int bits = (kUnitOf<E> - valid) * (int)sizeof(E) * 8;
    if (bits & 64) r = i32x4{r[2], r[3], 0, 0};
    if (bits & 32) r = i32x4{r[1], r[2], r[3], 0};
    if (sizeof(E) == 2 && (bits & 16)) {
#pragma unroll
        for (int w = 0; w < 4; ++w) r[w] = (int)((unsigned)r[w] >> 16 | (w < 3 ? (unsigned)r[w + 1] << 16 : 0));
    }
}
template <typename E>
__device__ inline vec<float, kUnitOf<E>> floats(i32x4 bits) {
    return __builtin_convertvector(__builtin_bit_cast(vec<E, kUnitOf<E>>, bits), vec<float, kUnitOf<E>>);
}

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

__device__ inline bool finite_f32(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
// |x| where x is a number below infinity, else 0.
__device__ inline float finite_abs(float x) { return finite_f32(x) ? fabsf(x) : 0.0f; }

struct OpSum {
    static __device__ float of(float a, float b) { return a + b; }
};
struct OpMax {
    static __device__ float of(float a, float b) { return fmaxf(a, b); }
};

// All lanes get the reduction over the wave, in a fixed order: within rows of 16
// lanes by their data-parallel moves, then across rows by swapping them.
template <int kMove>
__device__ inline float moved(float x) {
    return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), kMove, 0xf, 0xf, true));
}
template <typename Op>
__device__ inline float wave_reduce(float x) {
    x = Op::of(x, moved<0xB1>(x));   // neighbours
    x = Op::of(x, moved<0x4E>(x));   // pairs of four
    x = Op::of(x, moved<0x141>(x));  // fours of eight, mirrored
    x = Op::of(x, moved<0x140>(x));  // eights of sixteen, mirrored
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = Op::of(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return Op::of(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
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

// One block's share of the sums over a table's rows: 32 columns from col0 on, by 256
// threads.  Strand g of eight adds rows g, g + 8, ..., then the strands are added in
// order: in place of float atomics, so that the result is the same every time.
template <typename T>
__device__ inline void column_sums_block(const float *__restrict__ partial, int rows, int64_t cols, int64_t col0, T *out) {
    __shared__ float strand[8][33];
    const int lane = threadIdx.x % 32, g = threadIdx.x / 32;
    const int64_t col = col0 + lane;
    float sum = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (int r = g; r < rows; r += 8) sum += partial[r * cols + col];
    }
    strand[g][lane] = sum;
    __syncthreads();
    if (g == 0 && col < cols) {
#pragma unroll
        for (int h = 1; h < 8; ++h) sum += strand[h][lane];
        out[col] = (T)sum;
    }
}

// out[c] = the sum of partial[r][c] over rows r (reduce.hip: ascending r within
// eight interleaved strands, then the strands in order).
hipError_t launch_column_sums(const float *partial, int rows, int64_t cols, void *out, int type, hipStream_t s);
// The same of two tables, one behind the other; an output that is NULL is left out.
hipError_t launch_column_sums_of_two(const float *partial, int rows, int64_t cols, void *out, void *out2, int type, hipStream_t s);

}  // namespace tg
