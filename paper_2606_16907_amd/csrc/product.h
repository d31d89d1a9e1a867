// product.h -- the matrix products of the layer operators: tiles, kernels, epilogues
// and what chooses among them (included by linear.hip, gated.hip and block_linear.hip,
// which each compile the forms that they call).
//
// All products are C[i][j] = sum over r of P(i, r) Q(j, r), written row by row.  In
// some, two matrices take the place of one (Form).
#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "layer_device.h"
#include "linear_cut.h"

namespace tg {
namespace {

// ---------------------------------------------------------------------------
// tiles of an operand in LDS and the fragments of the matrix instructions
// ---------------------------------------------------------------------------
// A tile holds kStepBytes (128) of r for each of its rows (or columns).  With r along
// the rows ("along") it is [rows][128 bytes], and the 16-byte units of a row are
// permuted by the row, unit ^ (row / 2 & 7), so that 16 rows of one unit fill
// the 64 banks once: even rows one half of them, odd rows the other.  With r down
// the columns ("down", 16-bit types) it is [64 r][columns], read through the
// transposing LDS load, and the 32-byte units of a row are permuted by the row's
// bits 0, 1 and 3, the ones in which the rows of one load differ.
__device__ inline int along_at(int row, int unit) { return row * kStepBytes + ((unit ^ ((row >> 1) & 7)) << 4); }
__device__ inline int down_bits(int r) { return (r & 3) | ((r >> 1) & 4); }

// The wave's number, known to the compiler to be the same in all its lanes.
__device__ inline int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }

// 16 x 16 matrix instructions: a lane holds 8 elements of row lane % 16.
template <typename T>
struct Matrix;
template <>
struct Matrix<bf16> {
    using frag = vec<bf16, 8>;
    static __device__ f32x4 mma(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Matrix<f16> {
    using frag = vec<f16, 8>;
    static __device__ f32x4 mma(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// Products with one matrix in every place, and those that do two matrices' work:
//   kGated   Q is two matrices of as many rows, side by side in every tile; C is
//            act(gate) up of their products
//   kSeam    r goes through two matrices: up to `seam` Q is the first of them, from
//            there on the second; each has `half` rows, the rest of r is zeros in P
//   kHalves  C's rows up to `seam` go to one output and those from there on to
//            another, the first `half` of each
//   kBlocks, kExponents  one matrix in every place, of e4m3 with scales for blocks of
//            128 of r: floats, or exponents of powers of two
enum Form { kOne, kGated, kSeam, kHalves, kBlocks, kExponents };

// ---------------------------------------------------------------------------
// epilogue
// ---------------------------------------------------------------------------
struct Epilogue {
    const float *x_scale, *w_scale;
    const void *bias, *residual;
    void *out, *pre;
    int64_t ldr, ldo, ldp;
    int act;
    // Sums over shares of r.  Where all of C is shared out (kOne, product_few): [splits, ni,
    // nj], of kGated [splits, ni, 2 nj], up's columns behind gate's, which join_kernel
    // finishes; NULL: finished at once.  After a tail cut: [tile of the tail][share], each a
    // whole tile row by row, of kGated gate's half of a row and then up's, for join_body.
    float *partial;
    // the second matrix's (kHalves: out)
    const float *w_scale2;
    const void *bias2;
    void *out2, *pre2;
    int64_t ldo2, ldp2;
    int64_t seam, half;
};

__device__ inline float exp_f32(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// The normal distribution function from exp(-z^2 / 2), which its caller may need
// too.  Below 0 it is bell erfcx(|z| / sqrt 2) / 2, and that quotient is t P(t) with
// t = 1 / (1 + 0.265 |z|): P of degree 6 was fitted to it by least squares, weighted
// until its largest relative error up to |z| = 14.5 was least.  In 32 bits it is off by 1e-6
// of its value, so gelu keeps its relative accuracy where it is small.
__device__ inline float normal_cdf(float z, float bell) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.265f, fabsf(z), 1.0f));
    float p = fmaf(t, -0.067787044f, 0.19527312f);
    p = fmaf(t, p, -0.06636293f);
    p = fmaf(t, p, 0.14249334f);
    p = fmaf(t, p, 0.08294658f);
    p = fmaf(t, p, 0.10783678f);
    p = fmaf(t, p, 0.105599836f);
    const float tail = bell * t * p;
    return z >= 0.0f ? 1.0f - tail : tail;
}

// The activation, or its slope, of N values.
template <int N>
__device__ inline void activate(vec<float, N> &z, int act) {
    if (act == TG_ACT_RELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) z[c] = z[c] < 0.0f ? 0.0f : z[c];  // NaN stays
    } else if (act == TG_ACT_SILU) {
#pragma unroll
        for (int c = 0; c < N; ++c) z[c] *= __builtin_amdgcn_rcpf(1.0f + exp_f32(-z[c]));
    } else if (act == TG_ACT_GELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) z[c] *= normal_cdf(z[c], exp_f32(-0.5f * z[c] * z[c]));
    }
}
// z comes in 16 bits, where one that was finite may be an infinity.  At |z| = 128
// the slopes of silu and gelu are 0 and 1 in 32 bits, so z is held there; NaN stays.
__device__ inline float held(float z) { return fabsf(z) > 128.0f ? copysignf(128.0f, z) : z; }
template <int N>
__device__ inline vec<float, N> slope(vec<float, N> z, int act) {
    if (act == TG_ACT_SILU || act == TG_ACT_GELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) z[c] = held(z[c]);
    }
    if (act == TG_ACT_RELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) z[c] = z[c] > 0.0f ? 1.0f : 0.0f;
    } else if (act == TG_ACT_SILU) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const float t = __builtin_amdgcn_rcpf(1.0f + exp_f32(-z[c]));
            z[c] = t * fmaf(z[c], 1.0f - t, 1.0f);
        }
    } else if (act == TG_ACT_GELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const float bell = exp_f32(-0.5f * z[c] * z[c]);
            z[c] = fmaf(z[c] * 0.39894228f, bell, normal_cdf(z[c], bell));
        }
    }
    return z;
}

// N columns from j on of row i, from the sums z and what the row's and the columns'
// operands are: sx the row's scale, sw the columns', `residual` theirs.
template <int N>
struct Columns {
    vec<float, N> sw, bias;
};
template <typename O, int N>
__device__ inline Columns<N> load_columns(int64_t j, int valid, const Epilogue &e) {
    Columns<N> c{vec<float, N>(1.0f), vec<float, N>(0.0f)};
    if (e.w_scale) c.sw = load_f32<float, N>(e.w_scale + j, valid);
    if (e.bias) c.bias = load_f32<O, N>((const O *)e.bias + j, valid);
    return c;
}
template <typename O, int N>
__device__ inline void finish(vec<float, N> z, float sx, const Columns<N> &c, vec<float, N> residual, int64_t i, int64_t j, int valid,
                              const Epilogue &e) {
    if (e.x_scale) z = z * sx * c.sw;
    z += c.bias;
    if (e.pre) store_f32<O, N>((O *)e.pre + i * e.ldp + j, z, valid);
    activate<N>(z, e.act);
    if (e.residual) z += residual;
    store_f32<O, N>((O *)e.out + i * e.ldo + j, z, valid);
}
// kGated: from the sums of both matrices.
template <typename O, int N>
__device__ inline Columns<N> load_columns_up(int64_t j, int valid, const Epilogue &e) {
    Columns<N> c{vec<float, N>(1.0f), vec<float, N>(0.0f)};
    if (e.w_scale2) c.sw = load_f32<float, N>(e.w_scale2 + j, valid);
    if (e.bias2) c.bias = load_f32<O, N>((const O *)e.bias2 + j, valid);
    return c;
}
template <typename O, int N>
__device__ inline void finish_gated(vec<float, N> gate, vec<float, N> up, float sx, const Columns<N> &cg, const Columns<N> &cu, int64_t i, int64_t j,
                                    int valid, const Epilogue &e) {
    if (e.x_scale) gate = gate * sx * cg.sw, up = up * sx * cu.sw;
    gate += cg.bias, up += cu.bias;
    if (e.pre) {
        store_f32<O, N>((O *)e.pre + i * e.ldp + j, gate, valid);
        store_f32<O, N>((O *)e.pre2 + i * e.ldp2 + j, up, valid);
    }
    activate<N>(gate, e.act);
    store_f32<O, N>((O *)e.out + i * e.ldo + j, gate * up, valid);
}
template <typename O, int N>
__device__ inline void finish_gated(vec<float, N> gate, vec<float, N> up, int64_t i, int64_t j, int valid, const Epilogue &e) {
    finish_gated<O, N>(gate, up, e.x_scale ? e.x_scale[i] : 1.0f, load_columns<O, N>(j, valid, e), load_columns_up<O, N>(j, valid, e), i, j, valid, e);
}
// kHalves: the sums are the result.
template <typename O, int N>
__device__ inline void finish_halves(vec<float, N> z, int64_t i, int64_t j, int valid, const Epilogue &e) {
    const bool second = i >= e.seam;
    const int64_t row = second ? i - e.seam : i;
    if (row < e.half) store_f32<O, N>((second ? (O *)e.out2 + row * e.ldo2 : (O *)e.out + row * e.ldo) + j, z, valid);
}
template <typename O, int N>
__device__ inline void finish(vec<float, N> z, int64_t i, int64_t j, int valid, const Epilogue &e) {
    vec<float, N> residual(0.0f);
    if (e.residual) residual = load_f32<O, N>((const O *)e.residual + i * e.ldr + j, valid);
    finish<O, N>(z, e.x_scale ? e.x_scale[i] : 1.0f, load_columns<O, N>(j, valid, e), residual, i, j, valid, e);
}

// ---------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------
struct Product {
    const void *p, *q;
    int64_t ldp, ldq;     // elements
    int64_t ni, nj, nr;   // rows and columns of C, length of the sums
    const void *q2;       // kGated, kSeam: Q's second matrix
    int64_t ldq2;
    int64_t seam, half;   // kSeam: of r
    const void *ps, *qs;  // kBlocks, kExponents: scales [ni, blocks] and [ceil(nj / 128), blocks]
    int64_t ldps, ldqs;
};

constexpr int kScaled = 128;  // elements of r, and rows of Q, that share a scale
// 2^(code - 127), NaN for code 255.
__device__ inline float power_of(unsigned code) {
    return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7fc00000u : code << 23);
}
// The scales of blocks b .. b + 3 of a row, in one load: powers of two a byte at a time
// took 19.1 us for one row through 14336 x 4096, so 14.9, as floats do; and of block b.
template <bool kPowers>
__device__ inline f32x4 load_scales(const void *row, int64_t b) {
    f32x4 s;
    if constexpr (kPowers) {
        const unsigned codes = ((const Global<Loose<unsigned, 1>> *)((const unsigned char *)row + b))->v;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = power_of(codes >> 8 * e & 255);
    } else {
        s = ((const Global<Loose<f32x4, 4>> *)((const float *)row + b))->v;
    }
    return s;
}
template <bool kPowers>
__device__ inline float load_scale(const void *row, int64_t b) {
    if constexpr (kPowers)
        return power_of(((const Global<unsigned char> *)row)[b]);
    else
        return ((const Global<float> *)row)[b];
}

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
    // The same for a row of `row` elements that ends there, valid being 0 or less past its
    // end: read up to that end, with what lies before the unit, and shifted.
    static __device__ raw load_last(const T *p, int64_t valid, int64_t row) {
        if (row < 8) return load(p, valid);
        const int cut = valid < 8 ? 8 - (int)valid : 0, bits = (cut < 8 ? cut : 0) * 8 * (int)sizeof(T);
        raw r = reinterpret_cast<const Loose<raw, alignof(T)> *>(p - cut)->v;
        uint64_t words[sizeof(T)];
        __builtin_memcpy(words, &r, sizeof(r));
        if constexpr (sizeof(T) == 1) {
            words[0] >>= bits;
        } else {
            const uint64_t low = bits >= 64 ? words[1] : words[0], high = bits >= 64 ? 0 : words[1];
            const int rest = bits % 64;
            words[0] = low >> rest | (high << 1) << (63 - rest);
            words[1] = high >> rest;
        }
#pragma unroll
        for (int w = 0; w < (int)sizeof(T); ++w) words[w] = cut < 8 ? words[w] : 0;
        __builtin_memcpy(&r, words, sizeof(r));
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

// ---------------------------------------------------------------------------
// the product for operands whose rows start at 16-byte addresses
// ---------------------------------------------------------------------------
// Bound by the matrix units and, at the largest sizes, by power.  Tiles go from
// memory to LDS without passing through registers; bytes past an operand's end
// arrive as zeros, which is how rows, columns and sums that end inside a tile are
// handled.  LDS holds two tiles of P and three of Q: while one is read the next are
// on their way, loads spread over the whole step.  A step's r is multiplied in two
// halves, and the fragments of a half are read while the half before is
// multiplied, across steps too, so the matrix instructions wait at one barrier a
// step, which stands between the halves: there every wave has read all of the
// step's tiles, whose places later ones take, and the next have arrived.  Four
// waves of 128 x 128 read a step's tiles twice, P and Q alike; eight of 128 x 64
// would read P four times.  8192^3 in bf16 takes 780 to 880 us in every order of
// the operands (1250 to 1420 TFLOP/s; this card's library products 680 to 800 for x w^T,
// 780 to 900 for dz w and 920 to 1020 for dz^T x), in 8 bits 379 (2900); leaving out
// the loads saves 12% of that, the reads 13%: what remains is the matrix
// instructions at the 1.4 to 1.8 GHz that the power allows.
template <typename T>
struct Wide;  // 32 x 32 matrix instructions: kDeep of them over half a step's r
template <>
struct Wide<bf16> {
    static constexpr int kDeep = 2;
    using frag = vec<bf16, 8>;
    static __device__ f32x16 mma(frag a, frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Wide<f16> {
    static constexpr int kDeep = 2;
    using frag = vec<f16, 8>;
    static __device__ f32x16 mma(frag a, frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
// The 8-bit instruction aligns groups of eight products to the largest of them
// and cuts each off, towards 0, at 2^-13 of the power of two in it (measured: beside
// 448 * 448 - 448 * 448 in its group a product of 7 is lost and one of 8 stays),
// then adds in 32 bits.  Over random products that comes to 1e-5 of the result, a
// hundredth of what rounding y to 16 bits costs, and is twice the speed of bf16.
template <>
struct Wide<e4m3> {
    static constexpr int kDeep = 1;
    using frag = vec<int, 8>;
    static __device__ f32x16 mma(frag a, frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
    }
};

// Where a lane reads its parts of an operand's tile.  A part's byte is a lane's
// own offset, of which there are four (the wave's rows or columns begin at a
// multiple of 64, so the permutations leave the rest alone), plus a number the
// compiler knows: the reads need no arithmetic.
// From its 32 rows number kGapAt on a wave reads kGap rows further down.
template <typename T, bool kDown, int kWidth, int kGapAt = 64, int kGap = 0>
struct Reader {
    using frag = typename Wide<T>::frag;
    int lane_at[4];  // in the operand's first tile
    int from[2][4];  // in the tile of this step and of the next (constants reach 2^16 bytes only)
    // The wave's rows (columns) begin at w0, the operand's first tile `begin` bytes into LDS.
    __device__ void init(int w0, int begin) {
        const int lane = threadIdx.x % 64;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if constexpr (kDown) {  // by the 32 columns; rows of r are constants
                const int r = (lane / 32) * 8 + (lane % 16) / 4;
                lane_at[c] = begin + r * kWidth * 2 + (((w0 / 16 + 2 * c + (lane / 16) % 2) ^ down_bits(r)) << 5) + (lane % 4) * 8;
            } else {  // by the pair of units
                lane_at[c] = begin + along_at(w0 + lane % 32, 2 * c + lane / 32);
            }
        }
    }
    // From now on `set` reads the tile `offset` bytes after the first.
    __device__ void aim(int set, int offset) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            from[set][c] = lane_at[c] + offset;
            asm volatile("" : "+v"(from[set][c]));  // a register of its own, not an addition at every read
        }
    }
    // Rows (columns) 32 n .. 32 n + 31 of the wave, instruction d of half `half`.
    template <int set, int half, int d, int n>
    __device__ frag read(const char *lds) const {
        constexpr int kRowAt = (n * 32 + (n >= kGapAt ? kGap : 0)) * kStepBytes;
        if constexpr (sizeof(T) == 1) {
            const i32x4 lo = *(const i32x4 *)(lds + from[set][half * 2] + kRowAt);
            const i32x4 hi = *(const i32x4 *)(lds + from[set][half * 2 + 1] + kRowAt);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else if constexpr (!kDown) {
            return *(const frag *)(lds + from[set][half * 2 + d] + kRowAt);
        } else {
            using s16x4 = vec<short, 4>;
            using s16x8 = vec<short, 8>;
            s16x4 part[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // rows of r 4 on: bit 2, which the permutation does not see
                const char *const at = lds + from[set][n] + (half * 32 + d * 16 + 4 * h) * kWidth * 2;
                part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
            }
            return __builtin_bit_cast(frag, (s16x8)__builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// A block's share of one operand on its way to LDS: each wave moves kLoads KB a
// tile, lane l the 16 bytes at l * 16 of each, from offsets that stay the same
// relative to the step's first byte.
// kSeam: down the columns, its rows of r go on in a second matrix.
template <typename T, bool kDown, int kWidth, bool kTwo = false, int kWaves = 4>
struct Stream {
    static constexpr int kLoads = kWidth * kStepBytes / 1024 / kWaves;
    static constexpr int kRowBytes = kDown ? kWidth * 2 : kStepBytes;
    int at[kLoads];
    int unit;        // along: bytes of the step's r before the lane's unit, in even loads; odd ones are half a row on
    const char *base;      // of step 0
    int64_t left;          // bytes from there to the operand's end
    int64_t step;          // bytes from one step to the next
    int64_t r_bytes_left;  // along: bytes of r from there on
    i32x4 d;               // the step's buffer descriptor
    const char *base2;     // of the second matrix's first row, which begins step `seam`
    int64_t left2;
    int seam;

    // rows0: rows of the tile that lie before this wave's matrix
    __device__ void init(const void *p, int64_t ld, int64_t at0, int64_t n_at, int64_t r0, int64_t nr, int64_t r_bytes, int rows0 = 0) {
        const int wave = wave_index(), lane = threadIdx.x % 64;
        const int64_t row_bytes = ld * (int64_t)sizeof(T);
        if constexpr (kDown) {
            base = (const char *)p + r0 * row_bytes + at0 * 2;
            // the last row may end inside a 4-byte word, which is read whole or not at all
            left = (nr - r0 - 1) * row_bytes + ((n_at - at0) * 2 + 3) / 4 * 4;
            step = 64 * row_bytes;
            unit = 0;
            r_bytes_left = 0;
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                const int place = (wave * kLoads + n) * 1024 + lane * 16, r = place / kRowBytes, b = place % kRowBytes;
                at[n] = (int)(r * row_bytes) + ((((b >> 5) ^ down_bits(r)) << 5) | (b & 16));
            }
        } else {
            base = (const char *)p + at0 * row_bytes + r0 * (int64_t)sizeof(T);
            left = (n_at - at0 - 1) * row_bytes + r_bytes - r0 * (int64_t)sizeof(T);
            step = kStepBytes;
            unit = ((lane % 8) ^ (lane / 16)) * 16;
            r_bytes_left = r_bytes - r0 * (int64_t)sizeof(T);
#pragma unroll
            for (int n = 0; n < kLoads; ++n) at[n] = (int)(((wave * kLoads + n) * 8 - rows0 + lane / 8) * row_bytes) + (unit ^ n % 2 * 64);
        }
    }
    // After init with the first matrix's `half` rows as nr: rows from r = seam_r on
    // are the second's, of the same row stride.
    __device__ void join(const void *p2, int64_t ld, int64_t at0, int64_t n_at, int64_t r0, int64_t seam_r, int64_t half) {
        static_assert(kDown, "r goes down the columns");
        const int64_t row_bytes = ld * (int64_t)sizeof(T);
        base2 = (const char *)p2 + at0 * 2;
        left2 = (half - 1) * row_bytes + ((n_at - at0) * 2 + 3) / 4 * 4;
        seam = (int)((seam_r - r0) / 64);
    }
    // The buffer descriptor of step h: loads past the operand's end give zeros, and
    // so do offsets of 2^31 and more, which the lanes get whose unit lies past the
    // row's end (and keep: later steps lie past it as a whole).
    __device__ void open(int h) {
        const bool second = kTwo && h >= seam;
        if (second) h -= seam;
        const int64_t left_h = (second ? left2 : left) - h * step;
        if (!kDown) {
            const int64_t r_left = r_bytes_left - h * step;
            const int outside[2] = {unit >= r_left ? (int)0x80000000 : 0, (unit ^ 64) >= r_left ? (int)0x80000000 : 0};
#pragma unroll
            for (int n = 0; n < kLoads; ++n) at[n] |= outside[n % 2];
        }
        const uint64_t from = (uint64_t)(second ? base2 : base) + h * step;
        d[0] = __builtin_amdgcn_readfirstlane((int)from);
        d[1] = __builtin_amdgcn_readfirstlane((int)(from >> 32) & 0xffff);
        d[2] = __builtin_amdgcn_readfirstlane((int)(left_h < 0 ? 0 : left_h > 0x7ffffff0 ? 0x7ffffff0 : left_h));
        d[3] = 0x00027000;
    }
    // The next step's, while two whole steps at least follow it: no row and no unit
    // ends in it that did not end before, so only the address moves.  Rows past the
    // last (along) begin past the first step's end too; columns past the last
    // (down) are the beginnings of rows that exist.
    __device__ void advance() {
        const uint64_t from = ((uint64_t)(unsigned)d[1] << 32 | (unsigned)d[0]) + (uint64_t)step;
        d[0] = (int)from;
        d[1] = (int)(from >> 32);
    }
    // A scalar register that a vector instruction wrote may be read by a load five
    // cycles later; the compiler counts them for its own loads only.
    __device__ void settle() { asm volatile("s_nop 4" : "+s"(d)); }
    // Starts load n of the step's tile, `tile` bytes into LDS.  As an instruction of
    // its own, since the compiler would make every later read of LDS wait for it;
    // the loop's waits are written out instead.  It has no output registers.  The
    // pause is for m0, which belongs to no one between instructions.
    template <int n>
    __device__ void load(unsigned tile) const {
        asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :
                     : "s"(tile), "v"(at[n]), "s"(d), "n"(n * 1024)
                     : "memory", "scc");
    }
};

// Block b's tile.  Blocks go to the eight XCDs in turn, so each XCD gets a run of
// consecutive tiles, and runs go down eight rows of tiles before they move on a
// column: the tiles that an L2 serves at one time share rows and columns.
__device__ inline void tile_of(int64_t b, int ti, int tj, int *i, int *j) {
    const int total = ti * tj, share = total / 8, rest = total % 8;
    const int xcd = (int)(b % 8), turn = (int)(b / 8);
    const int id = xcd * share + (xcd < rest ? xcd : rest) + turn;
    constexpr int kGroup = 8;
    const int group = id / (kGroup * tj), in = id % (kGroup * tj);
    const int high = ti - group * kGroup < kGroup ? ti - group * kGroup : kGroup;
    *i = group * kGroup + in % high;
    *j = in / high;
}

// What block b of a tail cut does: its tile, its share of r, and where a share's sums
// go, tile by tile.
struct TailBlock {
    int tile, share;
    bool split;
    int64_t part;  // of the sums, tiles of them
};
__device__ inline TailBlock tail_block(int64_t b, int64_t whole, int64_t tiles, int splits) {
    if (b < whole || splits == 1) return {(int)b, 0, false, 0};
    const int64_t x = b - whole, tail = tiles - whole;
    return {(int)(whole + x % tail), (int)(x / tail), true, x % tail * splits + x / tail};
}

// f(kFrom), ..., f(kTo - 1) with the numbers known to the compiler.
template <int kFrom, int kTo, typename F>
__device__ inline void each(F f) {
    if constexpr (kFrom < kTo) {
        f(std::integral_constant<int, kFrom>{});
        each<kFrom + 1, kTo>(f);
    }
}
// How many of `of` things are to come before slot n, spread evenly over `slots`.
constexpr int share(int n, int slots, int of) { return n >= slots ? of : (n * of + slots - 1) / slots; }

template <int kTI, int kTJ>
constexpr int kPlace = (2 * 64 * kTI + 3 * 64 * kTJ) * kStepBytes;

// 64 kTI x 64 kTJ of C by four waves of 32 kTI x 32 kTJ, in kPlace bytes of LDS.
//   kGated: two of the waves bring rows of one matrix and two of the other, and each
// wave multiplies half its share of Q's tile from one and half from the other, so a
// lane's sums are of gate and up for the same rows and columns.
template <typename T, typename O, bool kDownP, bool kDownQ, int kTI, int kTJ, Form kForm>
__device__ __forceinline__ void product_body(char *tiles, const TailBlock &block, const Product &a, const Epilogue &e, int tiles_i, int tiles_j,
                                             int64_t r_bytes_p, int64_t r_bytes_q, int share_steps) {
    constexpr int kBI = 64 * kTI, kBJ = 64 * kTJ;
    constexpr bool kPair = kForm == kGated;
    constexpr int kDeep = Wide<T>::kDeep;
    constexpr int64_t kStep = kStepBytes / sizeof(T);
    constexpr int kTileP = kBI * kStepBytes, kTileQ = kBJ * kStepBytes;
    using frag = typename Wide<T>::frag;
    int bi, bj;
    tile_of(block.tile, tiles_i, tiles_j, &bi, &bj);
    const int64_t i0 = (int64_t)bi * kBI, j0 = (int64_t)bj * (kPair ? kBJ / 2 : kBJ);
    const int wave = wave_index(), lane = threadIdx.x % 64;
    const int wi = (wave / 2) * 32 * kTI, wj = (wave % 2) * (kPair ? 16 : 32) * kTJ;  // in C's tile

    Stream<T, kDownP, kBI> sp;
    Stream<T, kDownQ, kBJ, kForm == kSeam> sq;
    Reader<T, kDownP, kBI> rp;
    Reader<T, kDownQ, kBJ, kPair ? kTJ / 2 : 64, 16 * kTJ> rq;
    // this block's share of r: all of it where there are no splits
    const int64_t r0 = (int64_t)block.share * share_steps * kStep, r1 = block.split ? std::min<int64_t>(a.nr, r0 + share_steps * kStep) : a.nr;
    sp.init(a.p, a.ldp, i0, a.ni, r0, r1, r1 < a.nr ? r1 * (int64_t)sizeof(T) : r_bytes_p);
    if constexpr (kForm == kSeam) {
        sq.init(a.q, a.ldq, j0, a.nj, r0, a.half, r_bytes_q);
        sq.join(a.q2, a.ldq, j0, a.nj, r0, a.seam, a.half);
    } else {
        const bool second = kPair && wave >= 2;
        sq.init(second ? a.q2 : a.q, second ? a.ldq2 : a.ldq, j0, a.nj, r0, r1, r1 < a.nr ? r1 * (int64_t)sizeof(T) : r_bytes_q, second ? kBJ / 2 : 0);
    }
    rp.init(wi, 0);
    rq.init(wj, 2 * kTileP);
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)&tiles[0];
    const unsigned to_p = lds + wave * sp.kLoads * 1024, to_q = lds + 2 * kTileP + wave * sq.kLoads * 1024;
    f32x16 acc[kTI][kTJ] = {};
    frag p[2][kDeep][kTI], q[2][kDeep][kTJ];
    // Fragment f and matrix instruction n of a half, in the order of use.
    constexpr int kFrags = kDeep * (kTI + kTJ), kMma = kDeep * kTI * kTJ;
    const auto read = [&](auto set, auto half, auto f) {
        constexpr int d = f / (kTI + kTJ), n = f % (kTI + kTJ);
        if constexpr (n < kTJ)
            q[half][d][n] = rq.template read<set, half, d, n>(&tiles[0]);
        else
            p[half][d][n - kTJ] = rp.template read<set, half, d, n - kTJ>(&tiles[0]);
    };
    const auto multiply = [&](auto half, auto n) {
        constexpr int d = n / (kTI * kTJ), x = n / kTJ % kTI, y = n % kTJ;
        acc[x][y] = Wide<T>::mma(q[half][d][y], p[half][d][x], acc[x][y]);
        __builtin_amdgcn_sched_barrier(0);  // the order is as written
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};
    // The barrier comes before the last kTail instructions of the first half, so
    // that they keep the matrix unit busy while the waves meet.  From there to the
    // next one P's tile of step t + 2 is loaded first and Q's of step t + 3 after it,
    // which the next barrier does not wait for.  A slot is the gap before a matrix
    // instruction, and little may stand in it: there is one wave to a SIMD, any
    // instruction takes it some 4 cycles, a matrix instruction 32.
    constexpr int kTail = kMma / 8, kReadSlots = kMma * 5 / 8, kSlotsP = (kMma + kTail) / 2, kSlotsQ = kMma + kTail - kSlotsP;
    static_assert(kReadSlots + 2 <= kMma - kTail, "the descriptors are made between the reads and the barrier");
    // Step t, whose tiles of P and Q are in places `now` and `place`; `inner`: steps
    // t + 2 and t + 3 are ones that advance() may reach.
    const auto step = [&](auto now, auto inner, int t, int place) {
        const int after = place == 2 ? 0 : place + 1;
        each<0, kMma - kTail>([&](auto n) {
            each<share(n, kReadSlots, kFrags), share(n + 1, kReadSlots, kFrags)>([&](auto f) { read(now, second, f); });
            if constexpr (n == 0) rq.aim(1 - now, after * kTileQ);
            if constexpr (n == kReadSlots) inner ? sp.advance() : sp.open(t + 2);
            if constexpr (n == kReadSlots + 1) inner ? sq.advance() : sq.open(t + 3);
            multiply(first, n);
        });
        if constexpr (!inner) sp.settle(), sq.settle();
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(sq.kLoads) : "memory");
        const auto load = [&](auto slot) {
            each<share(slot, kSlotsP, sp.kLoads), share(slot + 1, kSlotsP, sp.kLoads)>([&](auto l) { sp.template load<l>(to_p + now * kTileP); });
            if constexpr (slot >= kSlotsP)
                each<share(slot - kSlotsP, kSlotsQ, sq.kLoads), share(slot - kSlotsP + 1, kSlotsQ, sq.kLoads)>(
                    [&](auto l) { sq.template load<l>(to_q + place * kTileQ); });
        };
        each<kMma - kTail, kMma>([&](auto n) {
            load(std::integral_constant<int, n - kMma + kTail>{});
            multiply(first, n);
        });
        each<0, kMma>([&](auto n) {
            each<share(n, kReadSlots, kFrags), share(n + 1, kReadSlots, kFrags)>([&](auto f) { read(std::integral_constant<int, 1 - now>{}, first, f); });
            load(std::integral_constant<int, n + kTail>{});
            multiply(second, n);
        });
        return after;
    };
    // loads past the end of r give zeros, so two steps at a time are right for any number
    const int steps = (int)((r1 - r0 + kStep - 1) / kStep), whole = (int)((r1 - r0) / kStep);
    if (steps > 0) {
        const auto load_p = [&](auto h) {
            sp.open(h), sp.settle();
            each<0, sp.kLoads>([&](auto l) { sp.template load<l>(to_p + h * kTileP); });
        };
        const auto load_q = [&](auto h) {
            sq.open(h), sq.settle();
            each<0, sq.kLoads>([&](auto l) { sq.template load<l>(to_q + h * kTileQ); });
        };
        load_p(first), load_q(first);
        load_p(second), load_q(second);
        load_q(std::integral_constant<int, 2>{});
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(sp.kLoads + 2 * sq.kLoads) : "memory");
        rp.aim(0, 0), rp.aim(1, kTileP), rq.aim(0, 0);
        each<0, kFrags>([&](auto f) { read(first, first, f); });
        int t = 0, place = 0;
        const auto steady = [&](int stop) {
            for (; t + 6 < stop; t += 2) {
                place = step(first, std::true_type{}, t, place);
                place = step(second, std::true_type{}, t + 1, place);
            }
        };
        const auto careful = [&](int stop) {
            for (; t < stop; t += 2) {
                place = step(first, std::false_type{}, t, place);
                place = step(second, std::false_type{}, t + 1, place);
            }
        };
        if constexpr (kForm == kSeam) {  // advance() does not pass from one matrix to the other
            while (t < steps) {
                const bool before = t < sq.seam && sq.seam < whole;
                steady(before ? sq.seam : whole);
                careful(before ? sq.seam : steps);
            }
        } else {
            steady(whole);
            careful(steps);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // the last loads, before this LDS has another use
    }
    // A lane has columns 8 (c / 4) + 4 (lane / 32) + c % 4 of row lane % 32 of
    // each 32 x 32 part.  32 rows at a time go through the wave's share of LDS, in
    // rows 16 bytes longer than their values so that the rows of a column meet
    // different banks, and come back 8 columns a lane, whole rows side by side.
    // The residual's units and the rows' scales of the next 32 rows are on their way
    // meanwhile, and wait beside the sums: the loop over a lane's units is not
    // unrolled, so that the activations' code stays small.
    __syncthreads();
    constexpr int kRow = 32 * kTJ + 4, kUnits = 2 * kTJ, kShare = 32 * kRow * 4 + 32 * 32 * kTJ * 2 + 128;
    static_assert(4 * kShare <= kPlace<kTI, kTJ>, "the waves' shares fit the tiles' place");
    float *const rows = (float *)(&tiles[0] + wave * kShare);
    // where a share's sums go, row by row of the tile
    float *const part = kForm != kOne && block.split ? e.partial + block.part * kBI * kBJ : nullptr;
    if constexpr (kPair) {  // gate's 16 kTJ columns first in a row, then up's
        constexpr int kTurns = kTJ, kAcross = 2 * kTJ;
        float *const x_scales = rows + 32 * kRow;
        const int col = lane % kAcross * 8;
        const int64_t j = j0 + wj + col;
        const int valid = (int)std::min<int64_t>(8, a.nj - j);
        Columns<8> gates{}, ups{};
        if (!part && valid > 0) gates = load_columns<O, 8>(j, valid, e), ups = load_columns_up<O, 8>(j, valid, e);
#pragma unroll
        for (int x = 0; x < kTI; ++x) {
#pragma unroll
            for (int y = 0; y < kTJ; ++y) {
#pragma unroll
                for (int c = 0; c < 16; c += 4) {
                    const f32x16 v = acc[x][y];
                    *(f32x4 *)(rows + (lane % 32) * kRow + y * 32 + 2 * c + (lane / 32) * 4) = f32x4{v[c], v[c + 1], v[c + 2], v[c + 3]};
                }
            }
            if (e.x_scale && lane < 32) {
                const int64_t i = i0 + wi + x * 32 + lane;
                x_scales[lane] = i < a.ni ? e.x_scale[i] : 1.0f;
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll 1
            for (int n = 0; n < kTurns; ++n) {
                const int row = n * (64 / kAcross) + lane / kAcross;
                const int64_t i = i0 + wi + x * 32 + row;
                if (i >= a.ni || valid <= 0) continue;
                const float *const at = rows + row * kRow + col;
                const f32x4 g0 = *(const f32x4 *)at, g1 = *(const f32x4 *)(at + 4);
                const f32x4 u0 = *(const f32x4 *)(at + 16 * kTJ), u1 = *(const f32x4 *)(at + 16 * kTJ + 4);
                const vec<float, 8> gate = __builtin_shufflevector(g0, g1, 0, 1, 2, 3, 4, 5, 6, 7);
                const vec<float, 8> up = __builtin_shufflevector(u0, u1, 0, 1, 2, 3, 4, 5, 6, 7);
                if (part) {
                    float *const to = part + (i - i0) * kBJ + (j - j0);
                    store_f32<float, 8>(to, gate, valid);
                    store_f32<float, 8>(to + kBJ / 2, up, valid);
                } else {
                    finish_gated<O, 8>(gate, up, e.x_scale ? x_scales[row] : 1.0f, gates, ups, i, j, valid, e);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        return;
    }
    vec<O, 8> *const kept = (vec<O, 8> *)(rows + 32 * kRow);
    float *const scales = (float *)(kept + 32 * 4 * kTJ);
    const int col = lane % (4 * kTJ) * 8;  // the same in all of a lane's units
    const int64_t j = j0 + wj + col;
    const int valid = (int)std::min<int64_t>(8, a.nj - j);
    Columns<8> columns{};
    vec<O, 8> fetched[kUnits];
    float scale = 1.0f;
    const auto row_of = [&](int x, int n) { return i0 + wi + x * 32 + n * (64 / (4 * kTJ)) + lane / (4 * kTJ); };
    const auto fetch = [&](int x) {
        if (e.residual) {
#pragma unroll
            for (int n = 0; n < kUnits; ++n) {
                const int64_t i = row_of(x, n);
                fetched[n] = load_part<O, 8>((const O *)e.residual + i * e.ldr + j, i < a.ni ? valid : 0);
            }
        }
        const int64_t i = i0 + wi + x * 32 + lane % 32;
        if (e.x_scale) scale = i < a.ni ? e.x_scale[i] : 1.0f;
    };
    const bool finished = kForm == kOne ? !e.partial : !part;
    if (finished) {
        if (valid > 0) columns = load_columns<O, 8>(j, valid, e);
        fetch(0);
    }
#pragma unroll
    for (int x = 0; x < kTI; ++x) {
#pragma unroll
        for (int y = 0; y < kTJ; ++y) {
#pragma unroll
            for (int c = 0; c < 16; c += 4) {
                const f32x16 v = acc[x][y];
                *(f32x4 *)(rows + (lane % 32) * kRow + y * 32 + 2 * c + (lane / 32) * 4) = f32x4{v[c], v[c + 1], v[c + 2], v[c + 3]};
            }
        }
        if (finished) {
            if (e.residual) {
#pragma unroll
                for (int n = 0; n < kUnits; ++n) kept[n * 64 + lane] = fetched[n];
            }
            if (e.x_scale && lane < 32) scales[lane] = scale;
            if (x + 1 < kTI) fetch(x + 1);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int n = 0; n < kUnits; ++n) {
            const int64_t i = row_of(x, n);
            if (i >= a.ni || valid <= 0) continue;
            const int row = (int)(i - i0 - wi) - x * 32;
            const f32x4 lo = *(const f32x4 *)(rows + row * kRow + col), hi = *(const f32x4 *)(rows + row * kRow + col + 4);
            const vec<float, 8> z = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            if (kForm == kOne && e.partial) {
                store_f32<float, 8>(e.partial + (blockIdx.y * a.ni + i) * a.nj + j, z, valid);
                continue;
            }
            if constexpr (kForm != kOne) {
                if (part) {
                    store_f32<float, 8>(part + (i - i0) * kBJ + (j - j0), z, valid);
                    continue;
                }
            }
            if constexpr (kForm == kHalves) {
                finish_halves<O, 8>(z, i, j, valid, e);
                continue;
            }
            vec<float, 8> residual(0.0f);
            if (e.residual) residual = __builtin_convertvector(kept[n * 64 + lane], vec<float, 8>);
            finish<O, 8>(z, e.x_scale ? scales[row] : 1.0f, columns, residual, i, j, valid, e);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T, typename O, bool kDownP, bool kDownQ, int kTI, int kTJ, Form kForm = kOne>
__global__ __launch_bounds__(256, kTI * kTJ > 4 ? 1 : 2) void product_direct(Product a, Epilogue e, int tiles_i, int tiles_j, int64_t r_bytes_p,
                                                                             int64_t r_bytes_q, int share_steps, int whole_tiles, int splits) {
    __shared__ __attribute__((aligned(1024))) char tiles[kPlace<kTI, kTJ>];
    // kOne: every tile in gridDim.y shares; else a tail cut
    const TailBlock block = kForm == kOne ? TailBlock{(int)blockIdx.x, (int)blockIdx.y, true, 0}
                                          : tail_block(blockIdx.x, whole_tiles, (int64_t)tiles_i * tiles_j, splits);
    product_body<T, O, kDownP, kDownQ, kTI, kTJ, kForm>(tiles, block, a, e, tiles_i, tiles_j, r_bytes_p, r_bytes_q, share_steps);
}

// ---------------------------------------------------------------------------
// x w^T for a few rows of x
// ---------------------------------------------------------------------------
// Bound by reading w once.  A block has 16 rows of w and all rows of x, 16 kRows
// of them; its eight waves take turns at r, 512 bytes of each row of w a turn, and
// add up their sums through LDS: one row through 4096 x 14336 in bf16 takes 23.5
// us, 5.0 TB/s (256 bytes a turn 25.2; the library's product 27.3), in 8 bits 16.2,
// and eight rows 17.9.  Operands go from memory to registers, so
// rows may start anywhere; rows past an operand's end repeat its last, and what comes
// of them is dropped.  8-bit operands become bf16, which is exact and costs
// nothing that shows.
//   kGated: eight of the rows are of one matrix and eight of the other.
constexpr int kFewWaves = 8, kTurnBytes = 512;
template <typename T, typename O, int kRows, Form kForm = kOne>
__global__ __launch_bounds__(512) void product_few(Product a, Epilogue e, int64_t share_turns) {
    using C = std::conditional_t<sizeof(T) == 1, bf16, T>;
    using frag = typename Matrix<C>::frag;
    using raw = typename Unit<T>::raw;
    constexpr int kWaves = kFewWaves, kUnits = kTurnBytes / sizeof(T) / 32;  // of 8 elements, of a lane in a turn
    constexpr int kTurn = kTurnBytes / sizeof(T);                            // elements of r in a turn
    __shared__ f32x4 sums[kWaves][kRows][64];
    const int wave = wave_index(), lane = threadIdx.x % 64;
    constexpr bool kPair = kForm == kGated;
    const int64_t n0 = (int64_t)blockIdx.x * (kPair ? 8 : 16);
    const bool second = kPair && lane % 16 >= 8;
    const T *const w = (const T *)(second ? a.q2 : a.q) + std::min<int64_t>(n0 + lane % (kPair ? 8 : 16), a.nj - 1) * (second ? a.ldq2 : a.ldq);
    const T *x[kRows];
#pragma unroll
    for (int m = 0; m < kRows; ++m) x[m] = (const T *)a.p + std::min<int64_t>(m * 16 + lane % 16, a.ni - 1) * a.ldp;
    f32x4 acc[kRows] = {};
    // Unit u of a lane: 8-bit units lie in pairs, so that a lane reads 16 bytes.
    const auto at = [&](int u) { return sizeof(T) == 1 ? (u / 2) * 64 + (lane / 16) * 16 + u % 2 * 8 : u * 32 + (lane / 16) * 8; };
    // With scales: a block's sum, of four units of each lane, is added when it is whole.
    constexpr bool kScales = kForm == kBlocks || kForm == kExponents;
    constexpr int kScaleSize = kForm == kExponents ? 1 : 4;
    const char *const w_scales = (const char *)a.qs + n0 / kScaled * a.ldqs * kScaleSize;
    const char *x_scales[kRows];
#pragma unroll
    for (int m = 0; m < kRows; ++m) x_scales[m] = (const char *)a.ps + std::min<int64_t>(m * 16 + lane % 16, a.ni - 1) * a.ldps * kScaleSize;
    const auto multiply = [&](int64_t turn, const raw (&uw)[kUnits], const raw (&ux)[kRows][kUnits]) {
        if constexpr (kScales) {
            static_assert(kTurn == 4 * kScaled, "four blocks a turn");
            const f32x4 sw = load_scales<kForm == kExponents>(w_scales, turn * 4);
            f32x4 s[kRows];
#pragma unroll
            for (int m = 0; m < kRows; ++m) s[m] = load_scales<kForm == kExponents>(x_scales[m], turn * 4) * sw;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                f32x4 part[kRows] = {};
#pragma unroll
                for (int u = 4 * b; u < 4 * b + 4; ++u) {
                    const frag fw = __builtin_bit_cast(frag, widened(uw[u]));
#pragma unroll
                    for (int m = 0; m < kRows; ++m) part[m] = Matrix<C>::mma(fw, __builtin_bit_cast(frag, widened(ux[m][u])), part[m]);
                }
#pragma unroll
                for (int m = 0; m < kRows; ++m) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[m][c] = fmaf(part[m][c], s[m][b], acc[m][c]);
                }
            }
            return;
        }
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const frag fw = __builtin_bit_cast(frag, widened(uw[u]));
#pragma unroll
            for (int m = 0; m < kRows; ++m) acc[m] = Matrix<C>::mma(fw, __builtin_bit_cast(frag, widened(ux[m][u])), acc[m]);
        }
    };
    // this block's share of the turns, whole ones but for the last of all
    const int64_t begin = blockIdx.y * share_turns, whole = a.nr / kTurn, end = std::min(whole, begin + share_turns);
    for (int64_t turn = begin + wave; turn < end; turn += kWaves) {
        raw uw[kUnits], ux[kRows][kUnits];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) uw[u] = Unit<T>::load(w + turn * kTurn + at(u), 8);
#pragma unroll
        for (int m = 0; m < kRows; ++m)
#pragma unroll
            for (int u = 0; u < kUnits; ++u) ux[m][u] = Unit<T>::load(x[m] + turn * kTurn + at(u), 8);
        multiply(turn, uw, ux);
    }
    const bool last = whole * kTurn < a.nr && blockIdx.y + 1 == gridDim.y;  // the turn that the row's end cuts
    if constexpr (kForm == kOne) {
        if (last && wave == (whole - begin) % kWaves) {
            raw uw[kUnits], ux[kRows][kUnits];
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                const int64_t r = whole * kTurn + at(u);
                uw[u] = Unit<T>::load(w + r, a.nr - r);
#pragma unroll
                for (int m = 0; m < kRows; ++m) ux[m][u] = Unit<T>::load(x[m] + r, a.nr - r);
            }
            multiply(whole, uw, ux);
        }
    } else if (last) {  // its units in turn among the waves: 1040 e4m3 elements, one row through 26558, take 15 us, by one wave 31
#pragma unroll
        for (int n = 0; n < kUnits / kWaves; ++n) {
            const int u = wave + n * kWaves;
            const int64_t r = whole * kTurn + at(u);
            if (whole * kTurn + at(u) - at(0) >= a.nr) continue;
            const raw uw = Unit<T>::load_last(w + r, a.nr - r, a.nr);
            raw ux[kRows];
#pragma unroll
            for (int m = 0; m < kRows; ++m) ux[m] = Unit<T>::load_last(x[m] + r, a.nr - r, a.nr);
            const frag fw = __builtin_bit_cast(frag, widened(uw));
#pragma unroll
            for (int m = 0; m < kRows; ++m) {
                if constexpr (kScales) {
                    const int64_t b = whole * 4 + u / 4;
                    const f32x4 part = Matrix<C>::mma(fw, __builtin_bit_cast(frag, widened(ux[m])), f32x4(0.0f));
                    const float s = load_scale<kForm == kExponents>(x_scales[m], b) * load_scale<kForm == kExponents>(w_scales, b);
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[m][c] = fmaf(part[c], s, acc[m][c]);
                } else {
                    acc[m] = Matrix<C>::mma(fw, __builtin_bit_cast(frag, widened(ux[m])), acc[m]);
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < kRows; ++m) sums[wave][m][lane] = acc[m];
    __syncthreads();
    if constexpr (kPair) {  // the second half of the lanes has up for the first half's columns
        for (int u = threadIdx.x; u < kRows * 32; u += 512) {
            f32x4 z[2];
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                z[o] = sums[0][u / 32][u % 32 + 32 * o];
#pragma unroll
                for (int h = 1; h < kWaves; ++h) z[o] += sums[h][u / 32][u % 32 + 32 * o];
            }
            const int64_t i = u / 32 * 16 + u % 16, j = n0 + u % 32 / 16 * 4;
            if (i >= a.ni || j >= a.nj) continue;
            const int valid = (int)std::min<int64_t>(4, a.nj - j);
            if (e.partial) {
                float *const to = e.partial + (blockIdx.y * a.ni + i) * (2 * a.nj) + j;
                store_f32<float, 4>(to, z[0], valid);
                store_f32<float, 4>(to + a.nj, z[1], valid);
            } else {
                finish_gated<O, 4>(z[0], z[1], i, j, valid, e);
            }
        }
        return;
    }
    // lane l of part m has columns 4 (l / 16) .. + 3 of row 16 m + l % 16
    for (int u = threadIdx.x; u < kRows * 64; u += 512) {
        f32x4 z = sums[0][u / 64][u % 64];
#pragma unroll
        for (int h = 1; h < kWaves; ++h) z += sums[h][u / 64][u % 64];
        const int64_t i = u / 64 * 16 + u % 16, j = n0 + u % 64 / 16 * 4;
        if (i >= a.ni || j >= a.nj) continue;
        const int valid = (int)std::min<int64_t>(4, a.nj - j);
        if (e.partial)
            store_f32<float, 4>(e.partial + (blockIdx.y * a.ni + i) * a.nj + j, z, valid);
        else
            finish<O, 4>(z, i, j, valid, e);
    }
}

// Adds the shares of r in their order and finishes, 8 columns a thread.
template <typename O, Form kForm = kOne>
__global__ __launch_bounds__(256) void join_kernel(Epilogue e, int splits, int64_t ni, int64_t nj) {
    const int64_t units = (nj + 7) / 8, u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= ni * units) return;
    const int64_t i = u / units, j = u % units * 8;
    const int valid = (int)std::min<int64_t>(8, nj - j);
    const int64_t ld = kForm == kGated ? 2 * nj : nj;
    const auto sum = [&](int64_t column) {
        vec<float, 8> z = load_f32<float, 8>(e.partial + i * ld + column, valid);
        for (int s = 1; s < splits; ++s) z += load_f32<float, 8>(e.partial + (s * ni + i) * ld + column, valid);
        return z;
    };
    if constexpr (kForm == kGated)
        finish_gated<O, 8>(sum(j), sum(nj + j), i, j, valid, e);
    else
        finish<O, 8>(sum(j), i, j, valid, e);
}

// The same after a tail cut: 8 columns of a tile a thread, kTile^2 / 2048 blocks a
// tile (of gated ones half as many).
template <typename O, Form kForm, int kTile>
__device__ inline void join_body(int block, const Epilogue &e, int whole, int splits, int tiles_i, int tiles_j, int64_t ni, int64_t nj) {
    constexpr int kColumns = kForm == kGated ? kTile / 2 : kTile, kUnits = kColumns / 8, kPerTile = kTile * kUnits / 256;
    const int tile = block / kPerTile, u = block % kPerTile * 256 + threadIdx.x, row = u / kUnits, col = u % kUnits * 8;
    int bi, bj;
    tile_of(whole + tile, tiles_i, tiles_j, &bi, &bj);
    const int64_t i = (int64_t)bi * kTile + row, j = (int64_t)bj * kColumns + col;
    if (i >= ni || j >= nj) return;
    const int valid = (int)std::min<int64_t>(8, nj - j);
    const float *const from = e.partial + (int64_t)tile * splits * kTile * kTile + row * kTile + col;
    const auto sum = [&](int column) {
        vec<float, 8> z = load_f32<float, 8>(from + column, 8);
        for (int s = 1; s < splits; ++s) z += load_f32<float, 8>(from + column + (int64_t)s * kTile * kTile, 8);
        return z;
    };
    if constexpr (kForm == kGated)
        finish_gated<O, 8>(sum(0), sum(kTile / 2), i, j, valid, e);
    else if constexpr (kForm == kHalves)
        finish_halves<O, 8>(sum(0), i, j, valid, e);
    else
        finish<O, 8>(sum(0), i, j, valid, e);
}
template <typename O, Form kForm, int kTile>
__global__ __launch_bounds__(256) void join_tiles(Epilogue e, int whole, int splits, int tiles_i, int tiles_j, int64_t ni, int64_t nj) {
    join_body<O, kForm, kTile>(blockIdx.x, e, whole, splits, tiles_i, tiles_j, ni, nj);
}
template <Form kForm>
unsigned join_blocks(const TailCut &c) {
    return c.splits == 1 ? 0 : (unsigned)(c.tail * (c.tile * c.tile / 2048) / (kForm == kGated ? 2 : 1));
}
template <typename O, Form kForm>
hipError_t join_tail(const Product &a, const Epilogue &e, const TailCut &c, int ti, int tj, hipStream_t s) {
    const hipError_t r = hipGetLastError();
    if (r != hipSuccess || c.splits == 1) return r;
    const dim3 grid(join_blocks<kForm>(c));
    if (c.tile == 256)
        hipLaunchKernelGGL((join_tiles<O, kForm, 256>), grid, dim3(256), 0, s, e, c.whole, c.splits, ti, tj, a.ni, a.nj);
    else
        hipLaunchKernelGGL((join_tiles<O, kForm, 128>), grid, dim3(256), 0, s, e, c.whole, c.splits, ti, tj, a.ni, a.nj);
    return hipGetLastError();
}

constexpr int64_t kMostLd = 1 << 21;  // elements of a row of a product's operands

inline size_t cut_bytes(const Cut &c, int64_t ni, int64_t nj) { return c.splits > 1 ? round256((size_t)c.splits * ni * nj * 4) : 0; }

// Rows into rows that start at 16-byte addresses and end in zeros on a whole unit
// of 16 bytes, for one operand, two or three.  Bound by memory, 4 TB/s read and written
// together; reading unaligned rows in the product itself took 2.5 to 4.7 us a
// step of 128 tiles where aligned ones take 0.65 to 1.05.
struct Packing {
    const void *from[3];
    void *to[3];
    int64_t rows[3], cols[3], ld[3], ld_to[3];  // rows 0: none
};
template <typename T>
__device__ inline void pack_body(const Packing &a, int o, int64_t block, int64_t blocks) {
    constexpr int kN = 16 / sizeof(T);
    const int64_t units = a.ld_to[o] / kN, all = a.rows[o] * units;
    for (int64_t u = block * 256 + threadIdx.x; u < all; u += blocks * 256) {
        const int64_t row = u / units, col = u % units * kN;
        const T *const from = (const T *)a.from[o] + row * a.ld[o] + col;
        vec<T, kN> v;
        if (a.cols[o] - col >= kN) {
            v = load_loose<T, kN>(from);
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) v[e] = col + e < a.cols[o] ? from[e] : (T)0;
        }
        *(vec<T, kN> *)((T *)a.to[o] + row * a.ld_to[o] + col) = v;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(Packing a) {
    pack_body<T>(a, blockIdx.y, blockIdx.x, gridDim.x);
}
// Operand o of a packing: `cols` columns of each of `rows` rows, which are the packed ones from now on.
inline void pack_operand(Packing &k, int o, const void *&from, int64_t &ld, int64_t rows, int64_t cols, int size, char *to) {
    k.from[o] = from, k.to[o] = to, k.ld[o] = ld;
    k.rows[o] = rows, k.cols[o] = cols;
    k.ld_to[o] = ld = ceil_div(cols * size, 16) * 16 / size;
    from = to;
}

// Whether operand rows start at 16-byte addresses, an operand with r along its
// rows ends on a whole unit (`r_bytes` of each row may be read), and a tile's
// offsets fit 31 bits.
inline bool streams(const void *p, int64_t ld, int size, int64_t r_bytes, bool down) {
    return (uintptr_t)p % 16 == 0 && ld * size % 16 == 0 && (down || r_bytes % 16 == 0) && ld < kMostLd;
}
inline int64_t whole_ld(int64_t cols, int size) { return ceil_div(cols * size, 16) * 16 / size; }

// How a product of one call is done (kOne, kGated, kBlocks and kExponents): the kernel,
// the operands that are packed first, and what lies where in the workspace: packed P,
// packed Q (both of its matrices), shares.
struct Plan {
    bool few, pack_p, pack_q;
    Cut cut;       // kOne, and `few`
    TailCut tail;  // the other forms
    size_t p_bytes, q_bytes, bytes;
};
// What a step of a form takes, of one in 16 bits: 0.63 us with 256 tiles of gated 8-bit
// operands and 112 steps each, 0.72 with scales that are powers of two and 0.89 with
// floats, where 16 bits take 0.58.
template <Form kForm>
constexpr double pace_of(int size) { return kForm == kBlocks ? 1.4 : kForm == kExponents ? 1.25 : size == 1 ? 1.1 : 1.0; }
template <Form kForm = kOne>
Plan plan_product(const Product &a, int size, int64_t r_bytes_p, bool down_p, bool down_q) {
    Plan p{};
    if (a.ni == 0 || a.nj == 0) return p;
    constexpr bool kPair = kForm == kGated;
    const int64_t columns = kPair ? 2 * a.nj : a.nj;  // of the sums
    p.pack_p = !streams(a.p, a.ldp, size, r_bytes_p, down_p);
    p.pack_q = !streams(a.q, a.ldq, size, a.nr * size, down_q) || (kPair && !streams(a.q2, a.ldq2, size, a.nr * size, down_q));
    // From some 8 rows on tiles of 128 and splits are as fast with one weight: 4096 x
    // 14336 in bf16, 25 us for one row against 28, 28 for both at 8, 34 against 28 at
    // 16.  Where an operand would have to be packed, up to 64 rows.
    const bool packs = p.pack_p || p.pack_q;
    int64_t most_few = packs ? 64 : 8;
    if (kForm != kOne) {
        const auto words = [&](const void *q, int64_t ld) { return ((uintptr_t)q | (uintptr_t)(ld * size)) % 4 == 0; };
        most_few = packs ? few_packed_rows(columns, a.nr * size, words(a.p, a.ldp) && words(a.q, a.ldq) && (!kPair || words(a.q2, a.ldq2)))
                         : few_rows(columns, a.nr * size);
    }
    p.few = !down_p && !down_q && a.ni <= most_few;
    if (p.few) {
        // Few rows of w leave most of the chip idle: sums of 40 turns and more are
        // shared out among blocks then, a turn a wave at least.  4 rows through 689 x
        // 10803, whose rows are not aligned, take 23.5 us in one share and 12.8 in
        // five, one through 1024 x 14336 18.6 and 13.2; through 1024 x 8192 11.5 and
        // 13.4, which is another launch.
        const int64_t blocks = ceil_div(columns, 16), turns = a.nr * size / kTurnBytes;
        const int64_t most = blocks < 128 && turns >= 40 ? std::min<int64_t>(8, ceil_div(256, blocks)) : 1;
        p.cut.splits = (int)std::max<int64_t>(1, std::min(most, turns / kFewWaves));
        p.cut.share = (int)ceil_div(std::max<int64_t>(1, turns), p.cut.splits);
        p.cut.splits = (int)std::max<int64_t>(1, ceil_div(turns, p.cut.share));
        p.bytes = cut_bytes(p.cut, a.ni, columns);
        return p;
    }
    if constexpr (kForm == kOne)
        p.cut = cut_product(a.ni, columns, a.nr, size);
    else
        p.tail = cut_tail(a.ni, columns, a.nr, size, false, pace_of<kForm>(size));
    const auto packed = [&](int64_t n, int64_t r, bool down) { return round256(down ? r * whole_ld(n, size) * size : n * whole_ld(r, size) * size); };
    p.p_bytes = p.pack_p ? packed(a.ni, a.nr, down_p) : 0;
    p.q_bytes = p.pack_q ? packed(a.nj, a.nr, down_q) * (kPair ? 2 : 1) : 0;
    p.bytes = p.p_bytes + p.q_bytes + (kForm == kOne ? cut_bytes(p.cut, a.ni, columns) : round256(p.tail.bytes()));
    return p;
}

// After a product's launch: its error, or the launch that adds up its shares.
template <typename O, Form kForm>
hipError_t join(const Product &a, const Epilogue &e, int splits, hipStream_t s) {
    const hipError_t r = hipGetLastError();
    if (r != hipSuccess || !e.partial) return r;
    hipLaunchKernelGGL((join_kernel<O, kForm>), dim3((unsigned)ceil_div(a.ni * ceil_div(a.nj, 8), 256)), dim3(256), 0, s, e, splits, a.ni, a.nj);
    return hipGetLastError();
}

// The operands that the plan packs, into the workspace; `a` and the bytes of r that
// may be read of P's rows are then the packed ones'.
template <typename T, Form kForm, bool kDownP, bool kDownQ>
hipError_t pack_operands(Product &a, const Plan &p, int64_t &r_bytes_p, char *ws, hipStream_t s) {
    constexpr int kSize = sizeof(T);
    constexpr bool kPair = kForm == kGated;
    if (!(p.pack_p || p.pack_q) || a.nr == 0) return hipSuccess;
    Packing k{};
    const auto pack = [&](int o, const void *&from, int64_t &ld, int64_t n, int64_t r, bool down, char *to) {
        pack_operand(k, o, from, ld, down ? r : n, down ? n : r, kSize, to);
    };
    if (p.pack_p) pack(0, a.p, a.ldp, a.ni, a.nr, kDownP, ws), r_bytes_p = a.ldp * kSize;
    if (p.pack_q) pack(1, a.q, a.ldq, a.nj, a.nr, kDownQ, ws + p.p_bytes);
    if (p.pack_q && kPair) pack(2, a.q2, a.ldq2, a.nj, a.nr, kDownQ, ws + p.p_bytes + p.q_bytes / 2);
    const int64_t units = std::max({k.rows[0] * k.ld_to[0], k.rows[1] * k.ld_to[1], k.rows[2] * k.ld_to[2]}) * kSize / 16;
    using Moved = std::conditional_t<kSize == 1, unsigned char, T>;
    const dim3 grid((unsigned)std::min<int64_t>(2048, ceil_div(units, 256)), kPair ? 3 : 2);
    hipLaunchKernelGGL(pack_kernel<Moved>, grid, dim3(256), 0, s, k);
    return hipGetLastError();
}

// A product that the plan gives to product_few.
template <typename T, typename O, Form kForm>
hipError_t launch_few(const Product &a, Epilogue e, const Plan &p, char *ws, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div(a.nj, kForm == kGated ? 8 : 16), p.cut.splits);
    e.partial = p.cut.splits > 1 ? (float *)ws : nullptr;
    switch ((a.ni + 15) / 16) {
        case 1: hipLaunchKernelGGL((product_few<T, O, 1, kForm>), grid, dim3(512), 0, s, a, e, p.cut.share); break;
        case 2: hipLaunchKernelGGL((product_few<T, O, 2, kForm>), grid, dim3(512), 0, s, a, e, p.cut.share); break;
        case 3: hipLaunchKernelGGL((product_few<T, O, 3, kForm>), grid, dim3(512), 0, s, a, e, p.cut.share); break;
        default: hipLaunchKernelGGL((product_few<T, O, 4, kForm>), grid, dim3(512), 0, s, a, e, p.cut.share);
    }
    return join<O, kForm>(a, e, p.cut.splits, s);
}

// C in a tail cut's tiles, from operands that may be streamed; the cut's bytes are at `sums`.
template <typename T, typename O, bool kDownP, bool kDownQ, Form kForm>
hipError_t launch_tiles(const Product &a, Epilogue e, int64_t r_bytes_p, int64_t r_bytes_q, const TailCut &c, float *sums, hipStream_t s) {
    if (a.ni == 0 || a.nj == 0) return hipSuccess;
    e.seam = a.seam, e.half = a.half;
    e.partial = sums;
    const int ti = (int)ceil_div(a.ni, c.tile), tj = (int)ceil_div(a.nj, kForm == kGated ? c.tile / 2 : c.tile);
    const dim3 grid((unsigned)(c.whole + c.tail * c.splits));
    if (c.tile == 256)
        hipLaunchKernelGGL((product_direct<T, O, kDownP, kDownQ, 4, 4, kForm>), grid, dim3(256), 0, s, a, e, ti, tj, r_bytes_p, r_bytes_q, c.share, c.whole, c.splits);
    else
        hipLaunchKernelGGL((product_direct<T, O, kDownP, kDownQ, 2, 2, kForm>), grid, dim3(256), 0, s, a, e, ti, tj, r_bytes_p, r_bytes_q, c.share, c.whole, c.splits);
    return join_tail<O, kForm>(a, e, c, ti, tj, s);
}

// C; `ws` holds the plan's bytes.
template <typename T, typename O, bool kDownP, bool kDownQ, Form kForm = kOne>
hipError_t launch_product(Product a, Epilogue e, int64_t r_bytes_p, char *ws, hipStream_t s) {
    constexpr int kSize = sizeof(T);
    if (a.ni == 0 || a.nj == 0) return hipSuccess;
    const Plan p = plan_product<kForm>(a, kSize, r_bytes_p, kDownP, kDownQ);
    if constexpr (!kDownP && !kDownQ) {
        if (p.few) return launch_few<T, O, kForm>(a, e, p, ws, s);
    }
    const hipError_t r = pack_operands<T, kForm, kDownP, kDownQ>(a, p, r_bytes_p, ws, s);
    if (r != hipSuccess) return r;
    const int64_t r_bytes_q = p.pack_q ? a.ldq * kSize : a.nr * kSize;
    float *const sums = (float *)(ws + p.p_bytes + p.q_bytes);
    if constexpr (kForm == kOne) {
        const Cut &c = p.cut;
        const int ti = (int)ceil_div(a.ni, c.tile), tj = (int)ceil_div(a.nj, c.tile);
        e.partial = c.splits > 1 ? sums : nullptr;
        if (c.tile == 256)
            hipLaunchKernelGGL((product_direct<T, O, kDownP, kDownQ, 4, 4>), dim3(ti * tj, c.splits), dim3(256), 0, s, a, e, ti, tj, r_bytes_p, r_bytes_q, c.share, 0, c.splits);
        else
            hipLaunchKernelGGL((product_direct<T, O, kDownP, kDownQ, 2, 2>), dim3(ti * tj, c.splits), dim3(256), 0, s, a, e, ti, tj, r_bytes_p, r_bytes_q, c.share, 0, c.splits);
        return join<O, kForm>(a, e, c.splits, s);
    } else {
        return launch_tiles<T, O, kDownP, kDownQ, kForm>(a, e, r_bytes_p, r_bytes_q, p.tail, sums, s);
    }
}

// ---------------------------------------------------------------------------
// checks and sizes on the host
// ---------------------------------------------------------------------------
inline tg_status check_matrix(const void *p, int64_t ld, int64_t rows, int64_t cols, int type, const char *what) {
    if (rows == 0 || cols == 0) return TG_OK;
    if (!p) return call_failed(TG_EINVAL, "%s is NULL", what);
    if ((uintptr_t)p % size_of(type)) return call_failed(TG_EINVAL, "%s is not aligned to its elements", what);
    if (rows > 1 && ld < cols)
        return call_failed(TG_EINVAL, "%s: row stride %lld below the row length %lld", what, (long long)ld, (long long)cols);
    return TG_OK;
}

inline tg_status check_workspace(const void *ws, size_t bytes, size_t need) {
    if ((uintptr_t)ws % 256) return call_failed(TG_EINVAL, "the workspace is not 256-byte aligned");
    if (need && (!ws || bytes < need)) return call_failed(TG_ENOMEM, "workspace of %zu bytes, %zu needed", ws ? bytes : 0, need);
    return TG_OK;
}

inline bool sizes_fit(int64_t m, int64_t n, int64_t k) {
    const int64_t most = kMostLd - 64;
    return m >= 0 && n >= 0 && k >= 0 && m <= 0x7fffffff - 256 && n <= most && k <= most &&
           // a grid holds fewer than 2^32 threads, 256 a tile of 128 x 128 (shares are joined for 2^26 elements at most)
           ceil_div(m, 128) * ceil_div(std::max(n, k), 128) < (1 << 24) && ceil_div(n, 128) * ceil_div(k, 128) < (1 << 24);
}

// A row stride that may be used where there are fewer than two rows, too.
inline int64_t ld_of(int64_t ld, int64_t rows, int64_t cols, int type) { return rows < 2 ? whole_ld(cols, (int)size_of(type)) : ld; }

inline bool valid_types(int type, int out_type) {
    if (type == TG_E4M3) return out_type == TG_BF16 || out_type == TG_F16;
    return (type == TG_BF16 || type == TG_F16) && out_type == type;
}

// Where a gradient's pass over dy leaves sums of its rows.
inline int slope_rows(int64_t m, int64_t n) {  // blocks down the rows: about 2048 blocks in all, 8 rows at least in each
    const int64_t want = std::max<int64_t>(1, 2048 / std::max<int64_t>(1, ceil_div(n, 256)));
    return (int)std::min<int64_t>(want, std::max<int64_t>(1, ceil_div(m, 8)));
}

}  // namespace
}  // namespace tg
