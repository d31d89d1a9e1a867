// block_linear.hip -- matrix product of 8-bit operands with a scale for every 128
// elements of a row of x and for every 128 x 128 of w (tg_block_linear).
//
// With P = x and Q = w, r along their rows, and b the blocks of 128 of r:
//        C[i][j] = sum over b of ps(i, b) qs(j / 128, b) (sum over r in b of P(i, r) Q(j, r))
// A block of r is a step of the loop over r, one row of a tile in LDS, and one
// 16 x 16 x 128 matrix instruction.
#include "product.h"

namespace tg {
namespace {

using i32x8 = vec<int, 8>;

// With scales that are powers of two the instruction multiplies by them itself.
__device__ inline f32x4 mma_block(i32x8 a, i32x8 b, f32x4 c, int code_a, int code_b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, code_a, 0, code_b);
}
__device__ inline f32x4 mma_block(i32x8 a, i32x8 b) { return mma_block(a, b, f32x4(0.0f), 0, 0); }  // zeros: no scales

// A buffer descriptor that moves through an operand: `bytes` further on, with as many
// bytes fewer up to the operand's end.  Its registers may come from vector
// instructions; the pause stands before any load of this file (Stream::settle has why).
__device__ inline i32x4 descriptor(uint64_t from, int64_t left) {
    i32x4 d;
    d[0] = __builtin_amdgcn_readfirstlane((int)from);
    d[1] = __builtin_amdgcn_readfirstlane((int)(from >> 32) & 0xffff);
    d[2] = __builtin_amdgcn_readfirstlane((int)std::min<int64_t>(left, 0x7ffffff0));
    d[3] = 0x00027000;
    asm volatile("s_nop 4" : "+s"(d));
    return d;
}
__device__ inline void advance(i32x4 &d, int bytes) {
    const uint64_t from = ((uint64_t)(unsigned)d[1] << 32 | (unsigned)d[0]) + bytes;
    d[0] = (int)from, d[1] = (int)(from >> 32);
    d[2] = d[2] > bytes ? d[2] - bytes : 0;
}

// The sum is made here, not where it is next used.
__device__ inline void settled(f32x4 &v) { asm volatile("" : "+v"(v)); }

// The scales of a tile on their way to LDS: groups of four blocks of r, [rows][4]
// words, of a row 16 bytes.  A load brings 16 rows: lane l the block l % 4 of row
// l / 4, so that a row's four lie in one access.  Rows past the last get the last
// one's, whose products are dropped; blocks past the last are not read.
template <bool kPowers, int kLoads>
struct ScaleStream {
    static constexpr int kSize = kPowers ? 1 : 4;
    i32x4 d;  // of the next group
    int at[kLoads];

    // Rows first, first + apart, ... (16 from each on) of those from row0 on; n_blocks blocks from b0 on.
    __device__ void init(const void *p, int64_t ld, int64_t row0, int64_t n_rows, int64_t b0, int n_blocks, int first, int apart) {
        const int lane = threadIdx.x % 64, row_bytes = (int)ld * kSize, last = (int)std::min<int64_t>(n_rows - row0, 256) - 1;
        d = descriptor((uint64_t)p + row0 * ld * kSize + b0 * kSize, (int64_t)last * row_bytes + n_blocks * kSize);
#pragma unroll
        for (int n = 0; n < kLoads; ++n) at[n] = std::min(first + n * apart + lane / 4, last) * row_bytes + lane % 4 * kSize;
    }
    // Load n of the next group, to 256 bytes at `to` of LDS.
    template <int n>
    __device__ void load(unsigned to) const {
        if constexpr (kPowers)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_ubyte %1, %2, 0 offen lds" ::"s"(to), "v"(at[n]), "s"(d) : "memory");
        else
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(at[n]), "s"(d) : "memory");
    }
    __device__ void advance() { tg::advance(d, 4 * kSize); }
};

// A wave's sums to C, from row i0 and column j0 on, or where they are a share's to
// `part`, rows of `ld`.  A lane has columns 4 (lane / 16) +
// c of row lane % 16 of each 16 x 16 part.  Two of them at a time go through the
// wave's place in LDS, in rows 16 bytes longer than their values, and come back 8
// columns a lane.
template <typename O, int kTI, int kTJ>
__device__ inline void finish_blocks(const f32x4 (&acc)[kTI][kTJ], float *rows, const Product &a, const Epilogue &e, int64_t i0, int64_t j0, float *part, int ld) {
    constexpr int kRow = 16 * kTJ + 4, kUnits = 2 * kTJ, kTurns = 32 * kUnits / 64;
    const int lane = threadIdx.x % 64;
    const int col = lane % kUnits * 8;
    const int64_t j = j0 + col;
    const int valid = (int)std::min<int64_t>(8, a.nj - j);
    Columns<8> columns{};
    if (!part && valid > 0) columns = load_columns<O, 8>(j, valid, e);
#pragma unroll
    for (int x = 0; x < kTI; x += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int y = 0; y < kTJ; ++y) *(f32x4 *)(rows + (h * 16 + lane % 16) * kRow + y * 16 + lane / 16 * 4) = acc[x + h][y];
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int n = 0; n < kTurns; ++n) {
            const int row = n * (64 / kUnits) + lane / kUnits;
            const int64_t i = i0 + x * 16 + row;
            if (i >= a.ni || valid <= 0) continue;
            const f32x4 lo = *(const f32x4 *)(rows + row * kRow + col), hi = *(const f32x4 *)(rows + row * kRow + col + 4);
            const vec<float, 8> z = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            if (part) {
                store_f32<float, 8>(part + (x * 16 + row) * ld + col, z, valid);
            } else {
                vec<float, 8> residual(0.0f);
                if (e.residual) residual = load_f32<O, 8>((const O *)e.residual + i * e.ldr + j, valid);
                finish<O, 8>(z, 1.0f, columns, residual, i, j, valid, e);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// 16 kTI kDown x 16 kTJ kAcross of C by kDown x kAcross waves.
template <typename O, bool kPowers, int kDown, int kAcross, int kTI, int kTJ>
__global__ __launch_bounds__(64 * kDown * kAcross, 2) void product_blocks(Product a, Epilogue e, int tiles_i, int tiles_j, int64_t r_bytes_p,
                                                                          int64_t r_bytes_q, int share_steps, int whole_tiles, int splits) {
    constexpr int kWaves = kDown * kAcross, kBI = 16 * kTI * kDown, kBJ = 16 * kTJ * kAcross;
    constexpr int kTileP = kBI * kStepBytes, kTileQ = kBJ * kStepBytes, kGroup = (kBI + 16) * 16;
    static_assert(kStepBytes == kScaled, "a step is a block of r");
    static_assert(kBJ / kScaled <= 16 && kScaled % (16 * kTJ) == 0, "a wave's columns share their scales");
    __shared__ __attribute__((aligned(1024))) char tiles[2 * kTileP + 2 * kTileQ + 2 * kGroup];
    const TailBlock block = tail_block(blockIdx.x, whole_tiles, (int64_t)tiles_i * tiles_j, splits);
    int bi, bj;
    tile_of(block.tile, tiles_i, tiles_j, &bi, &bj);
    const int64_t i0 = (int64_t)bi * kBI, j0 = (int64_t)bj * kBJ;
    const int wave = wave_index(), lane = threadIdx.x % 64;
    const int wi = wave / kAcross * 16 * kTI, wj = wave % kAcross * 16 * kTJ;
    const int64_t r0 = (int64_t)block.share * share_steps * kScaled, r1 = block.split ? std::min<int64_t>(a.nr, r0 + share_steps * kScaled) : a.nr;
    const int steps = (int)((r1 - r0 + kScaled - 1) / kScaled);

    Stream<e4m3, false, kBI, false, kWaves> sp;
    Stream<e4m3, false, kBJ, false, kWaves> sq;
    constexpr int kScaleLoads = kBI / 16 / kWaves;
    ScaleStream<kPowers, kScaleLoads> xs;
    ScaleStream<kPowers, 1> ws;
    sp.init(a.p, a.ldp, i0, a.ni, r0, r1, r1 < a.nr ? r1 : r_bytes_p);
    sq.init(a.q, a.ldq, j0, a.nj, r0, r1, r1 < a.nr ? r1 : r_bytes_q);
    const int64_t b0 = r0 / kScaled;
    xs.init(a.ps, a.ldps, i0, a.ni, b0, steps, wave * 16, kWaves * 16);
    ws.init(a.qs, a.ldqs, j0 / kScaled, (a.nj + kScaled - 1) / kScaled, b0, steps, 0, 0);
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)&tiles[0];
    const unsigned to_p = lds + wave * sp.kLoads * 1024, to_q = lds + 2 * kTileP + wave * sq.kLoads * 1024;
    constexpr int kScalesAt = 2 * kTileP + 2 * kTileQ;
    const auto load_scales = [&](int g) {
        const unsigned to = lds + kScalesAt + g % 2 * kGroup;
        each<0, kScaleLoads>([&](auto n) { xs.template load<n>(to + (n * kWaves + wave) * 256); });
        if (wave == 0) ws.template load<0>(to + kBI * 16);
        xs.advance(), ws.advance();
    };
    const auto load_p = [&](int h) {
        sp.open(h), sp.settle();
        each<0, sp.kLoads>([&](auto l) { sp.template load<l>(to_p + h % 2 * kTileP); });
    };
    const auto load_q = [&](int h) {
        sq.open(h), sq.settle();
        each<0, sq.kLoads>([&](auto l) { sq.template load<l>(to_q + h % 2 * kTileQ); });
    };
    f32x4 acc[kTI][kTJ] = {};
    if (steps > 0) {
        load_scales(0);
        load_p(0), load_q(0), load_q(1);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(sq.kLoads) : "memory");
        const int p_at = along_at(wi + lane % 16, lane / 16), q_at = 2 * kTileP + along_at(wj + lane % 16, lane / 16);
        const int p_at2 = along_at(wi + lane % 16, lane / 16 + 4), q_at2 = 2 * kTileP + along_at(wj + lane % 16, lane / 16 + 4);
        const auto fragment = [&](int lo, int hi) {
            return (i32x8)__builtin_shufflevector(*(const i32x4 *)(&tiles[0] + lo), *(const i32x4 *)(&tiles[0] + hi), 0, 1, 2, 3, 4, 5, 6, 7);
        };
        for (int t = 0; t < steps; ++t) {
            const int set = t % 2;
            if (t % 4 == 0) load_scales(t / 4 + 1);
            load_p(t + 1);
            i32x8 q[kTJ];
#pragma unroll
            for (int y = 0; y < kTJ; ++y) q[y] = fragment(q_at + set * kTileQ + y * 16 * kStepBytes, q_at2 + set * kTileQ + y * 16 * kStepBytes);
            const int scales_at = kScalesAt + t / 4 % 2 * kGroup + t % 4 * 4;
            const char *const x_scale = &tiles[0] + scales_at + (wi + lane % 16) * 16;
            const char *const w_scale = &tiles[0] + scales_at + (kBI + wj / kScaled) * 16;
            using word = std::conditional_t<kPowers, int, float>;
            const word sw = *(const word *)w_scale;
            word s[kTI];
#pragma unroll
            for (int x = 0; x < kTI; ++x) s[x] = *(const word *)(x_scale + x * 256);
            // every wave has what it wants of Q's tile, whose place the one after next takes
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            load_q(t + 2);
#pragma unroll
            for (int x = 0; x < kTI; ++x) {
                const i32x8 p = fragment(p_at + set * kTileP + x * 16 * kStepBytes, p_at2 + set * kTileP + x * 16 * kStepBytes);
                if constexpr (kPowers) {
#pragma unroll
                    for (int y = 0; y < kTJ; ++y) acc[x][y] = mma_block(q[y], p, acc[x][y], sw, s[x]);
                } else {
                    const float scale = s[x] * sw;
                    f32x4 part[kTJ];
#pragma unroll
                    for (int y = 0; y < kTJ; ++y) part[y] = mma_block(q[y], p);
#pragma unroll
                    for (int y = 0; y < kTJ; ++y) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[x][y][c] = fmaf(part[y][c], scale, acc[x][y][c]);
                    }
                }
            }
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(sq.kLoads) : "memory");
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // the last loads, before this LDS has another use
    }
    __syncthreads();
    static_assert(32 * (16 * kTJ + 4) * 4 * kWaves <= (int)sizeof(tiles), "the waves' shares fit the tiles' place");
    finish_blocks<O, kTI, kTJ>(acc, (float *)&tiles[0] + wave * 32 * (16 * kTJ + 4), a, e, i0 + wi, j0 + wj,
                               block.split ? e.partial + block.part * kBI * kBJ + wi * kBJ + wj : nullptr, kBJ);
}

// Rows of an operand on their way to a tile in LDS: kLoads times eight of them, from
// rows of the tile that the caller names (every other one a multiple of 16).
template <int kLoads>
struct RowStream {
    int at[kLoads];
    unsigned to[kLoads];  // bytes into LDS from the first tile on

    template <typename F>
    __device__ void init(unsigned tile, int64_t ld, F row_of) {
        const int lane = threadIdx.x % 64, unit = ((lane % 8) ^ (lane / 16)) * 16;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            to[n] = tile + row_of(n) * kStepBytes;
            at[n] = (int)((row_of(n) + lane / 8) * ld) + (unit ^ n % 2 * 64);
        }
    }
    // From now on lanes whose unit lies past the row's end, `left` bytes into the step,
    // load zeros.
    __device__ void end(int left) {
        const int lane = threadIdx.x % 64, unit = ((lane % 8) ^ (lane / 16)) * 16;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) at[n] |= (unit ^ n % 2 * 64) >= left ? (int)0x80000000 : 0;
    }
    // The descriptor's step, to the tile `place` bytes after the first.
    __device__ void load(i32x4 d, unsigned place) const {
#pragma unroll
        for (int n = 0; n < kLoads; ++n)
            asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds" ::"s"(place), "s"(to[n]), "v"(at[n]), "s"(d)
                         : "memory", "scc");
    }
};

// 256 x 256 of C by eight waves of 128 x 64, two to a SIMD that take turns: while one
// multiplies, the other reads its next fragments from LDS and starts loads.  A step
// has four turns, ended by a barrier each: a wave reads Q's fragments and the first
// half of its rows of P, multiplies those, reads the second half, multiplies; the
// waves of the upper half of the tile are a turn ahead of the lower half's.  Loads go
// to the place of a tile's half as soon as both have read it, one and a half steps
// before it is read again.  A wave issues an instruction every four or five cycles,
// so a turn of 512 cycles of the matrix unit has room for some hundred: descriptors
// and addresses only move from step to step (made anew at each they cost as much as
// the products).  A step has 2048 cycles of the matrix unit; with powers of two it
// takes 2750, with floats, whose sums go through as many multiplications and
// additions again, 3050, at the 1.7 to 1.9 GHz that the power allows.  8192 x 7168 x
// 8192 takes 353 to 390 us with powers of two (2460 to 2720 TFLOP/s; the plain 8-bit
// product 359 to 404), with floats 433 to 480; the same loop by eight waves that go
// in step took 546.
template <typename O, bool kPowers>
__global__ __launch_bounds__(512, 2) void product_blocks_large(Product a, Epilogue e, int tiles_i, int tiles_j, int64_t r_bytes_p, int64_t r_bytes_q,
                                                               int share_steps, int whole_tiles, int splits) {
    constexpr int kB = 256, kTI = 8, kTJ = 4, kHalf = kTI / 2, kTile = kB * kStepBytes, kGroup = (kB + 16) * 16, kScalesAt = 4 * kTile;
    __shared__ __attribute__((aligned(1024))) char tiles[4 * kTile + 2 * kGroup];
    const TailBlock block = tail_block(blockIdx.x, whole_tiles, (int64_t)tiles_i * tiles_j, splits);
    int bi, bj;
    tile_of(block.tile, tiles_i, tiles_j, &bi, &bj);
    const int64_t i0 = (int64_t)bi * kB, j0 = (int64_t)bj * kB;
    const int wave = wave_index(), lane = threadIdx.x % 64;
    const int wi = wave / 4 * 128, wj = wave % 4 * 64;
    const bool behind = wave >= 4;
    const int64_t r0 = (int64_t)block.share * share_steps * kScaled, r1 = block.split ? std::min<int64_t>(a.nr, r0 + share_steps * kScaled) : a.nr;
    const int steps = (int)((r1 - r0 + kScaled - 1) / kScaled);
    f32x4 acc[kTI][kTJ] = {};
    if (steps > 0) {
        RowStream<2> lo, hi;
        RowStream<4> sq;
        ScaleStream<kPowers, 2> xs;
        ScaleStream<kPowers, 1> ws;
        const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)&tiles[0];
        const int row = wave / 4 * 128 + wave % 4 * 16;
        lo.init(lds, a.ldp, [&](int n) { return row + 8 * n; });
        hi.init(lds, a.ldp, [&](int n) { return row + 64 + 8 * n; });
        sq.init(lds + 2 * kTile, a.ldq, [&](int n) { return wave * 32 + 8 * n; });
        const int64_t b0 = r0 / kScaled;
        xs.init(a.ps, a.ldps, i0, a.ni, b0, steps, wave * 16, 128);
        ws.init(a.qs, a.ldqs, j0 / kScaled, (a.nj + kScaled - 1) / kScaled, b0, steps, 0, 0);
        // descriptors: for `hi` of the step after the one that is multiplied, for the others of the one after that
        const int64_t end_p = r1 < a.nr ? r1 : r_bytes_p, end_q = r1 < a.nr ? r1 : r_bytes_q;
        i32x4 d_hi = descriptor((uint64_t)a.p + i0 * a.ldp + r0, (std::min<int64_t>(a.ni - i0, kB) - 1) * a.ldp + end_p - r0);
        i32x4 dq = descriptor((uint64_t)a.q + j0 * a.ldq + r0, (std::min<int64_t>(a.nj - j0, kB) - 1) * a.ldq + end_q - r0);
        const int last_p = (int)(end_p - r0 - (int64_t)(steps - 1) * kStepBytes), last_q = (int)(end_q - r0 - (int64_t)(steps - 1) * kStepBytes);
        i32x4 d_lo = d_hi;
        const auto load_scales = [&](int g) {
            const unsigned to = lds + kScalesAt + g % 2 * kGroup;
            each<0, 2>([&](auto n) { xs.template load<n>(to + (n * 8 + wave) * 256); });
            if (wave == 0) ws.template load<0>(to + kB * 16);
            xs.advance(), ws.advance();
        };
        // The turn's end.  Eight loads may be on their way where the next readers' tiles
        // have to be there: the half tiles after those (2 and 6).
        const auto meet = [&](auto arrived) {
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (arrived)
                asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            else
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        const auto end_lo_q = [&]() { lo.end(last_p), sq.end(last_q); };
        load_scales(0);
        if (steps == 1) end_lo_q(), hi.end(last_p);
        const auto load_lo_q = [&](unsigned place) {
            sq.load(dq, place), lo.load(d_lo, place);
            advance(dq, kStepBytes), advance(d_lo, kStepBytes);
        };
        const auto load_hi = [&](unsigned place) {
            hi.load(d_hi, place);
            advance(d_hi, kStepBytes);
        };
        load_lo_q(0), load_hi(0);
        if (steps == 2) end_lo_q();
        load_lo_q(kTile);
        meet(std::true_type{});
        // units lane / 16 and four on; the tiles' first bytes are multiples of 128
        int p_at[2] = {along_at(wi + lane % 16, lane / 16), along_at(wi + lane % 16, lane / 16 + 4)};
        int q_at[2] = {2 * kTile + along_at(wj + lane % 16, lane / 16), 2 * kTile + along_at(wj + lane % 16, lane / 16 + 4)};
        const int x_scale = kScalesAt + (wi + lane % 16) * 16, w_scale = kScalesAt + (kB + wj / kScaled) * 16;
        const auto fragment = [&](const int (&at)[2], int more) {
            return (i32x8)__builtin_shufflevector(*(const i32x4 *)(&tiles[0] + at[0] + more), *(const i32x4 *)(&tiles[0] + at[1] + more), 0, 1, 2, 3, 4, 5, 6, 7);
        };
        using word = std::conditional_t<kPowers, int, float>;
        i32x8 q[kTJ], p[kHalf];
        word s[kHalf];
        word sw;
        // A block's products wait here for their scale while three further ones begin:
        // the result of a matrix instruction may be read 11 instructions later.
        constexpr int kLag = 3, kParts = 4;
        f32x4 part[kParts];
        const auto add = [&](auto half, auto n) {
            constexpr int x = half * kHalf + n / kTJ, y = n % kTJ;
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[x][y][c] = fmaf(part[n % kParts][c], s[n / kTJ], acc[x][y][c]);
            settled(acc[x][y]);
        };
        // scales: bytes of the step's among them
        const auto read = [&](auto half, int scales) {
            if constexpr (half == 0) {
#pragma unroll
                for (int y = 0; y < kTJ; ++y) q[y] = fragment(q_at, y * 16 * kStepBytes);
                sw = *(const word *)(&tiles[0] + w_scale + scales);
            }
#pragma unroll
            for (int x = 0; x < kHalf; ++x) p[x] = fragment(p_at, (half * kHalf + x) * 16 * kStepBytes);
            const char *const from = &tiles[0] + x_scale + scales;
#pragma unroll
            for (int x = 0; x < kHalf; ++x) s[x] = *(const word *)(from + (half * kHalf + x) * 256);
            if constexpr (!kPowers) {
#pragma unroll
                for (int x = 0; x < kHalf; ++x) s[x] *= sw;
            }
        };
        const auto multiply = [&](auto half) {
            each<0, kHalf * kTJ>([&](auto n) {
                constexpr int x = n / kTJ, y = n % kTJ;
                if constexpr (kPowers) {
                    acc[half * kHalf + x][y] = mma_block(q[y], p[x], acc[half * kHalf + x][y], sw, s[x]);
                } else {
                    part[n % kParts] = mma_block(q[y], p[x]);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (n >= kLag) add(half, std::integral_constant<int, n - kLag>{});
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            if constexpr (kPowers)
                each<0, kHalf * kTJ>([&](auto n) { settled(acc[half * kHalf + n / kTJ][n % kTJ]); });
        };
        // what multiply leaves over runs beside the other wave's matrix instructions
        const auto rest = [&](auto half) {
            if constexpr (!kPowers) each<kHalf * kTJ - kLag, kHalf * kTJ>([&](auto n) { add(half, n); });
        };
        constexpr std::integral_constant<int, 0> first{};
        constexpr std::integral_constant<int, 1> second{};
        const auto run = [&](auto late) {
            constexpr std::integral_constant<bool, !late> early{};
            if constexpr (late) meet(early);
            unsigned place = 0;  // of this step's tiles
            for (int t = 0; t < steps; ++t) {
                const int scales = t / 4 % 2 * kGroup + t % 4 * 4;
                read(first, scales);
                if (t % 4 == 0) load_scales(t / 4 + 1);
                if (t == steps - 2) hi.end(last_p);
                load_hi(place ^ kTile);
                meet(late);
                multiply(first);
                meet(early);
                rest(first);
                read(second, scales);
                if (t == steps - 3) end_lo_q();
                load_lo_q(place);
                place ^= kTile;
#pragma unroll
                for (int c = 0; c < 2; ++c) p_at[c] ^= kTile, q_at[c] ^= kTile;
                meet(late);
                multiply(second);
                meet(early);
                rest(second);
            }
            if constexpr (early) meet(late);
        };
        if (behind)
            run(std::true_type{});
        else
            run(std::false_type{});
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // the last loads, before this LDS has another use
    }
    __syncthreads();
    finish_blocks<O, kTI, kTJ>(acc, (float *)&tiles[0] + wave * 32 * (16 * kTJ + 4), a, e, i0 + wi, j0 + wj,
                               block.split ? e.partial + block.part * kB * kB + wi * kB + wj : nullptr, kB);
}

template <typename O, bool kPowers>
hipError_t launch_blocks(Product a, Epilogue e, char *ws, hipStream_t s) {
    constexpr Form kForm = kPowers ? kExponents : kBlocks;
    if (a.ni == 0 || a.nj == 0) return hipSuccess;
    int64_t r_bytes_p = a.nr;
    const Plan p = plan_product<kForm>(a, 1, r_bytes_p, false, false);
    if (p.few) return launch_few<e4m3, O, kForm>(a, e, p, ws, s);
    const hipError_t r = pack_operands<e4m3, kForm, false, false>(a, p, r_bytes_p, ws, s);
    if (r != hipSuccess) return r;
    const int64_t r_bytes_q = p.pack_q ? a.ldq : a.nr;
    const TailCut &c = p.tail;
    e.partial = (float *)(ws + p.p_bytes + p.q_bytes);
    const int ti = (int)ceil_div(a.ni, c.tile), tj = (int)ceil_div(a.nj, c.tile);
    const dim3 grid((unsigned)(c.whole + c.tail * c.splits));
    if (c.tile == 256)
        hipLaunchKernelGGL((product_blocks_large<O, kPowers>), grid, dim3(512), 0, s, a, e, ti, tj, r_bytes_p, r_bytes_q, c.share, c.whole, c.splits);
    else
        hipLaunchKernelGGL((product_blocks<O, kPowers, 2, 2, 4, 4>), grid, dim3(256), 0, s, a, e, ti, tj, r_bytes_p, r_bytes_q, c.share, c.whole, c.splits);
    return join_tail<O, kForm>(a, e, c, ti, tj, s);
}

Product product_of(const tg_block_linear_args &q) {
    Product a{q.x, q.w, ld_of(q.ldx, q.m, q.k, TG_E4M3), ld_of(q.ldw, q.n, q.k, TG_E4M3), q.m, q.n, q.k};
    a.ps = q.x_scale, a.qs = q.w_scale;
    a.ldps = q.m > 1 ? q.ldxs : 0, a.ldqs = q.n > kScaled ? q.ldws : 0;
    return a;
}

// A scale's offset in a tile of 256 rows fits 31 bits.
constexpr int64_t kMostScaleLd = 1 << 21;

tg_status check_scales(const void *p, int64_t ld, int64_t rows, int64_t cols, int type, const char *what) {
    if (rows == 0 || cols == 0) return TG_OK;
    if (!p) return call_failed(TG_EINVAL, "%s is NULL", what);
    if (type == TG_F32 && (uintptr_t)p % 4) return call_failed(TG_EINVAL, "%s is not aligned to its elements", what);
    if (rows > 1 && (ld < cols || ld >= kMostScaleLd))
        return call_failed(TG_EINVAL, "%s: row stride %lld, %lld to %lld expected", what, (long long)ld, (long long)cols, (long long)kMostScaleLd - 1);
    return TG_OK;
}

}  // namespace
}  // namespace tg

using namespace tg;

extern "C" {

size_t tg_block_linear_workspace_bytes(const tg_block_linear_args *q) {
    if (!q || !sizes_fit(q->m, q->n, q->k)) return 0;
    const Product a = product_of(*q);
    return (q->scale_type == TG_F32 ? plan_product<kBlocks>(a, 1, q->k, false, false) : plan_product<kExponents>(a, 1, q->k, false, false)).bytes;
}

tg_status tg_block_linear(const tg_block_linear_args *q, void *d_ws, size_t ws_bytes, tg_stream stream) {
    if (!q) return call_failed(TG_EINVAL, "arguments are NULL");
    if (q->reserved) return call_failed(TG_EINVAL, "reserved must be 0");
    if (q->scale_type != TG_F32 && q->scale_type != TG_E8M0) return call_failed(TG_EINVAL, "scale_type %d", q->scale_type);
    if (q->out_type != TG_BF16 && q->out_type != TG_F16) return call_failed(TG_EINVAL, "out_type %d", q->out_type);
    if (q->act < TG_ACT_NONE || q->act > TG_ACT_GELU) return call_failed(TG_EINVAL, "act %d", q->act);
    if (!sizes_fit(q->m, q->n, q->k))
        return call_failed(TG_EINVAL, "m %lld, n %lld, k %lld", (long long)q->m, (long long)q->n, (long long)q->k);
    const int64_t blocks = ceil_div(q->k, kScaled);
    TG_TRY(check_matrix(q->x, q->ldx, q->m, q->k, TG_E4M3, "x"));
    TG_TRY(check_matrix(q->w, q->ldw, q->n, q->k, TG_E4M3, "w"));
    TG_TRY(check_scales(q->x_scale, q->ldxs, q->m, blocks, q->scale_type, "x_scale"));
    TG_TRY(check_scales(q->w_scale, q->ldws, ceil_div(q->n, kScaled), blocks, q->scale_type, "w_scale"));
    TG_TRY(check_matrix(q->y, q->ldy, q->m, q->n, q->out_type, "y"));
    if (q->residual) TG_TRY(check_matrix(q->residual, q->ldr, q->m, q->n, q->out_type, "residual"));
    if (q->bias) TG_TRY(check_matrix(q->bias, 0, 1, q->n, q->out_type, "bias"));
    TG_TRY(check_workspace(d_ws, ws_bytes, tg_block_linear_workspace_bytes(q)));
    Epilogue e{};
    e.bias = q->bias, e.residual = q->residual, e.out = q->y;
    e.ldr = q->ldr, e.ldo = q->ldy, e.act = q->act;
    const Product a = product_of(*q);
    const hipStream_t s = (hipStream_t)stream;
    char *const ws = (char *)d_ws;
    hipError_t r;
    if (q->scale_type == TG_F32)
        r = q->out_type == TG_BF16 ? launch_blocks<bf16, false>(a, e, ws, s) : launch_blocks<f16, false>(a, e, ws, s);
    else
        r = q->out_type == TG_BF16 ? launch_blocks<bf16, true>(a, e, ws, s) : launch_blocks<f16, true>(a, e, ws, s);
    return r == hipSuccess ? TG_OK : device_failed(r, "the block-scaled product");
}

}  // extern "C"
