// Projection by weights of 4 bits with a scale and a zero point per group (apex_linear_w4).
//
// y[t, n] = sum over groups g of s(n, g) * (sum_k q x - z(n, g) * sum_k x), k in g.  The codes go to the
// matrix cores as bf16 without arithmetic: bits 3 to 6 of the word 0x4180 are the upper bits of the
// mantissa of 16, so a code q put there makes 16 + q, exactly, two values for a shift and an
// and-or.  The group's product is then sum (16 + q) x, and a product with ones gives sum x:
//   s * (sum (16 + q) x - (16 + z) * sum x),
// in fp32, without rounding a weight.  fp32 values of x are cut into three bf16 pieces of 8 bits
// whose sum they are, so no operand is rounded there either.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 128;         // codes of a row that stand together, 64 bytes

struct LinearArgs {
    const uint8_t *codes;
    const uint32_t *words;
    const uint16_t *x;              // bf16, or the pieces of fp32
    int64_t x_stride, x_piece;      // in values
    int x_cols;                     // values of a row of x that there are (a multiple of 8)
    const float *bias;
    const void *residual;
    void *y;
    int64_t residual_stride, y_stride;
    int N, T, blocks;               // blocks of kBlock codes in a row
    int pieces;                     // of x: 1 (bf16) or 3 (fp32; in memory where !STAGE)
    bool y32;
};

// Codes 2 i and 2 i + 1 of a word as bf16 pairs 16 + q.
__device__ __forceinline__ bf16x8 widen(uint32_t w) {
    uint4 b;
    b.x = ((w << 3) & 0x00780078u) | 0x41804180u;
    b.y = ((w >> 1) & 0x00780078u) | 0x41804180u;
    b.z = ((w >> 5) & 0x00780078u) | 0x41804180u;
    b.w = ((w >> 9) & 0x00780078u) | 0x41804180u;
    return __builtin_bit_cast(bf16x8, b);
}

__device__ __forceinline__ uint32_t word_of(const uint4 &v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// A group's scale and zero point, and its part of a sum: s (sum (16 + q) x - (16 + z) sum x).
struct Scale {
    float s, z;
    __device__ __forceinline__ explicit Scale(uint32_t word)
        : s(__uint_as_float(word & 0xffff0000u)), z(16.f + __uint_as_float(word << 16)) {}
    __device__ __forceinline__ void add(float &sum, float prod, float total) const {
        sum = fmaf(s, fmaf(-z, total, prod), sum);
    }
};

__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float load_y(bool f32, const void *p, int64_t i) {
    if (f32) return static_cast<const float *>(p)[i];
    return __uint_as_float(uint32_t(static_cast<const uint16_t *>(p)[i]) << 16);
}
__device__ __forceinline__ void store_y(bool f32, void *p, int64_t i, float v) {
    if (f32)
        static_cast<float *>(p)[i] = v;
    else
        static_cast<uint16_t *>(p)[i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// Bias and residual, and the result's own rounding.
__device__ __forceinline__ void put(const LinearArgs &a, int64_t t, int n, float y) {
    if (a.bias) y += a.bias[n];
    if (a.residual) y += load_y(a.y32, a.residual, t * a.residual_stride + n);
    store_y(a.y32, a.y, t * a.y_stride + n, y);
}

// 8 fp32 values as three rows of bf16 pieces whose sum they are: the upper 8 bits of the value, of
// what is left, and of what is left then.
__device__ __forceinline__ void cut(const float (&v)[8], uint4 (&p)[3]) {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = v[e];
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        uint32_t top[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            top[e] = __float_as_uint(f[e]) & 0xffff0000u;
            f[e] -= __uint_as_float(top[e]);
        }
        p[j] = make_uint4(top[0] >> 16 | top[1], top[2] >> 16 | top[3], top[4] >> 16 | top[5], top[6] >> 16 | top[7]);
    }
}

// A workgroup's way through the weights: tiles of 16 R rows; of a tile, wavefront w takes the blocks of
// 128 codes w, w + kWaves, ... along K, `steps` of them.  Workgroups go to the 8 XCDs in turn, and each XCD
// has an eighth of the tiles, so that tiles side by side, which share lines of group words, share an L2.
struct Walk {
    int tile, end, step;
    __device__ __forceinline__ Walk(int tiles) : step(0) {
        const int per = (tiles + 7) / 8, xcd = blockIdx.x & 7;
        tile = xcd * per + (blockIdx.x >> 3);
        end = min((xcd + 1) * per, tiles);
    }
    __device__ __forceinline__ void next(int steps) {
        if (++step == steps) step = 0, tile += gridDim.x >> 3;
    }
};
constexpr int kWaves = 8;
constexpr int kPad = 64;            // bytes behind a staged row: rows begin 16 banks apart

// The codes and the group words of a block of 16 R rows, D blocks ahead of their use.  Descriptors end
// with the tile's rows, and are empty for blocks that are not there: such loads move nothing.  A quarter of
// the wavefront loads the words of one group (of less than 128 codes) and gets the others' from it.
template <int GROUP, int R>
struct Block {
    static constexpr int PER = kBlock / GROUP;
    uint4 code[R];
    uint32_t word[R];
    __device__ __forceinline__ void load(const LinearArgs &a, int n0, int b, bool there, int lane) {
        const int rows = min(16 * R, a.N - n0), pitch = a.blocks * 64;
        const auto codes = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t *>(a.codes) + (there ? int64_t(n0) * pitch + b * 64 : 0), 0,
            there ? (rows - 1) * pitch + 64 : 0, 0x00027000);
        const auto words = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint32_t *>(a.words) + (there ? int64_t(b) * PER * a.N + n0 : 0), 0,
            there ? ((PER - 1) * a.N + rows) * 4 : 0, 0x00027000);
        const int col = lane & 15, quarter = lane >> 4;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            code[r] = __builtin_bit_cast(
                uint4, __builtin_amdgcn_raw_buffer_load_b128(codes, (16 * r + col) * pitch + 16 * quarter, 0, 0));
            word[r] = __builtin_amdgcn_raw_buffer_load_b32(words, (quarter % PER * a.N + 16 * r + col) * 4, 0, 0);
        }
    }
    __device__ __forceinline__ void words_of(int r, uint32_t (&w)[PER]) const {
        if constexpr (PER == 1) {
            w[0] = word[r];
        } else if constexpr (PER == 2) {
            const auto v = __builtin_amdgcn_permlane16_swap(word[r], word[r], false, false);
            w[0] = v[0], w[1] = v[1];
        } else {
            const auto h = __builtin_amdgcn_permlane32_swap(word[r], word[r], false, false);
            const auto lo = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false);
            const auto hi = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);
            w[0] = lo[0], w[1] = lo[1], w[2] = hi[0], w[3] = hi[1];
        }
    }
};

// How the rows of x stand in the 16 rows of a matrix instruction, whose lane holds rows 4 q + i, i =
// 0..3, of the result (q = lane / 16):
enum Rows {
    kFew,       // up to 4 rows of bf16, row q at i = 0: one result a lane
    kPieces,    // up to 4 rows of fp32, the pieces of row q at i = 0..2: one result a lane, their sum
    kMore       // up to 16 rows of bf16
};
constexpr int staged_rows(int rows, int T) { return rows == kPieces ? 3 * T : T; }

// Few rows: all of x goes to LDS first, at most stage_bytes() of it.  The wavefronts join their sums in LDS
// in a fixed order.
template <int GROUP, int R, int ROWS>
__global__ __launch_bounds__(64 * kWaves) void linear_few(LinearArgs a) {
    extern __shared__ uint4 lds[];
    constexpr int PER = kBlock / GROUP, STEPS = GROUP / 32;
    constexpr int NI = ROWS == kFew ? 1 : ROWS == kPieces ? 3 : 4;    // results of a lane,
    constexpr int NO = ROWS == kMore ? 4 : 1;                         // and after adding the pieces
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
    const int tiles = (a.N + 16 * R - 1) / (16 * R), steps = (a.blocks + kWaves - 1) / kWaves;
    // x on its way first (memory answers in order), then the first codes, then x into LDS
    const int x_pitch = a.blocks * 256 + kPad;
    const auto fetch = [&](int t, int i, uint4 (&v)[ROWS == kPieces ? 2 : 1]) {       // values 8 i .. of row t
        const bool there = t < a.T && 8 * i < a.x_cols;
        const uint16_t *from = a.x + (there ? (t * a.x_stride + 8 * i) * (ROWS == kPieces ? 2 : 1) : 0);
#pragma unroll
        for (int h = 0; h < (ROWS == kPieces ? 2 : 1); ++h) {
            v[h] = reinterpret_cast<const uint4 *>(from)[h];
            if (!there) v[h] = make_uint4(0u, 0u, 0u, 0u);
        }
    };
    const auto stage = [&](int t, int i, const uint4 (&v)[ROWS == kPieces ? 2 : 1]) {
        if (t >= a.T || i >= a.blocks * 16) return;
        char *to = reinterpret_cast<char *>(lds) + 16 * i;
        if constexpr (ROWS != kPieces) {
            *reinterpret_cast<uint4 *>(to + t * x_pitch) = v[0];
        } else {
            uint4 p[3];
            cut({__uint_as_float(v[0].x), __uint_as_float(v[0].y), __uint_as_float(v[0].z), __uint_as_float(v[0].w),
                 __uint_as_float(v[1].x), __uint_as_float(v[1].y), __uint_as_float(v[1].z), __uint_as_float(v[1].w)}, p);
#pragma unroll
            for (int j = 0; j < 3; ++j) *reinterpret_cast<uint4 *>(to + (3 * t + j) * x_pitch) = p[j];
        }
    };
    constexpr int FIRST = ROWS == kPieces ? 1 : 4;      // rows whose first values are on their way at once
    uint4 early[FIRST][ROWS == kPieces ? 2 : 1];
#pragma unroll
    for (int t = 0; t < FIRST; ++t) fetch(t, threadIdx.x, early[t]);
    Block<GROUP, R> next;
    Walk ahead(tiles);
    const auto load = [&] {
        const int b = wave + ahead.step * kWaves;
        next.load(a, ahead.tile * 16 * R, b, b < a.blocks && ahead.tile < ahead.end, lane);
        ahead.next(steps);
    };
    load();
#pragma unroll
    for (int t = 0; t < FIRST; ++t) stage(t, threadIdx.x, early[t]);
#pragma unroll 1
    for (int t = 0; t < a.T; ++t)
#pragma unroll 1
        for (int i = threadIdx.x + (t < FIRST ? 64 * kWaves : 0); i < a.blocks * 16; i += 64 * kWaves) {
            uint4 v[ROWS == kPieces ? 2 : 1];
            fetch(t, i, v);
            stage(t, i, v);
        }
    __syncthreads();
    // rows of the instruction that stand for none repeat one
    const int row = ROWS == kMore ? min(col, a.T - 1)
                                  : ROWS == kFew ? min(col >> 2, a.T - 1) : 3 * min(col >> 2, a.T - 1) + min(col & 3, 2);
    const char *staged = reinterpret_cast<const char *>(lds) + row * x_pitch + 16 * quarter;
    float *part = reinterpret_cast<float *>(reinterpret_cast<char *>(lds) + staged_rows(ROWS, a.T) * x_pitch);

    float sum[R][NI] = {};
    Walk now(tiles);
    int flip = 0;
    while (now.tile < now.end) {
        const int b = wave + now.step * kWaves;
        if (b < a.blocks) {
            uint4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const uint4 *>(staged + b * 256 + 64 * j);
            uint32_t words[R][PER];
#pragma unroll
            for (int r = 0; r < R; ++r) next.words_of(r, words[r]);
#pragma unroll
            for (int g = 0; g < PER; ++g) {
                floatx4 prod[R] = {}, total = {};
#pragma unroll
                for (int j = g * STEPS; j < (g + 1) * STEPS; ++j) {
                    const bf16x8 v = __builtin_bit_cast(bf16x8, x[j]);
                    total = mfma(v, ones, total);
#pragma unroll
                    for (int r = 0; r < R; ++r) prod[r] = mfma(v, widen(word_of(next.code[r], j)), prod[r]);
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const Scale w(words[r][g]);
#pragma unroll
                    for (int i = 0; i < NI; ++i) w.add(sum[r][i], prod[r][i], total[i]);
                }
            }
        }
        load();
        if (now.step == steps - 1) {               // the tile is done: join, then bias and residual
            float *mine = part + flip * (kWaves * R * NO * 64);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < NO; ++i) {
                    float v = sum[r][i];
                    if constexpr (ROWS == kPieces) v = sum[r][2] + sum[r][1] + v;
                    mine[((wave * R + r) * NO + i) * 64 + lane] = v;
                }
            __syncthreads();
            for (int e = threadIdx.x; e < R * NO * 64; e += 64 * kWaves) {
                float v = mine[e];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) v += mine[w * (R * NO * 64) + e];
                const int at = e & 63, i = (e >> 6) % NO, r = (e >> 6) / NO;
                const int64_t t = ROWS == kMore ? 4 * (at >> 4) + i : at >> 4;
                const int n = now.tile * 16 * R + 16 * r + (at & 15);
                if (t < a.T && n < a.N) put(a, t, n, v);
            }
            flip ^= 1;                              // the next tile's sums: other wavefronts may still read these
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < NI; ++i) sum[r][i] = 0.f;
        }
        now.next(steps);
    }
}

// Some rows, more than are staged at once: up to 16 TT rows, bf16 or (P = 3) the pieces of fp32.  A
// workgroup takes 16 R rows of the weights; each wavefront brings the part of x that belongs to its
// next block, P TT times 16 rows of 256 bytes, into LDS of its own, by loads of whole lines, and reads
// them as the matrix instructions want them.  Within a row 16-byte chunks stand in the place c ^ (row mod
// 16), so that 16 rows' chunks meet 64 banks.
template <int GROUP, int R, int TT, int P>
__global__ __launch_bounds__(64 * kWaves) void linear_some(LinearArgs a) {
    constexpr int PER = kBlock / GROUP, STEPS = GROUP / 32, LOADS = 4 * TT * P, OUT = R * TT * 4 * 64;
    __shared__ uint4 lds[kWaves * (LOADS * 64 > OUT / 4 ? LOADS * 64 : OUT / 4)];     // x, then the sums
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
    const int per = ((a.N + 16 * R - 1) / (16 * R) + 7) / 8;
    const int n0 = ((blockIdx.x & 7) * per + (blockIdx.x >> 3)) * 16 * R;      // as in Walk, one tile each
    if (n0 >= a.N) return;
    const int t0 = blockIdx.y * 16 * TT;
    uint4 x[LOADS];
    Block<GROUP, R> next;
    // load i of a block: rows 4 (i mod 4 TT) + quarter of a piece, chunk `col`
    const auto load_x = [&](int b) {
        const int k = b * kBlock + 8 * col;
        const bool there = k < a.x_cols;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int t = min(t0 + 4 * (i % (4 * TT)) + quarter, a.T - 1);
            uint4 v = *reinterpret_cast<const uint4 *>(a.x + i / (4 * TT) * a.x_piece + t * a.x_stride + (there ? k : 0));
            if (!there) v = make_uint4(0u, 0u, 0u, 0u);
            x[i] = v;
        }
    };
    char *mine = reinterpret_cast<char *>(lds) + wave * (LOADS * 1024);
    float sum[R][TT][4] = {};
    load_x(wave);
    next.load(a, n0, wave, wave < a.blocks, lane);
    for (int b = wave; b < a.blocks; b += kWaves) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int row = 4 * i + quarter;
            *reinterpret_cast<uint4 *>(mine + row * 256 + 16 * (col ^ (row & 15))) = x[i];
        }
        const Block<GROUP, R> now = next;
        load_x(b + kWaves);
        next.load(a, n0, b + kWaves, b + kWaves < a.blocks, lane);
        uint32_t words[R][PER];
#pragma unroll
        for (int r = 0; r < R; ++r) now.words_of(r, words[r]);
#pragma unroll
        for (int g = 0; g < PER; ++g) {
            floatx4 prod[R][TT] = {}, total[TT] = {};
#pragma unroll
            for (int j = g * STEPS; j < (g + 1) * STEPS; ++j) {
                bf16x8 q[R];
#pragma unroll
                for (int r = 0; r < R; ++r) q[r] = widen(word_of(now.code[r], j));
#pragma unroll
                for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                    for (int p = P - 1; p >= 0; --p) {
                        const bf16x8 v = *reinterpret_cast<const bf16x8 *>(mine + ((p * TT + tt) * 16 + col) * 256 +
                                                                           16 * ((4 * j + quarter) ^ col));
                        total[tt] = mfma(v, ones, total[tt]);
#pragma unroll
                        for (int r = 0; r < R; ++r) prod[r][tt] = mfma(v, q[r], prod[r][tt]);
                    }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const Scale w(words[r][g]);
#pragma unroll
                for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) w.add(sum[r][tt][i], prod[r][tt][i], total[tt][i]);
            }
        }
    }
    __syncthreads();
    float *part = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[wave * OUT + ((r * TT + tt) * 4 + i) * 64 + lane] = sum[r][tt][i];
    __syncthreads();
    for (int e = threadIdx.x; e < OUT; e += 64 * kWaves) {
        float v = part[e];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += part[w * OUT + e];
        const int at = e & 63, i = (e >> 6) & 3, tt = (e >> 8) % TT, r = (e >> 8) / TT;
        const int64_t t = t0 + 16 * tt + 4 * (at >> 4) + i;
        const int n = n0 + 16 * r + (at & 15);
        if (t < a.T && n < a.N) put(a, t, n, v);
    }
}

// Many rows.  A workgroup of 4 wavefronts takes 32 TT tokens by 32 R rows of the weights, each wavefront
// half of both, a block of 128 codes of one piece of x at a step.  x goes from memory to LDS
// directly (two stages, chunks placed as in linear_some), codes to registers, a step ahead; one
// barrier a step.  The sums of (16 + q) x are per group; the other half, (16 + z) sum x over groups, is
// a small product of its own, on the matrix cores in fp32, of sums of x that a launch before has
// made: 4 groups at a time, lane quarter q standing for group 4 m + q.
#define APEX_LDS __attribute__((address_space(3)))
constexpr int kManyThreads = 256;

__device__ __forceinline__ void barrier_after_loads() {       // every load of this wavefront has landed
    __builtin_amdgcn_s_waitcnt(0x0f70);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

struct ManyArgs {
    LinearArgs a;
    const float *totals;            // sums of x over groups, [T, blocks * 128 / GROUP]
    float *parts;                   // sums of a share of K, [splits][T][N]; NULL: one share, y is written
    int m_tiles, n_tiles, splits, share;      // blocks of a share, a multiple of 4
};

template <int GROUP, int TT, int R>
__global__ __launch_bounds__(kManyThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void linear_many(ManyArgs m) {
    constexpr int PER = kBlock / GROUP, STEPS = GROUP / 32, BM = 32 * TT, BN = 32 * R, LOADS = BM / 16;
    __shared__ __attribute__((aligned(1024))) uint8_t stage0[BM * 256], stage1[BM * 256];
    const LinearArgs &a = m.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    // an eighth of the tiles to each XCD, tokens first
    const int all = m.m_tiles * m.n_tiles * m.splits, id = (blockIdx.x & 7) * ((all + 7) / 8) + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= (all + 7) / 8 || id >= all) return;
    const int split = id / (m.m_tiles * m.n_tiles), tile = id - split * (m.m_tiles * m.n_tiles);
    const int n_tile = tile / m.m_tiles, t0 = (tile - n_tile * m.m_tiles) * BM, n0 = n_tile * BN;
    const int tw = t0 + (wave & 1) * 16 * TT, nw = n0 + (wave >> 1) * 16 * R;
    const int first = split * m.share, last = min(first + m.share, a.blocks);

    // row 4 i + quarter of this wavefront's part of the tile, its chunk for place `col`
    int from[LOADS];
    const int mine = wave * (BM / 4), rows = min(BM, a.T - t0);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int row = mine + 4 * i + quarter;
        from[i] = min(row, rows - 1) * int(a.x_stride) * 2 + 16 * (col ^ (row & 15));
    }
    const int x_bytes = (rows - 1) * int(a.x_stride) * 2 + a.x_cols * 2;
    const auto load_x = [&](uint8_t *stage, int b, int p) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(a.x) + p * a.x_piece + t0 * a.x_stride, 0,
                                                            x_bytes, 0x00027000);
        const bool tail = (b + 1) * kBlock > a.x_cols;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int at = from[i] + b * 256;
            if (tail && b * kBlock + 8 * (col ^ ((mine + 4 * i + quarter) & 15)) >= a.x_cols) at = 0x7ffffff0;   // zeros
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (APEX_LDS void *)(stage + (mine + 4 * i) * 256), 16, at, 0, 0, 0);
        }
    };
    Block<GROUP, R> next;
    float sum_x[TT];
    const auto load_w = [&](int b) {
        next.load(a, nw, b, b < last && nw < a.N, lane);
    };
    const int groups = a.blocks * PER;
    const auto load_totals = [&](int b) {              // of the 4 groups that block b is among
        const int g = b * PER / 4 * 4 + quarter;
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) {
            const float *p = m.totals + int64_t(min(tw + 16 * tt + col, a.T - 1)) * groups + min(g, groups - 1);
            sum_x[tt] = *p;
        }
    };
    floatx4 sum[R][TT] = {};
    uint32_t kept[R];                                  // words of 4 groups, one a lane quarter
#pragma unroll
    for (int r = 0; r < R; ++r) kept[r] = 0;

    const auto step = [&](const uint8_t *stage, uint8_t *other, int b, int p) {
        barrier_after_loads();
        const Block<GROUP, R> now = next;
        const bool ends = p == a.pieces - 1;           // of the block
        if (!ends)
            load_x(other, b, p + 1);
        else if (b + 1 < last)
            load_x(other, b + 1, 0);
        if (ends) load_w(b + 1);
        if (ends) {
            load_totals(b);
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (quarter / PER == b % (4 / PER)) kept[r] = now.word[r];
        }
        const uint8_t *at = stage + (wave & 1) * (16 * TT) * 256 + col * 256;
#pragma unroll
        for (int g = 0; g < PER; ++g) {
            bf16x8 x[STEPS][TT];
#pragma unroll
            for (int j = 0; j < STEPS; ++j)
#pragma unroll
                for (int tt = 0; tt < TT; ++tt)
                    x[j][tt] = *reinterpret_cast<const bf16x8 *>(at + tt * 4096 + 16 * ((4 * (g * STEPS + j) + quarter) ^ col));
#pragma unroll
            for (int r = 0; r < R; ++r) {
                uint32_t words[PER];
                now.words_of(r, words);
                const float s = __uint_as_float(words[g] & 0xffff0000u);
                floatx4 prod[TT] = {};
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    const bf16x8 q = widen(word_of(now.code[r], g * STEPS + j));
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt) prod[tt] = mfma(x[j][tt], q, prod[tt]);
                }
#pragma unroll
                for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[r][tt][i] = fmaf(s, prod[tt][i], sum[r][tt][i]);
            }
        }
        if (ends && (b % (4 / PER) == 4 / PER - 1 || b == last - 1)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const Scale w(kept[r]);
                const float c = -(w.s * w.z);
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) sum[r][tt] = __builtin_amdgcn_mfma_f32_16x16x4f32(sum_x[tt], c, sum[r][tt], 0, 0, 0);
                kept[r] = 0;
            }
        }
    };
    load_x(stage0, first, 0);
    next.load(a, nw, first, nw < a.N, lane);
    int b = first, p = 0;
    const auto forward = [&] {
        if (++p == a.pieces) p = 0, ++b;
    };
    while (b < last) {
        step(stage0, stage1, b, p);
        forward();
        if (b >= last) break;
        step(stage1, stage0, b, p);
        forward();
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);                // no load into LDS outlives the workgroup

#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int n = nw + 16 * r + col;
        if (n >= a.N) continue;
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t t = tw + 16 * tt + 4 * quarter + i;
                if (t >= a.T) continue;
                if (m.parts)
                    m.parts[(split * int64_t(a.T) + t) * a.N + n] = sum[r][tt][i];
                else
                    put(a, t, n, sum[r][tt][i]);
            }
    }
}

// The shares of K of every value of y, in order.
__global__ __launch_bounds__(256) void join(LinearArgs a, const float *parts, int splits) {
    const int64_t all = int64_t(a.T) * a.N;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        float v = parts[i];
        for (int s = 1; s < splits; ++s) v += parts[s * all + i];
        const int64_t t = i / a.N;
        put(a, t, int(i - t * a.N), v);
    }
}

// Sums of x over groups of GROUP values, [T, groups], and, of fp32 values (PIECES), their bf16 pieces, three
// rows of Kp with zeros behind K.  A lane takes 8 values, GROUP / 8 lanes a group.
template <int GROUP, bool PIECES>
__global__ __launch_bounds__(256) void survey(const void *x, int64_t stride, int T, int K, int Kp, float *totals,
                                              uint16_t *out) {
    const int lanes = Kp / 8;
    const int64_t all = int64_t(T) * lanes;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t t = i / lanes;
        const int k = int(i - t * lanes) * 8;
        float v[8] = {};
        if (k < K) {
            if constexpr (PIECES) {
                const float *from = static_cast<const float *>(x) + t * stride + k;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = from[e];
            } else {
                const uint4 w = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(x) + t * stride + k);
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[2 * e] = __uint_as_float(u[e] << 16);
                    v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
                }
            }
        }
        if constexpr (PIECES) {
            uint4 p[3];
            cut(v, p);
#pragma unroll
            for (int j = 0; j < 3; ++j) *reinterpret_cast<uint4 *>(out + (int64_t(j) * T + t) * Kp + k) = p[j];
        }
        float s = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        // 4, 8 or 16 lanes of a group, aligned, all of which are here: Kp is a multiple of 128
        s += __shfl_xor(s, 1);
        s += __shfl_xor(s, 2);
        if constexpr (GROUP >= 64) s += __shfl_xor(s, 4);
        if constexpr (GROUP >= 128) s += __shfl_xor(s, 8);
        if (totals && k % GROUP == 0) totals[t * (Kp / GROUP) + k / GROUP] = s;
    }
}

bool sizes_ok(int N, int K, int group) { return apex_linear_w4_bytes(N, K, group) != 0; }

int padded(int K) { return (K + kBlock - 1) / kBlock * kBlock; }

// Staged rows at most: with two buffers of sums, of four times the size for kMore, 64 KiB.
constexpr int stage_bytes(Rows rows) { return (rows == kMore ? 31 : 48) << 10; }

// Whether all of x goes to LDS, and in which rows.
bool stages(int T, int K, int pieces, Rows *rows) {
    *rows = pieces == 3 ? kPieces : T <= 4 ? kFew : kMore;
    return T <= (pieces == 3 ? 4 : 16) && int64_t(staged_rows(*rows, T)) * (padded(K) * 2 + kPad) <= stage_bytes(*rows);
}

template <int GROUP, int R, int ROWS>
void launch_few(const LinearArgs &a, hipStream_t st) {
    const size_t lds = staged_rows(ROWS, a.T) * (a.blocks * 256 + kPad) + 2 * 4 * (kWaves * R * 64 * (ROWS == kMore ? 4 : 1));
    const int tiles = (a.N + 16 * R - 1) / (16 * R);
    hipLaunchKernelGGL((linear_few<GROUP, R, ROWS>), dim3(std::min((tiles + 7) / 8 * 8, 768)), dim3(64 * kWaves), lds, st, a);
}

template <int GROUP, int R, int TT, int P>
void launch_some(const LinearArgs &a, hipStream_t st) {
    const int tiles = (a.N + 16 * R - 1) / (16 * R);
    hipLaunchKernelGGL((linear_some<GROUP, R, TT, P>), dim3((tiles + 7) / 8 * 8, (a.T + 16 * TT - 1) / (16 * TT)),
                       dim3(64 * kWaves), 0, st, a);
}

// Rows of the weights a workgroup takes: 16 while that leaves it a CU of its own, else 32.
bool narrow(int N) { return N <= 16 * 256; }

template <int GROUP, int R>
void launch(const LinearArgs &a, bool stage, Rows rows, hipStream_t st) {
    if (stage)
        rows == kFew      ? launch_few<GROUP, R, kFew>(a, st)
        : rows == kPieces ? launch_few<GROUP, R, kPieces>(a, st)
                          : launch_few<GROUP, R, kMore>(a, st);
    else if (a.pieces == 3)
        launch_some<GROUP, R, 1, 3>(a, st);
    else
        a.T <= 16 ? launch_some<GROUP, R, 1, 1>(a, st) : launch_some<GROUP, R, 2, 1>(a, st);
}

template <int GROUP>
void launch(const LinearArgs &a, bool stage, Rows rows, hipStream_t st) {
    narrow(a.N) ? launch<GROUP, 1>(a, stage, rows, st) : launch<GROUP, 2>(a, stage, rows, st);
}

bool is_type(int t) { return t == APEX_TYPE_FP32 || t == APEX_TYPE_BF16; }

// How a call is worked on.
struct Plan {
    enum { kStaged, kSome, kMany } kind;
    Rows rows;                       // kStaged
    int m_tiles, n_tiles, splits, share;     // kMany
    size_t pieces, totals, parts;    // bytes of the workspace, in this order
    size_t bytes() const { return pieces + totals + parts; }
};

constexpr size_t up256(size_t n) { return (n + 255) / 256 * 256; }

constexpr int kManyTokens = 128, kManyRows = 128;

Plan plan_of(int T, int N, int K, int group, int pieces) {
    Plan p{};
    const int Kp = padded(K), blocks = Kp / kBlock;
    if (stages(T, K, pieces, &p.rows)) {
        p.kind = Plan::kStaged;
        return p;
    }
    if (pieces == 3) p.pieces = up256(size_t(3) * T * Kp * 2);
    if (T <= (pieces == 3 ? 16 : 32)) {
        p.kind = Plan::kSome;
        return p;
    }
    p.kind = Plan::kMany;
    p.totals = up256(size_t(T) * (Kp / group) * 4);
    p.m_tiles = (T + kManyTokens - 1) / kManyTokens;
    p.n_tiles = (N + kManyRows - 1) / kManyRows;
    // shares of K until two workgroups a CU have work, of 4 blocks or more
    const int64_t tiles = int64_t(p.m_tiles) * p.n_tiles;
    const int fours = (blocks + 3) / 4, want = int(std::min<int64_t>(std::max<int64_t>(1, 512 / tiles), fours));
    p.share = (fours + want - 1) / want * 4;
    p.splits = (blocks + p.share - 1) / p.share;
    p.parts = p.splits > 1 ? up256(size_t(p.splits) * T * N * 4) : 0;
    return p;
}

}  // namespace

extern "C" size_t apex_linear_w4_workspace_bytes(int T, int N, int K, int group, int x_type) {
    if (T < 1 || T > APEX_MAX_STEP_TOKENS || !sizes_ok(N, K, group) || !is_type(x_type)) return 0;
    return plan_of(T, N, K, group, x_type == APEX_TYPE_FP32 ? 3 : 1).bytes();
}

extern "C" apex_status apex_linear_w4(const void *w, int N, int K, int group, const void *x, int x_type, int T,
                                      int64_t x_stride, const float *bias, const void *residual,
                                      int64_t residual_stride, void *y, int y_type, int64_t y_stride,
                                      void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const char *fn = "apex_linear_w4";
    APEX_REQUIRE(T >= 0, "%s: T=%d must be >= 0", fn, T);
    APEX_REQUIRE(sizes_ok(N, K, group),
                 "%s: N=%d (1 to 2^24), K=%d (multiple of 8 to 2^20) or group=%d (32, 64, 128) out of range", fn, N, K,
                 group);
    APEX_REQUIRE(is_type(x_type) && is_type(y_type), "%s: unknown type %d or %d", fn, x_type, y_type);
    const int per = x_type == APEX_TYPE_FP32 ? 4 : 8;
    APEX_REQUIRE(x_stride >= K && x_stride % per == 0, "%s: x_stride=%lld must be a multiple of %d and at least %d", fn,
                 static_cast<long long>(x_stride), per, K);
    APEX_REQUIRE(y_stride >= N && (!residual || residual_stride >= N), "%s: rows of %d values overlap", fn, N);
    if (T > APEX_MAX_STEP_TOKENS)
        return apex::fail(APEX_E_UNSUPPORTED, "%s: T=%d exceeds %d", fn, T, APEX_MAX_STEP_TOKENS);
    if (x_stride > (1 << 23))      // offsets in a tile of 128 rows are 32-bit numbers of bytes
        return apex::fail(APEX_E_UNSUPPORTED, "%s: x_stride=%lld exceeds 2^23", fn, static_cast<long long>(x_stride));
    if (T == 0) return APEX_OK;
    APEX_REQUIRE(w && x && y, "%s: NULL pointer", fn);
    APEX_REQUIRE(apex::aligned16(w) && apex::aligned16(x) && apex::aligned16(y) && apex::aligned16(bias) &&
                     apex::aligned16(residual) && apex::aligned16(workspace),
                 "%s: pointers must be 16-byte aligned", fn);
    APEX_REQUIRE(residual != y || residual_stride == y_stride, "%s: y is the residual with another stride", fn);
    const int Kp = padded(K), pieces = x_type == APEX_TYPE_FP32 ? 3 : 1;
    const Plan plan = plan_of(T, N, K, group, pieces);
    const size_t need = plan.bytes();
    APEX_REQUIRE(need == 0 || workspace, "%s: NULL workspace", fn);
    if (workspace_bytes < need)
        return apex::fail(APEX_E_CAPACITY, "%s: workspace of %zu bytes, %zu needed", fn, workspace_bytes, need);
    LinearArgs a{static_cast<const uint8_t *>(w),
                 reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(w) + size_t(N) * (Kp / 2)),
                 static_cast<const uint16_t *>(x), x_stride, 0, K, bias, residual, y, residual_stride, y_stride, N, T,
                 Kp / kBlock, pieces, y_type == APEX_TYPE_FP32};
    char *ws = static_cast<char *>(workspace);
    float *totals = reinterpret_cast<float *>(ws + plan.pieces);
    if (plan.kind != Plan::kStaged && (pieces > 1 || plan.kind == Plan::kMany)) {
        uint16_t *out = reinterpret_cast<uint16_t *>(ws);
        const int64_t items = int64_t(T) * (Kp / 8);
        const dim3 grid(unsigned(std::min<int64_t>((items + 255) / 256, 1 << 16)));
        const auto f = pieces > 1 ? (group == 32 ? survey<32, true> : group == 64 ? survey<64, true> : survey<128, true>)
                                  : (group == 32 ? survey<32, false> : group == 64 ? survey<64, false> : survey<128, false>);
        hipLaunchKernelGGL(f, grid, dim3(256), 0, stream, x, x_stride, T, K, Kp, plan.totals ? totals : nullptr, out);
        APEX_HIP(hipGetLastError());
        if (pieces > 1) {
            a.x = out;
            a.x_stride = Kp;
            a.x_piece = int64_t(T) * Kp;
            a.x_cols = Kp;
        }
    }
    if (plan.kind == Plan::kMany) {
        float *parts = plan.splits > 1 ? reinterpret_cast<float *>(ws + plan.pieces + plan.totals) : nullptr;
        const ManyArgs m{a, totals, parts, plan.m_tiles, plan.n_tiles, plan.splits, plan.share};
        const int64_t all = int64_t(plan.m_tiles) * plan.n_tiles * plan.splits;
        const auto f = group == 32 ? linear_many<32, 4, 4> : group == 64 ? linear_many<64, 4, 4> : linear_many<128, 4, 4>;
        hipLaunchKernelGGL(f, dim3(unsigned((all + 7) / 8 * 8)), dim3(kManyThreads), 0, stream, m);
        if (parts) {
            APEX_HIP(hipGetLastError());
            hipLaunchKernelGGL(join, dim3(unsigned(std::min<int64_t>((int64_t(T) * N + 255) / 256, 4096))), dim3(256), 0,
                               stream, a, parts, plan.splits);
        }
    } else {
        const bool stage = plan.kind == Plan::kStaged;
        group == 32   ? launch<32>(a, stage, plan.rows, stream)
        : group == 64 ? launch<64>(a, stage, plan.rows, stream)
                      : launch<128>(a, stage, plan.rows, stream);
    }
    APEX_HIP(hipGetLastError());
    return APEX_OK;
}
