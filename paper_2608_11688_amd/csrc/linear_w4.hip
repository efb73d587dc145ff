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
#include <type_traits>

#include "common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 128;         // codes of a row that stand together, 64 bytes
constexpr int kCUs = 256;

struct LinearArgs {
    const uint8_t *codes;
    const uint32_t *words;
    const uint16_t *x;              // bf16, or fp32; for linear_many bf16, or the pieces of fp32
    int64_t x_stride, x_piece;      // in values: of rows; for linear_many of the pieces of 128 values along K
    int x_cols;                     // values of a row of x that there are (a multiple of 8), but for linear_many
    const float *bias;
    const void *residual;
    void *y;
    int64_t residual_stride, y_stride;
    int N, T, blocks;               // blocks of kBlock codes in a row
    int pieces;                     // of x: 1 (bf16) or 3 (fp32)
    bool y32;
    int ways;                       // linear_some: of a workgroup's wavefronts along K, a power of two
    int token_groups;               // linear_some: of a workgroup's tokens
    bool by_tokens;                 // linear_some: which of the two an XCD has an eighth of
};

// Codes 2 i and 2 i + 1 of a word as bf16 pairs 16 + q.
__device__ __forceinline__ bf16x8 widen(uint32_t w) {
    uint32_t base = 0x41804180u;
    asm("" : "+v"(base));       // in a vector register: an instruction takes one scalar operand, the mask
    uint4 b;
    b.x = ((w << 3) & 0x00780078u) | base;
    b.y = ((w >> 1) & 0x00780078u) | base;
    b.z = ((w >> 5) & 0x00780078u) | base;
    b.w = ((w >> 9) & 0x00780078u) | base;
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

// Four values of one token from row n of the weights on; rows of y and of the residual may begin at any value.
__device__ __forceinline__ void put_row(const LinearArgs &a, int64_t t, int n, floatx4 v) {
    if (t >= a.T || n >= a.N) return;
    if (n + 4 > a.N) {                                 // the last values of a row
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (n + i < a.N) put(a, t, n + i, v[i]);
        return;
    }
    if (a.bias) {
        const float4 b = *reinterpret_cast<const float4 *>(a.bias + n);
        v[0] += b.x, v[1] += b.y, v[2] += b.z, v[3] += b.w;
    }
    const int64_t to = t * a.y_stride + n, from = t * a.residual_stride + n;
    if (a.y32) {
        if (a.residual) {
            floatx4 r;
            __builtin_memcpy(&r, static_cast<const float *>(a.residual) + from, 16);
            v += r;
        }
        __builtin_memcpy(static_cast<float *>(a.y) + to, &v, 16);
    } else {
        if (a.residual) {
            uint2 r;
            __builtin_memcpy(&r, static_cast<const uint16_t *>(a.residual) + from, 8);
            v[0] += __uint_as_float(r.x << 16), v[1] += __uint_as_float(r.x & 0xffff0000u);
            v[2] += __uint_as_float(r.y << 16), v[3] += __uint_as_float(r.y & 0xffff0000u);
        }
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = static_cast<__bf16>(v[i]);
        __builtin_memcpy(static_cast<uint16_t *>(a.y) + to, &y, 8);
    }
}

// A lane's values of row n of the weights and 4 tokens from t on.  4 lanes (n a multiple of 4 in the first) first trade
// places, so that each has 4 values of one token, side by side.
template <int CTRL>
__device__ __forceinline__ float quad(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ void put_four(const LinearArgs &a, int64_t t, int n, floatx4 v) {
    // lane l of the four, value i -> lane i, value l: by halves (l ^ 2 and i ^ 2), then by ones
    const int l = threadIdx.x & 3;
    const float p0 = quad<0x4e>(l & 2 ? v[0] : v[2]), p1 = quad<0x4e>(l & 2 ? v[1] : v[3]);
    if (l & 2) v[0] = p0, v[1] = p1;
    else v[2] = p0, v[3] = p1;
    const float q0 = quad<0xb1>(l & 1 ? v[0] : v[1]), q1 = quad<0xb1>(l & 1 ? v[2] : v[3]);
    if (l & 1) v[0] = q0, v[2] = q1;
    else v[1] = q0, v[3] = q1;
    t += l;
    n -= l;
    put_row(a, t, n, v);
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

// The words of a row's PER groups in a block, of which lane quarter q has loaded that of group q mod PER.
template <int PER>
__device__ __forceinline__ void words_of(uint32_t word, uint32_t (&w)[PER]) {
    if constexpr (PER == 1) {
        w[0] = word;
    } else if constexpr (PER == 2) {
        const auto v = __builtin_amdgcn_permlane16_swap(word, word, false, false);
        w[0] = v[0], w[1] = v[1];
    } else {
        const auto h = __builtin_amdgcn_permlane32_swap(word, word, false, false);
        const auto lo = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);
        w[0] = lo[0], w[1] = lo[1], w[2] = hi[0], w[3] = hi[1];
    }
}

// The codes and the group words of a block of 16 R rows, D blocks ahead of their use.  Descriptors end
// with the tile's rows, and are empty for blocks that are not there: such loads move nothing.
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
};

// Of those words two, of groups j and j + 1, made anew at each call.
__device__ __forceinline__ void two_words(uint32_t word, int j, uint32_t (&w)[4]) {
    asm volatile("" : "+v"(word));
    const auto h = __builtin_amdgcn_permlane32_swap(word, word, false, false);
    const auto v = __builtin_amdgcn_permlane16_swap(h[j / 2], h[j / 2], false, false);
    w[j] = v[0], w[j + 1] = v[1];
}

// How the rows of x stand in the 16 rows of a matrix instruction, whose lane holds rows 4 q + i, i =
// 0..3, of the result (q = lane / 16):
enum Rows {
    kFew,       // up to 4 rows of bf16, row q at i = 0
    kPieces     // up to 4 rows of fp32, the pieces of row q at i = 0..2, added at the end
};
constexpr int staged_rows(int rows, int T) { return rows == kPieces ? 3 * T : T; }

// Up to 4 rows: all of x goes to LDS first, at most stage_bytes() of it, and the weights are read once, by workgroups that
// stay.  The wavefronts join their sums in LDS in a fixed order.  A long stream is bound by memory: 4 rows through
// 32768 x 4096 in groups of 32, 84 MB, 14.6 us, 5.8 TB/s, where the last-level cache holds the weights (a kernel that only reads 13.3),
// 19 from memory, 4.4 TB/s (15.4).  A short one by the way of a launch, x and the first weights one behind the other: one fp32
// row through 6144 x 4096, 13.4 MB, 5.9 us, through 2048 x 1024 3.3.
template <int GROUP, int R, int ROWS>
__global__ __launch_bounds__(64 * kWaves) void linear_few(LinearArgs a) {
    extern __shared__ uint4 lds[];
    constexpr int PER = kBlock / GROUP, STEPS = GROUP / 32;
    constexpr int NI = ROWS == kFew ? 1 : 3;           // results of a lane
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
    const int row = ROWS == kFew ? min(col >> 2, a.T - 1) : 3 * min(col >> 2, a.T - 1) + min(col & 3, 2);
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
            for (int r = 0; r < R; ++r) words_of<PER>(next.word[r], words[r]);
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
            float *mine = part + flip * (kWaves * R * 64);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float v = sum[r][0];
                if constexpr (ROWS == kPieces) v = sum[r][2] + sum[r][1] + v;
                mine[(wave * R + r) * 64 + lane] = v;
            }
            __syncthreads();
            const int e = threadIdx.x;
            if (e < R * 64) {
                float v = mine[e];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) v += mine[w * (R * 64) + e];
                const int t = (e & 63) >> 4, n = now.tile * 16 * R + 16 * (e >> 6) + (e & 15);
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

// Some rows, in tiles of 16 TT, bf16 or fp32 (P = 3 pieces).  A workgroup takes 16 R rows of the weights; each wavefront
// brings the part of x that belongs to its next block, 16 TT rows of 256 or 512 bytes, by loads of whole lines, fp32 values
// cut into their pieces on the way, into LDS of its own, and reads it as the matrix instructions want it.  Within
// a row 16-byte chunks stand in the place c ^ (row mod 16), so that 16 rows' chunks meet 64 banks.  Bound by a block's
// way, loads, LDS and matrix instructions, of which a wavefront has one on its way ahead: 32 rows through 4096 x 4096
// 8.2 to 9.4 us, 4 blocks each.  Two ahead were no faster (16384 x 4096 16.5 and 19.4: fewer workgroups on a CU).
template <int GROUP, int R, int TT, int P>
__global__ __launch_bounds__(64 * kWaves) void linear_some(LinearArgs a) {
    constexpr int PER = kBlock / GROUP, STEPS = GROUP / 32, LOADS = 4 * TT, PARTS = P == 3 ? 2 : 1;   // of 16 bytes for 8 values
    constexpr int STAGE = 4 * TT * P * 64, OUT = R * TT * 64;
    __shared__ uint4 lds[kWaves * (STAGE > OUT ? STAGE : OUT)];       // x, then the sums
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
    // an XCD has an eighth of the work, of the rows of the weights, as in Walk, or of the tokens, whichever are more bytes: 1086
    // fp32 rows through 144 x 7624 31 us by tokens and 69 by rows, 2000 bf16 rows through 60 x 6400 10 and 30
    const int tiles = (a.N + 16 * R - 1) / (16 * R), all = tiles * a.token_groups, per = (all + 7) / 8;
    const int unit = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if (unit >= all) return;
    const int n_tile = a.by_tokens ? unit % tiles : unit / a.token_groups;
    const int group = a.by_tokens ? unit / tiles : unit % a.token_groups;
    const int n0 = n_tile * 16 * R;
    // wavefronts along K, and of tokens the tiles of the others
    const int ways = a.ways, along = wave & (ways - 1);
    const int t0 = (group * (kWaves / ways) + wave / ways) * 16 * TT;
    uint4 x[LOADS][PARTS];
    Block<GROUP, R> next;
    // load i of a block: row 4 i + quarter, chunk `col` of 8 values
    const auto load_x = [&](int b) {
        const int k = b * kBlock + 8 * col;
        const bool there = k < a.x_cols;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int t = min(t0 + 4 * i + quarter, a.T - 1);
            const uint4 *from = reinterpret_cast<const uint4 *>(a.x + (t * a.x_stride + (there ? k : 0)) * PARTS);
#pragma unroll
            for (int h = 0; h < PARTS; ++h) {
                x[i][h] = from[h];
                if (!there) x[i][h] = make_uint4(0u, 0u, 0u, 0u);
            }
        }
    };
    char *mine = reinterpret_cast<char *>(lds) + wave * (STAGE * 16);
    floatx4 sum[R][TT] = {};
    const int first = t0 < a.T ? along : a.blocks;     // none for a tile that is not there
    load_x(first);
    next.load(a, n0, first, first < a.blocks, lane);
    for (int b = first; b < a.blocks; b += ways) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int row = 4 * i + quarter, at = row * 256 + 16 * (col ^ (row & 15));
            if constexpr (P == 1) {
                *reinterpret_cast<uint4 *>(mine + at) = x[i][0];
            } else {
                uint4 piece[3];
                cut({__uint_as_float(x[i][0].x), __uint_as_float(x[i][0].y), __uint_as_float(x[i][0].z), __uint_as_float(x[i][0].w),
                     __uint_as_float(x[i][1].x), __uint_as_float(x[i][1].y), __uint_as_float(x[i][1].z), __uint_as_float(x[i][1].w)},
                    piece);
#pragma unroll
                for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4 *>(mine + p * (TT * 4096) + at) = piece[p];
            }
        }
        const Block<GROUP, R> now = next;
        load_x(b + ways);
        next.load(a, n0, b + ways, b + ways < a.blocks, lane);
        uint32_t words[R][PER];
#pragma unroll
        for (int r = 0; r < R; ++r) words_of<PER>(now.word[r], words[r]);
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
                    for (int i = 0; i < 4; ++i) {
                        float s = sum[r][tt][i];
                        w.add(s, prod[r][tt][i], total[tt][i]);
                        sum[r][tt][i] = s;
                    }
            }
        }
    }
    const auto out = [&](int t, int i, floatx4 v) {        // value i / 64 of lane i % 64
        put_four(a, t + 16 * ((i >> 6) % TT) + 4 * ((i & 63) >> 4), n0 + 16 * ((i >> 6) / TT) + (i & 15), v);
    };
    if (ways == 1) {
#pragma unroll
        for (int i = 0; i < R * TT; ++i) out(t0, i * 64 + lane, sum[i / TT][i % TT]);
        return;
    }
    __syncthreads();
    floatx4 *part = reinterpret_cast<floatx4 *>(lds);
#pragma unroll
    for (int i = 0; i < R * TT; ++i) part[wave * OUT + i * 64 + lane] = sum[i / TT][i % TT];
    __syncthreads();
    for (int e = along * 64 + lane; e < OUT; e += ways * 64) {
        const floatx4 *from = part + (wave - along) * OUT + e;
        floatx4 v = from[0];
#pragma unroll 1
        for (int w = 1; w < ways; ++w) v += from[w * OUT];
        out(t0, e, v);
    }
}

// Many rows.  A workgroup of 8 wavefronts takes a tile of 16 TT tokens by 256 rows of the weights, each
// wavefront all of the tokens by 32 rows, so that no code is widened twice; a step is a block of 128 codes
// and one piece of x.  x and codes go from memory to LDS directly (chunks of x placed as in
// linear_some) into three stages, from there to registers a quarter of a step ahead.  The one barrier
// of a step stands before its last quarter, when all of the stage has been read: the next step's first
// values are read behind it, and the stage takes the loads of the step after the next two.
// Of a group the zero points' half, (16 + z) sum x, is taken off the sums of (16 + q) x before these are scaled and added, on the
// matrix cores, from sums of x that a launch before has made.  The halves are 24 |x| times the group's size where x has a mean,
// which the difference has not: added up over a row and subtracted at its end they lose digits with its length, an error (2-norm)
// of 8.5e-6 for rows of mean 1 and deviation 0.3 through 2816 x 4104 in groups of 32, 3.0e-5 through 14337 x 16384; taken
// off group by group 1.1e-7 and 2.1e-7.  It takes 16 to 64 matrix instructions a step: 2048 rows through 6144 x 4096 in
// groups of 128, 64 and 32 110, 128 and 151 us without and 120, 135 and 171 with them.  Of fp32 rows it is taken
// off the first pieces' sums and off the others' apart: together, rounded at the size of the first, they came to 4.9e-6, apart to 1.6e-7.
//
// There is a workgroup a CU.  The last tiles, fewer than that, are cut along K into shares, whose sums go
// to memory in the order of the lanes and are joined by another launch.
//
// A step of 128 tokens in groups of 128, 80 matrix instructions and about 170 of the vector unit a wavefront, takes 2.2 us: widening
// codes and scaling sums fill the time that the matrix cores have free, which are busy 49 % of it, at 2.1 GHz.  2048 rows
// through 6144 x 4096: 120 us, 859 TFLOP/s (a library product of bf16 weights of this size 84 to 103).
#define APEX_LDS __attribute__((address_space(3)))
constexpr int kManyThreads = 512, kManyRows = 256, kManySlots = 256;
constexpr int kManyR = 2;                       // tiles of 16 rows of a wavefront

// Tokens for which sums of x over groups are kept.
__host__ __device__ constexpr int tokens32(int T) { return (T + 31) / 32 * 32; }

struct ManyArgs {
    LinearArgs a;
    const uint8_t *totals;          // sums of x over groups, negated, in pieces (sum_groups)
    float *parts;                   // of the tiles that are cut: [tile][split][tile's values]
    int m_tiles, tiles, whole;      // the first `whole` tiles are not cut
    int splits, share;              // blocks of a share
};

// Keeps the additions where they stand: put off, as they may be for all of a loop's body, they leave the products of
// every group in registers.
__device__ __forceinline__ void settle(floatx4 &v) { asm volatile("" : "+v"(v)); }

constexpr int vmcnt_only(int n) { return 0x0f70 | (n & 15) | (n >> 4 << 14); }   // the s_waitcnt operand

// The three bf16 pieces of an fp32 value whose sum it is, in the upper halves of words.
__device__ __forceinline__ void pieces_of(float v, uint32_t (&p)[3]) {
    const float rest = v - __uint_as_float(__float_as_uint(v) & 0xffff0000u);
    p[0] = __float_as_uint(v), p[1] = __float_as_uint(rest);
    p[2] = __float_as_uint(rest - __uint_as_float(p[1] & 0xffff0000u));
}
__device__ __forceinline__ uint32_t uppers(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

// A group's zero points' half, -(16 + z) sum x, as a matrix instruction: the left operand has in every lane quarter the pieces of -sum x,
// three places and a zero, of a token in one tile and of its neighbour 16 on, all of them finite; the right one for either tile 16
// thrice in quarter 0 and z thrice in quarter 1 against its half of the places, and nothing in the others. The shape is that of the
// instructions whose sums it goes into: behind one of another shape, two or three instructions back, sums have come
// out wrong.
struct Zeros {
    uint32_t sixteen, pick;         // the words of 16, by lane quarter, and which bytes of a group's word those of z are
    __device__ __forceinline__ explicit Zeros(int quarter)
        : sixteen(quarter == 0 ? 0x41804180u : 0u), pick(quarter == 1 ? 0x01000100u : 0x0c0c0c0cu) {}
    __device__ __forceinline__ void right(uint32_t word, bf16x8 (&of)[2]) const {
        const uint32_t z = __builtin_amdgcn_perm(word, word, pick) | sixteen, last = z & 0xffffu;
        of[0] = __builtin_bit_cast(bf16x8, make_uint4(z, last, 0u, 0u));
        of[1] = __builtin_bit_cast(bf16x8, make_uint4(0u, 0u, z, last));
    }
};

template <int GROUP, int TT, int P>
__global__ __launch_bounds__(kManyThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void linear_many(ManyArgs m) {
    constexpr int PER = kBlock / GROUP, STEPS = GROUP / 32, BM = 16 * TT, R = kManyR;
    constexpr int XLOADS = BM / 32, WLOADS = 2;        // of a wavefront a step: 4 rows of x, 16 rows of codes each
    constexpr int CODES = kManyRows * 64, SUMS = BM * PER * 8;     // bytes of a stage
    constexpr int SUM_PITCH = PER * 8;                  // of a token
    constexpr int SUM_PARTS = P == 1 ? 1 : 2;          // of a block
    constexpr int SUM_WAVES = (SUMS + 1023) / 1024;    // wavefronts that load the sums of x; the others' load goes behind them
    constexpr int W = CODES + (SUM_WAVES + 1) * 1024;
    __shared__ __attribute__((aligned(1024))) uint8_t x0[BM * 256], x1[BM * 256], x2[BM * 256], w0[W], w1[W], w2[W];
    const LinearArgs &a = m.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    // units, a tile or a share of one, in the order of the launch's rounds; of a round an eighth to each XCD
    const int units = m.whole + (m.tiles - m.whole) * m.splits;
    const int round = blockIdx.x / kManySlots, in_round = min(units - round * kManySlots, kManySlots);
    const int slot = blockIdx.x % kManySlots, per = (in_round + 7) / 8;
    if ((slot >> 3) >= per || (slot & 7) * per + (slot >> 3) >= in_round) return;
    const int unit = round * kManySlots + (slot & 7) * per + (slot >> 3);
    const bool cut_up = unit >= m.whole && m.splits > 1;
    const int rest = cut_up ? unit - m.whole : 0, split = cut_up ? rest % m.splits : 0;
    const int tile = cut_up ? m.whole + rest / m.splits : unit;
    const int n_tile = tile / m.m_tiles, t0 = (tile - n_tile * m.m_tiles) * BM, n0 = n_tile * kManyRows;
    const int nw = n0 + wave * (16 * R);
    const int first = split * m.share, last = cut_up ? min(first + m.share, a.blocks) : a.blocks;

    // x: rows 4 i + quarter of this wavefront's part of the tile, the chunk for place `col`; past T nothing
    const int mine = wave * (BM / 8), x_bytes = min(BM, a.T - t0) * 256;
    const int from = (mine + quarter) * 256 + 16 * (col ^ ((mine + quarter) & 15));
    const int pitch = a.blocks * 64, w_rows = min(kManyRows, a.N - n0);
    const int from_w = (wave * 32 + (lane >> 2)) * pitch + 16 * (lane & 3);
    const int64_t sums_pitch = int64_t(tokens32(a.T)) * SUM_PITCH;       // of a block's part
    const int sum_bytes = wave < SUM_WAVES ? min(BM, tokens32(a.T) - t0) * SUM_PITCH : 0, from_sums = wave * 1024 + lane * 16;
    const int to_sums = CODES + min(wave, SUM_WAVES) * 1024;
    // the step whose loads go out: how many are left, x, codes, sums.  P stages are a block.
    int ahead = (last - first) * P;
    const uint16_t *x_ahead = a.x + first * (P * a.x_piece) + t0 * a.x_stride;
    const uint8_t *w_ahead = a.codes + int64_t(n0) * pitch + first * 64;
    const uint8_t *sums_ahead = m.totals + first * SUM_PARTS * sums_pitch + t0 * SUM_PITCH;
    // as many loads whatever the step: past the last one they move nothing
    const auto load = [&](auto stage, uint8_t *x, uint8_t *w) {
        const auto codes = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(w_ahead), 0,
                                                             ahead > 0 ? (w_rows - 1) * pitch + 64 : 0, 0x00027000);
        const auto xs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(x_ahead), 0, ahead > 0 ? x_bytes : 0,
                                                          0x00027000);
#pragma unroll
        for (int i = 0; i < WLOADS; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(codes, (APEX_LDS void *)(w + (wave * 32 + 16 * i) * 64), 16,
                                                     from_w + 16 * i * pitch, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < XLOADS; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xs, (APEX_LDS void *)(x + (mine + 4 * i) * 256), 16, (from ^ 64 * i) + i * 1024, 0,
                                                     0, 0);
        --ahead;
        x_ahead += a.x_piece;                          // pieces of a block, and blocks, one behind the other
        if constexpr (stage % P == P - 1) w_ahead += 64;
    };
    // Sums of x for a stage: of x's first piece, and of the others together (with the second)
    int sums_left = (last - first) * SUM_PARTS;
    const auto load_sums = [&](uint8_t *w) {
        const auto sums = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(sums_ahead), 0, sums_left > 0 ? sum_bytes : 0,
                                                            0x00027000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(sums, (APEX_LDS void *)(w + to_sums), 16, from_sums, 0, 0, 0);
        --sums_left;
        sums_ahead += sums_pitch;
    };
    const int word_bytes = ((PER - 1) * a.N + min(a.N - nw, 16 * R)) * 4;      // of a block's words, this wavefront's rows
    const uint32_t *words_at = a.words + int64_t(first) * PER * a.N + nw;
    int words_left = nw < a.N ? last - first : 0;
    const auto load_words = [&](uint32_t (&to)[R]) {   // of the next block
        const auto words = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t *>(words_at), 0, words_left > 0 ? word_bytes : 0,
                                                             0x00027000);
#pragma unroll
        for (int r = 0; r < R; ++r)
            to[r] = __builtin_amdgcn_raw_buffer_load_b32(words, (quarter % PER * a.N + 16 * r + col) * 4, 0, 0);
        words_at += PER * a.N, --words_left;
    };
    constexpr int HT = TT / 2;
    bf16x8 v[2][HT];                                   // of half h of the tokens in v[h]
    bf16x8 sum_x[HT / 2];                              // of a group, of tiles of half of the tokens
    uint4 code_next[R];
    const int at_x = col * 256 + 16 * (quarter ^ col);
    const auto read_x = [&](const uint8_t *x, int j, int h) {
        int at = at_x;
        asm volatile("" : "+v"(at));                   // an exclusive or here instead of four registers for the four quarters
#pragma unroll
        for (int i = 0; i < HT; ++i) v[h][i] = *reinterpret_cast<const bf16x8 *>(x + (h * HT + i) * 4096 + (at ^ 64 * j));
    };
    const auto read_sums = [&](const uint8_t *w, int g, int h, int lo, int hi) {
#pragma unroll
        for (int i = lo / 2; 2 * i < hi; ++i)
            sum_x[i] = *reinterpret_cast<const bf16x8 *>(w + CODES + (((h * HT / 2 + i) * PER + g) * 16 + col) * 16);
    };
    const auto read_codes = [&](const uint8_t *w) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            code_next[r] = *reinterpret_cast<const uint4 *>(w + (wave * 32 + 16 * r + col) * 64 + 16 * quarter);
    };

    const Zeros zeros(quarter);
    floatx4 sum[R][TT] = {}, prod[R][TT] = {};
    uint32_t word[3][R];                               // P == 1: of each stage's block; else of this block and the next one
    bf16x8 q_next[R];
    float s_before[R] = {};                            // of the group before, whose second half is still to be added
    const auto add = [&](int h, int r, float s) {
#pragma unroll
        for (int i = h * HT; i < (h + 1) * HT; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[r][i][e] = fmaf(s, prod[r][i][e], sum[r][i][e]);
            settle(sum[r][i]);
        }
    };
    // One step; its stage, the next step's.  Eight phases: a quarter of the block's codes by half of the tokens.  What the
    // vector unit does in a phase is for other values than its matrix instructions': the codes of the next
    // quarter are widened, and a group's sums scaled, half a quarter later.  The zero points' half of a group's sums goes in
    // halfway through its codes.
    const auto step = [&](auto stage, uint8_t *x, uint8_t *w, const uint8_t *x_next, uint8_t *w_next, uint8_t *w_last) {
        constexpr bool SUMS = stage % P < 2;
        constexpr int SPREAD = STEPS == 4 ? 2 : 1;     // of groups of 64 both in one go: registers
        uint4 code[R];
        uint32_t words[R][PER];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            code[r] = code_next[r];
            if constexpr (PER < 4) words_of<PER>(word[P == 1 ? stage : 0][r], words[r]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x8 q[R];
#pragma unroll
            for (int r = 0; r < R; ++r) q[r] = q_next[r];
            if constexpr (PER == 4) {
                if (j % 2 == 0) {                      // words of two groups at a time: registers
#pragma unroll
                    for (int r = 0; r < R; ++r) two_words(word[P == 1 ? stage : 0][r], j, words[r]);
                }
            }
            // the tiles of a half whose zero points' half goes in now: the sums' own first part, then the second
            const int part = j % STEPS - (STEPS - 1) / 2, lo = max(part, 0) * (HT / SPREAD);
            const int hi = SUMS && part >= 0 && part < SPREAD ? lo + HT / SPREAD : lo;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                __builtin_amdgcn_sched_barrier(0);
                const bool at_end = j == 3 && h == 1;
                if (at_end) {
                    // the next step's loads have landed; those of the one behind it, the last that went
                    // out, may be on their way
                    __builtin_amdgcn_s_waitcnt(vmcnt_only(XLOADS + WLOADS));
                    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                    read_codes(w_next);
                }
                read_sums(w, j / STEPS, h, lo, hi);
                if (!at_end) {
                    read_x(x, j + h, 1 - h);
                } else {
                    read_x(x_next, 0, 0);
                    if constexpr (P == 1) {
                        load_words(word[(stage + 2) % 3]);
                    } else if constexpr (stage == 0) {
                        load_words(word[1]);
                    } else if constexpr (stage == 2) {
#pragma unroll
                        for (int r = 0; r < R; ++r) word[0][r] = word[1][r];
                    }
                    if constexpr ((stage + 2) % 3 % P < 2) load_sums(w_last);
                    load(stage, x, w);
                }
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < HT; ++i)
                        prod[r][h * HT + i] = mfma(v[h][i], q[r], j % STEPS == 0 ? floatx4{} : prod[r][h * HT + i]);
                if (lo < hi) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        bf16x8 z[2];
                        zeros.right(words[r][j / STEPS], z);
#pragma unroll
                        for (int i = lo; i < hi; ++i) prod[r][h * HT + i] = mfma(sum_x[i / 2], z[i & 1], prod[r][h * HT + i]);
                    }
                }
                if (h == 0 && j % STEPS == 0) {
#pragma unroll
                    for (int r = 0; r < R; ++r) add(1, r, s_before[r]);
                }
                if (h == 1) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        q_next[r] = widen(j < 3 ? word_of(code[r], j + 1) : code_next[r].x);
                        if ((j + 1) % STEPS == 0) {    // a group ends
                            s_before[r] = __uint_as_float(words[r][j / STEPS] & 0xffff0000u);
                            add(0, r, s_before[r]);
                        }
                    }
                }
            }
        }
    };
    constexpr std::integral_constant<int, 0> k0;
    constexpr std::integral_constant<int, 1> k1;
    constexpr std::integral_constant<int, 2> k2;
    load_words(word[0]);
    if constexpr (P == 1) load_words(word[1]);
    load_sums(w0);
    load_sums(w1);
    load(k0, x0, w0);
    load(k1, x1, w1);
    load(k2, x2, w2);
    __builtin_amdgcn_s_waitcnt(vmcnt_only(2 * (XLOADS + WLOADS)));
    asm volatile("s_barrier" ::: "memory");
    read_codes(w0);
    read_x(x0, 0, 0);
#pragma unroll
    for (int r = 0; r < R; ++r) q_next[r] = widen(code_next[r].x);
    int left = (last - first) * P;
    for (; left >= 3; left -= 3) {
        step(k0, x0, w0, x1, w1, w2);
        step(k1, x1, w1, x2, w2, w0);
        step(k2, x2, w2, x0, w0, w1);
    }
    if constexpr (P == 1) {
        if (left >= 1) step(k0, x0, w0, x1, w1, w2);
        if (left >= 2) step(k1, x1, w1, x2, w2, w0);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) add(1, r, s_before[r]);
    __builtin_amdgcn_s_waitcnt(0x0f70);                // no load into LDS outlives the workgroup

    // what follows starts from a lane number of its own, so that none of its addresses is made, and kept in registers,
    // before the loop
    int lane_after = lane;
    asm volatile("" : "+v"(lane_after));
    if (cut_up) {
        floatx4 *to = reinterpret_cast<floatx4 *>(m.parts) + int64_t(rest) * (BM * kManyRows / 4) + lane_after;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) to[((wave * R + r) * TT + tt) * 64] = sum[r][tt];
        return;
    }
    // results by way of LDS, a token's 256 values side by side; 16 tokens in the place of 16 KiB of a stage, rows of 4
    // tokens 16 banks apart
    const auto place = [&](int tt) {
        uint8_t *at = TT == 4 ? (tt == 0 ? x0 : tt == 1 ? x1 : tt == 2 ? x2 : w0)
                              : (tt < 2 ? x0 : tt < 4 ? x1 : tt < 6 ? x2 : tt == 6 ? w0 : w1);
        return reinterpret_cast<float *>(at + (TT == 8 && tt < 6 ? (tt & 1) * 16384 : 0));
    };
    const int col_after = lane_after & 15, quarter_after = lane_after >> 4;
    __syncthreads();                                   // the last stage has been read
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                place(tt)[(4 * quarter_after + i) * 256 + ((wave * 32 + 16 * r + col_after) ^ (16 * quarter_after))] =
                    sum[r][tt][i];
    __syncthreads();
    constexpr int ROWS = BM / 8;                       // tokens of a wavefront, within one of those places
    const float *mine_out = place(wave * ROWS / 16) + wave * ROWS % 16 * 256;
#pragma unroll 4
    for (int i = 0; i < ROWS; ++i) {
        const int row = wave * ROWS % 16 + i, t = t0 + wave * ROWS + i;
        const floatx4 v = *reinterpret_cast<const floatx4 *>(mine_out + i * 256 + ((4 * lane_after) ^ (16 * (row >> 2))));
        if (t < a.T && n0 + 4 * lane_after < a.N) put_row(a, t, n0 + 4 * lane_after, v);
    }
}

// The shares of the tiles that were cut, in order.  A workgroup takes 4 tokens, its threads a row of the weights each.  Memory
// and a launch: 33.5 MB of shares in 8 us.
template <int TT>
__global__ __launch_bounds__(kManyRows) void join(ManyArgs m) {
    constexpr int values = 16 * TT * kManyRows / 4;    // of 4 tokens
    const int rest = blockIdx.x / (4 * TT), tt = blockIdx.x % (4 * TT) / 4, quarter = blockIdx.x % 4, n = threadIdx.x;
    const floatx4 *from = reinterpret_cast<const floatx4 *>(m.parts) + int64_t(rest) * m.splits * values +
                          ((n / 16 * TT + tt) * 64 + 16 * quarter + n % 16);
    floatx4 v = from[0];
#pragma unroll 4
    for (int s = 1; s < m.splits; ++s) v += from[int64_t(s) * values];
    const int tile = m.whole + rest, n_tile = tile / m.m_tiles;
    put_four(m.a, (tile - n_tile * m.m_tiles) * (16 * TT) + 16 * tt + 4 * quarter, n_tile * kManyRows + n, v);
}

// x as bf16 (PIECES: fp32 values as three pieces) in the order in which it is read, [block of 128 values][piece][T][128], zeros behind
// K, and its negated sums over groups of GROUP values, [block][part][32 tokens][group of the block][16 tokens][tile of 16] of 8
// bytes, three bf16 pieces and a zero; of fp32 rows a part of the first pieces and one of what is left of the values.  Two tokens' sums
// stand in one operand, so all are finite: those behind T are 0, and a group whose sum is not finite has the sum 0 and NaN for
// x.  linear_many's loads are side by side whatever the stride of x is; a chunk of 2048 rows through 6144 x 4096 took
// 139 us with x in this order and 146 with bf16 rows as they stand.  A lane takes 8 values, GROUP / 8 lanes a group.
// Memory: 16.8 MB read and written 7 to 10 us.
template <int GROUP, bool PIECES>
__global__ __launch_bounds__(256) void sum_groups(const void *x, int64_t stride, int T, int K, int Kp, uint2 *totals,
                                              uint16_t *out) {
    constexpr int PER = kBlock / GROUP, PARTS = PIECES ? 2 : 1;
    const int lanes = Kp / 8;
    const int64_t all = int64_t(tokens32(T)) * lanes;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t t = i / lanes;
        const int k = int(i - t * lanes) * 8, block = k / kBlock;
        const bool there = t < T && k < K;
        uint16_t *to = out + (int64_t(block) * (PIECES ? 3 : 1) * T + t) * kBlock + k % kBlock;
        float v[PARTS][8] = {};
        if constexpr (PIECES) {
            if (there) {
                const float4 *from = reinterpret_cast<const float4 *>(static_cast<const float *>(x) + t * stride + k);
                const float4 f = from[0], g = from[1];
                v[0][0] = f.x, v[0][1] = f.y, v[0][2] = f.z, v[0][3] = f.w, v[0][4] = g.x, v[0][5] = g.y, v[0][6] = g.z, v[0][7] = g.w;
            }
            uint4 p[3];
            cut(v[0], p);
            if (t < T) {
#pragma unroll
                for (int j = 0; j < 3; ++j) *reinterpret_cast<uint4 *>(to + j * int64_t(T) * kBlock) = p[j];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float first = __uint_as_float(__float_as_uint(v[0][e]) & 0xffff0000u);
                v[1][e] = v[0][e] - first;
                v[0][e] = first;
            }
        } else {
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (there) w = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(x) + t * stride + k);
            if (t < T) *reinterpret_cast<uint4 *>(to) = w;
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[0][2 * e] = __uint_as_float(u[e] << 16);
                v[0][2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
            }
        }
        bool finite = true;
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            const float (&f)[8] = v[part];
            float s = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
            // 4, 8 or 16 lanes of a group, aligned, all of which are here: Kp is a multiple of 128
            s += __shfl_xor(s, 1);
            s += __shfl_xor(s, 2);
            if constexpr (GROUP >= 64) s += __shfl_xor(s, 4);
            if constexpr (GROUP >= 128) s += __shfl_xor(s, 8);
            finite = finite && fabsf(s) < INFINITY;
            uint32_t p[3];
            pieces_of(finite ? -s : 0.f, p);
            const int64_t at = ((int64_t(block * PARTS + part) * (tokens32(T) / 32) + t / 32) * PER + k % kBlock / GROUP) * 16 + t % 16;
            if (k % GROUP == 0) totals[at * 2 + t / 16 % 2] = make_uint2(uppers(p[0], p[1]), p[2] >> 16);
        }
        if (!finite) *reinterpret_cast<uint4 *>(to) = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    }
}

bool sizes_ok(int N, int K, int group) { return apex_linear_w4_bytes(N, K, group) != 0; }

int padded(int K) { return (K + kBlock - 1) / kBlock * kBlock; }

// Staged rows at most; others go through linear_some.  fp32 rows while they fit into LDS, with room for the sums: us, staged and not, one
// row of 14336 (84 KiB) through 4096 12.5 and 26.9, 4 of 4096 (96 KiB) through 6144 7.8 and 12.0, 4 of 1024 through 2048 4.2
// and 5.0.  bf16 rows as long as several workgroups fit on a CU: 4 of 4096 (32 KiB) through 32768 13.6 and 18.8, one of
// 14336 (28 KiB) through 4096 11.9 and 13.1; above, 4 of 8192 (64 KiB) through 700 6.9 and 7.8, but 4 of 14336 (112 KiB)
// through 4096 14.6 and 13.3.
constexpr int stage_bytes(Rows rows) { return (rows == kPieces ? 136 : 48) << 10; }

// Whether all of x goes to LDS, and in which rows.
bool stages(int T, int K, int pieces, Rows *rows) {
    *rows = pieces == 3 ? kPieces : kFew;
    return T <= 4 && int64_t(staged_rows(*rows, T)) * (padded(K) * 2 + kPad) <= stage_bytes(*rows);
}

// Workgroups that stay, 3 a CU at most: with 256, 512, 768, 1280 and 2048 of them 4 rows through 32768 x 4096 take 17.7, 15.6, 15.4, 16.7
// and 17.0 us, through 60000 x 1024 9.7, 8.1, 8.0, 9.0 and 9.6.
template <int GROUP, int R, int ROWS>
void launch_few(const LinearArgs &a, hipStream_t st) {
    const size_t lds = staged_rows(ROWS, a.T) * (a.blocks * 256 + kPad) + 2 * 4 * (kWaves * R * 64);
    const int tiles = (a.N + 16 * R - 1) / (16 * R);
    hipLaunchKernelGGL((linear_few<GROUP, R, ROWS>), dim3(std::min((tiles + 7) / 8 * 8, 3 * kCUs)), dim3(64 * kWaves), lds, st, a);
}

template <int GROUP, int R, int TT, int P>
void launch_some(const LinearArgs &a, hipStream_t st) {
    const int tiles = (a.N + 16 * R - 1) / (16 * R), tokens = 16 * TT * (kWaves / a.ways);
    LinearArgs b = a;
    b.token_groups = (a.T + tokens - 1) / tokens;
    b.by_tokens = int64_t(a.T) * (P == 3 ? 8 : 4) > a.N;
    hipLaunchKernelGGL((linear_some<GROUP, R, TT, P>), dim3((tiles * b.token_groups + 7) / 8 * 8), dim3(64 * kWaves), 0, st, b);
}

template <int GROUP, int TT>
void launch_many(const ManyArgs &m, hipStream_t st) {
    const int units = m.whole + (m.tiles - m.whole) * m.splits;
    const int rounds = (units + kManySlots - 1) / kManySlots;
    const auto f = m.a.pieces == 3 ? linear_many<GROUP, TT, 3> : linear_many<GROUP, TT, 1>;
    hipLaunchKernelGGL(f, dim3(rounds * kManySlots), dim3(kManyThreads), 0, st, m);
    if (m.splits > 1)
        hipLaunchKernelGGL(join<TT>, dim3((m.tiles - m.whole) * (4 * TT)), dim3(kManyRows), 0, st, m);
}

template <int GROUP>
void launch_many(const ManyArgs &m, int tt, hipStream_t st) {
    tt == 4 ? launch_many<GROUP, 4>(m, st) : launch_many<GROUP, 8>(m, st);
}

bool is_type(int t) { return t == APEX_TYPE_FP32 || t == APEX_TYPE_BF16; }

// How a call is worked on.
struct Plan {
    enum { kStaged, kSome, kMany } kind;
    Rows rows;                       // kStaged
    int r, ways;                     // kStaged and kSome: 16 r rows of the weights a workgroup; kSome: wavefronts along K
    int tt, m_tiles, tiles, whole, splits, share;     // kMany
    size_t pieces, totals, parts;    // bytes of the workspace, in this order
    size_t bytes() const { return pieces + totals + parts; }
};

constexpr size_t up256(size_t n) { return (n + 255) / 256 * 256; }
size_t x_bytes(int T, int Kp, int pieces) { return up256(size_t(pieces) * T * Kp * 2); }
size_t sums_bytes(int T, int Kp, int group, int pieces) {
    return up256(size_t(tokens32(T)) * (Kp / group) * (pieces == 3 ? 16 : 8));
}

// linear_some: how many of the 8 wavefronts go along K, and whether for 16 or 32 rows of the weights.  Workgroups a CU
// times the steps of a wavefront and one more for its ends; 32 rows take 1.3 times as long as 16.  us, for 8, 4, 2 and 1
// along K: 1073 x 1288 x 128, 32 rows: 16.7, 14.3, 8.8, 5.9; 96 x 4096 x 4096, 32 rows: 14.9, 13.8, 22.4, 39.2, 16 rows:
// 16.9, 18.2, 19.6, 34.1; 64 x 2048 x 2048, 16 rows: 5.6, 6.9, 10.3, 16.9, 32 rows: 6.0, 8.2, 12.7, 20.9.  Returns an
// estimate of the time in us: a step of 16 and 32 tokens of bf16 takes 0.6 and 1.0, one of 16 of fp32 1.4.
double plan_some(int T, int N, int blocks, int pieces, Plan &p) {
    const int tokens = pieces == 1 && T > 16 ? 32 : 16, token_tiles = (T + tokens - 1) / tokens;
    double least = 0;
    for (int r = 1; r <= 2; ++r)
        for (int ways = kWaves; ways >= 1; ways /= 2) {
            const int each = kWaves / ways;
            const int64_t groups = int64_t((N + 16 * r - 1) / (16 * r)) * ((token_tiles + each - 1) / each);
            const double cost = double((groups + kCUs - 1) / kCUs) * ((blocks + ways - 1) / ways + 1) * (r == 1 ? 1.0 : 1.3);
            if (least > 0 && cost >= least) continue;
            least = cost;
            p.r = r, p.ways = ways;
        }
    return 2.5 + least * (pieces == 3 ? 1.4 : tokens == 16 ? 0.6 : 1.0);
}

// linear_many: tiles of 64 or 128 tokens, and into how many shares the last of them are cut, by the steps of a CU, 1.2 and
// 2.0 us each in groups of 128, 1.2 and 2.1 of 64, 1.3 and 2.3 of 32, and the shares' way through memory and their launch.
// Whole calls of bf16 rows in groups of 64, us, 64 and 128: 100 x 4096 x 4096 24.7 and 26.3, 512 x 6144 x 4096 53.0 and 53.1,
// 400 x 14336 x 4096 95.6 and 79.1, 8192 x 6144 x 4096 611 and 527.  Returns an estimate of the time in us, with x's way
// through memory and two launches.
double plan_many(int T, int N, int blocks, int group, int pieces, Plan &p) {
    double least = 0;
    const double step4 = group == 32 ? 1.3 : 1.2, step8 = group == 32 ? 2.3 : group == 64 ? 2.1 : 2.0;
    for (const int tt : {4, 8}) {
        const int m_tiles = (T + 16 * tt - 1) / (16 * tt), tiles = m_tiles * ((N + kManyRows - 1) / kManyRows);
        const int whole = tiles / kManySlots * kManySlots, rest = tiles - whole;
        const int most = rest > 0 ? std::min(kManySlots / rest, blocks) : 1;
        for (const int want : {most, most / 2, 1}) {
            if (want < 1) continue;
            const int share = (blocks + want - 1) / want, splits = (blocks + share - 1) / share;
            const size_t parts = splits > 1 ? size_t(rest) * splits * (16 * tt * kManyRows * 4) : 0;
            const double steps = (double(whole / kManySlots) * blocks + (rest > 0 ? share : 0)) * pieces;
            const double us = steps * (tt == 4 ? step4 : step8) + (parts > 0 ? 3 + double(parts) / 4e6 : 0);
            if (least > 0 && us >= least) continue;
            least = us;
            p.tt = tt, p.m_tiles = m_tiles, p.tiles = tiles, p.whole = whole, p.splits = splits, p.share = share, p.parts = parts;
        }
    }
    return 8 + least + double(T) * blocks * kBlock * (pieces == 3 ? 10 : 4) / 4.5e6;
}

// Up to 32 rows of bf16 and 16 of fp32, a tile of linear_some, take no workspace.  Of more rows linear_some reads the
// weights once for every tile, linear_many is two or three launches; us in groups of 64, some and many: bf16 rows, 239 x 12103 x 1312
// 31.1 and 23.9, 45 x 14783 x 2728 20.1 and 23.2, 249 x 3266 x 3736 22.0 and 25.1, 56 x 854 x 7008 9.7 and 21.4; fp32 rows,
// 298 x 669 x 3328 16.1 and 25.5, 24 x 8081 x 5120 21.5 and 31.0, 301 x 1361 x 5976 47.4 and 37.8, 104 x 69 x 3200 7.6 and
// 15.9.  Of 200 calls of mixed sizes, types and groups the estimates took a way that is slower by more than a twentieth six
// times, by 4.9 us at most.
Plan plan_of(int T, int N, int K, int group, int pieces) {
    Plan p{};
    const int Kp = padded(K), blocks = Kp / kBlock;
    if (stages(T, K, pieces, &p.rows)) {
        p.kind = Plan::kStaged;
        p.r = N <= 16 * kCUs ? 1 : 2;                  // 16 rows while that leaves a workgroup a CU of its own
        return p;
    }
    p.kind = Plan::kSome;
    const double some = plan_some(T, N, blocks, pieces, p);
    const int tokens = pieces == 3 ? 16 : 32, token_tiles = (T + tokens - 1) / tokens;
    if (token_tiles == 1) return p;
    Plan m{};
    m.kind = Plan::kMany;
    const double many = plan_many(T, N, blocks, group, pieces, m);
    const int64_t workgroups = int64_t(token_tiles + 8) * (N / 16 + 8);      // of linear_some, at most
    if (some <= many && workgroups < (int64_t(1) << 31)) return p;
    m.pieces = x_bytes(T, Kp, pieces);
    m.totals = sums_bytes(T, Kp, group, pieces);
    return m;
}

template <int GROUP, int R>
void launch(const LinearArgs &a, const Plan &p, hipStream_t st) {
    if (p.kind == Plan::kStaged)
        p.rows == kFew ? launch_few<GROUP, R, kFew>(a, st) : launch_few<GROUP, R, kPieces>(a, st);
    else if (a.pieces == 3)
        launch_some<GROUP, R, 1, 3>(a, st);
    else
        a.T <= 16 ? launch_some<GROUP, R, 1, 1>(a, st) : launch_some<GROUP, R, 2, 1>(a, st);
}

template <int GROUP>
void launch(const LinearArgs &a, const Plan &p, hipStream_t st) {
    p.r == 1 ? launch<GROUP, 1>(a, p, st) : launch<GROUP, 2>(a, p, st);
}

}  // namespace

extern "C" size_t apex_linear_w4_workspace_bytes(int T, int N, int K, int group, int x_type) {
    if (T < 1 || T > APEX_MAX_STEP_TOKENS || !sizes_ok(N, K, group) || !is_type(x_type)) return 0;
    const int pieces = x_type == APEX_TYPE_FP32 ? 3 : 1, Kp = padded(K), blocks = Kp / kBlock;
    if (T <= (pieces == 3 ? 16 : 32)) return 0;
    // a smaller T may be cut into more shares: the most of any number of tiles
    size_t parts = 0;
    for (int t = 64; t - 64 < T; t += 64) {
        Plan p{};
        plan_many(t, N, blocks, group, pieces, p);
        parts = std::max(parts, p.parts);
    }
    return x_bytes(T, Kp, pieces) + sums_bytes(T, Kp, group, pieces) + parts;
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
    const int64_t x_size = x_type == APEX_TYPE_FP32 ? 4 : 2, y_size = y_type == APEX_TYPE_FP32 ? 4 : 2;
    const apex::Rows y_rows{y, y_stride * y_size, N * y_size};
    APEX_REQUIRE(!apex::rows_overlap(y_rows, {x, x_stride * x_size, K * x_size}, T), "%s: rows of y overlap rows of x", fn);
    APEX_REQUIRE(!residual || residual == y ||
                     !apex::rows_overlap(y_rows, {residual, residual_stride * y_size, N * y_size}, T),
                 "%s: rows of y overlap others of the residual", fn);
    LinearArgs a{static_cast<const uint8_t *>(w),
                 reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(w) + size_t(N) * (Kp / 2)),
                 static_cast<const uint16_t *>(x), x_stride, 0, K, bias, residual, y, residual_stride, y_stride, N, T,
                 Kp / kBlock, pieces, y_type == APEX_TYPE_FP32, plan.ways, 1, false};
    if (plan.kind == Plan::kMany) {
        char *ws = static_cast<char *>(workspace);
        uint2 *totals = reinterpret_cast<uint2 *>(ws + plan.pieces);
        uint16_t *tiled = reinterpret_cast<uint16_t *>(ws);
        const int64_t items = int64_t(tokens32(T)) * (Kp / 8);
        // workgroups at most: any number from 1024 on takes as long (2048 rows of 4096 10.2, 9.5 with 4096 of them and 9.8 so)
        const dim3 grid(unsigned(std::min<int64_t>((items + 255) / 256, 1 << 16)));
        const auto f = pieces > 1 ? (group == 32 ? sum_groups<32, true> : group == 64 ? sum_groups<64, true> : sum_groups<128, true>)
                                  : (group == 32 ? sum_groups<32, false> : group == 64 ? sum_groups<64, false> : sum_groups<128, false>);
        hipLaunchKernelGGL(f, grid, dim3(256), 0, stream, x, x_stride, T, K, Kp, totals, tiled);
        APEX_HIP(hipGetLastError());
        a.x = tiled;
        a.x_stride = kBlock;
        a.x_piece = int64_t(T) * kBlock;
        const ManyArgs m{a, reinterpret_cast<const uint8_t *>(totals), reinterpret_cast<float *>(ws + plan.pieces + plan.totals), plan.m_tiles, plan.tiles,
                         plan.whole, plan.splits, plan.share};
        group == 32 ? launch_many<32>(m, plan.tt, stream) : group == 64 ? launch_many<64>(m, plan.tt, stream)
                                                                        : launch_many<128>(m, plan.tt, stream);
    } else {
        group == 32 ? launch<32>(a, plan, stream) : group == 64 ? launch<64>(a, plan, stream) : launch<128>(a, plan, stream);
    }
    APEX_HIP(hipGetLastError());
    return APEX_OK;
}
