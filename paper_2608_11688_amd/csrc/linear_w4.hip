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
__device__ __forceinline__ void cut(uint4 u, uint4 v, uint4 (&p)[3]) {
    float f[8] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w),
                  __uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)};
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
            cut(v[0], v[1], p);
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

// Rows of fp32 values as three rows of bf16 pieces whose sum they are, zeros behind K.
__global__ __launch_bounds__(256) void split_x(const float *x, int64_t stride, int T, int K, int Kp, uint16_t *out) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int lanes = Kp / 8;
    const int64_t t = i / lanes;
    const int k = int(i - t * lanes) * 8;
    if (t >= T) return;
    uint4 p[3] = {};
    if (k < K) {
        const uint4 *from = reinterpret_cast<const uint4 *>(x + t * stride + k);
        cut(from[0], from[1], p);
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) *reinterpret_cast<uint4 *>(out + (int64_t(j) * T + t) * Kp + k) = p[j];
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

}  // namespace

extern "C" size_t apex_linear_w4_workspace_bytes(int T, int N, int K, int group, int x_type) {
    if (T < 1 || T > APEX_MAX_STEP_TOKENS || !sizes_ok(N, K, group) || x_type != APEX_TYPE_FP32) return 0;
    Rows rows;
    if (stages(T, K, 3, &rows)) return 0;
    return size_t(3) * T * padded(K) * 2;
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
    const size_t need = apex_linear_w4_workspace_bytes(T, N, K, group, x_type);
    APEX_REQUIRE(need == 0 || workspace, "%s: NULL workspace", fn);
    if (workspace_bytes < need)
        return apex::fail(APEX_E_CAPACITY, "%s: workspace of %zu bytes, %zu needed", fn, workspace_bytes, need);
    const int Kp = padded(K), pieces = x_type == APEX_TYPE_FP32 ? 3 : 1;
    LinearArgs a{static_cast<const uint8_t *>(w),
                 reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(w) + size_t(N) * (Kp / 2)),
                 static_cast<const uint16_t *>(x), x_stride, 0, K, bias, residual, y, residual_stride, y_stride, N, T,
                 Kp / kBlock, pieces, y_type == APEX_TYPE_FP32};
    Rows rows;
    const bool stage = stages(T, K, pieces, &rows);
    if (!stage && pieces > 1) {
        uint16_t *out = static_cast<uint16_t *>(workspace);
        const int64_t items = int64_t(T) * (Kp / 8);
        hipLaunchKernelGGL(split_x, dim3(unsigned((items + 255) / 256)), dim3(256), 0, stream,
                           static_cast<const float *>(x), x_stride, T, K, Kp, out);
        APEX_HIP(hipGetLastError());
        a.x = out;
        a.x_stride = Kp;
        a.x_piece = int64_t(T) * Kp;
        a.x_cols = Kp;
    }
    group == 32   ? launch<32>(a, stage, rows, stream)
    : group == 64 ? launch<64>(a, stage, rows, stream)
                  : launch<128>(a, stage, rows, stream);
    APEX_HIP(hipGetLastError());
    return APEX_OK;
}
