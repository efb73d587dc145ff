// Attention of new tokens over a paged cache (apex_attention_paged).
//
// A tile is a group of query rows of one request and key/value head that are worked on together;
// the positions it sees fall into units.  Launches of a call (for up to 512 tiles each):
//   attend    Every workgroup lists the tiles and their units for itself (build_list), then its
//             workers take their shares.  By the lengths, tiles are of one token (attend_token, a
//             wavefront a worker) or of up to 128 query rows, heads of one group and consecutive
//             tokens (attend_tile, a workgroup a worker).  The units of a head, tile after tile,
//             are shared out evenly over its workers (or, many large tiles: whole tiles).  A tile
//             within one share is written to `out`; where shares end inside a tile, its weighted
//             sums, maxima and normalisers go to the workspace.
//   merge     the parts of such tiles joined by the log-sum-exp rule.
//
// Both kinds compute S^T = K Q^T and O^T = V^T P^T on the matrix cores: a lane then holds the
// scores of one query row in its registers, so that maxima, sums and rescaling are a lane's own
// (but for one or two exchanges between lanes of a row), and the scores' registers are the
// second product's operand as they stand.  The order of the positions within a step, which the
// first product's registers give, is taken over by the loads of V^T (transposing reads of LDS).
// Keys and values go from memory to LDS directly, by buffer loads whose descriptor is a page's
// 16 rows: rows past the last position, under the window or of a bad page lie past the
// descriptor's end and are written as zeros, so nothing that is not visible to a tile is read.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "common.h"
#include "ffn_device.h"
#include "ffn_internal.h"
#include "paged_internal.h"

namespace {

using apex::ffn::kWave;
using apex::ffn::sum_xor16;
using apex::ffn::sum_xor32;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef int intx2 __attribute__((ext_vector_type(2)));

#define APEX_LDS __attribute__((address_space(3)))

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Read-only memory at addresses that are the same for a whole wavefront: the constant address
// space makes these scalar loads, which do not count among the vector loads a wait is for.
template <class T>
__device__ __forceinline__ T scalar_load(const T *p, int64_t i) {
    static_assert(sizeof(T) == 4, "one register");
    typedef const __attribute__((address_space(4))) T *Scalar;
    return ((Scalar)(p))[i];
}

constexpr int kCus = 256;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMaxGroup = 16;      // query heads per key/value head
constexpr float kLog2e = 1.4426950408889634f;
// Weights are 2^(score - m) for a reference m that is raised to the running maximum only when
// that is more than kSlack above it: they stay below 2^kSlack, where sums in 32 bits and
// roundings, which are relative, are as good, and rescaling is rare.  Of tiles of many rows
// (attend_tile), those of up to kExactRows, where a new maximum is rare enough, raise it at once:
// their largest weight is 1, which no rounding to bf16 moves.  (Tokens of a mixed batch over bf16
// pages: error 1.09 times that of the result's rounding on average and at most 1.35 in 850 drawn
// cases; with the slack 1.20 and 1.73.  Chunks of 4096 and 2048 tokens take 4 to 7 % longer without it.)
constexpr float kSlack = 8.f;
constexpr int kExactRows = 16;

// --------------------------------------------------------------------------------- tiles
// The first position a token at position p sees besides the sinks.  Tokens that lengths place
// before 0 see nothing, and p - window would pass the range of an int there.
__device__ __forceinline__ int lower_edge(int p, int window) { return window > 0 ? max(0, max(p, 0) - window + 1) : 0; }

// The positions a tile of tokens [q0, q1) of a request sees: sink units from 0 up, then the
// units from `first` up to the last token's position.  A unit has 2^shift positions.
struct Span {
    int sinks, first, units;
    __device__ __forceinline__ int base(int u, int shift) const {
        return (u < sinks ? u : first + u - sinks) << shift;
    }
};
__device__ __forceinline__ Span span_of(int p_first, int p_last, int window, int sinks, int shift) {
    Span s;
    s.first = lower_edge(p_first, window) >> shift;
    s.sinks = window > 0 ? min(int((unsigned(min(sinks, p_last + 1)) + (1u << shift) - 1) >> shift), s.first) : 0;
    s.units = p_last < 0 ? 0 : (p_last >> shift) + 1 - s.first + s.sinks;
    return s;
}
constexpr int kTokenShift = 5, kTokenUnit = 1 << kTokenShift;   // of tiles of one token
constexpr int kTileShift = 6, kTileUnit = 1 << kTileShift;      // of tiles of many rows

// The new tokens [a, b) of request r among the rows of q, and its length, from device memory
// and so held to their ranges.
struct Request {
    int row0, n, seq;
};
__device__ __forceinline__ Request request_of(const int32_t *cu_new, const int32_t *seq_len, int r,
                                              int T, int room) {
    const int a = min(max(cu_new[r], 0), T), b = min(max(cu_new[r + 1], a), T);
    return {a, b - a, min(max(seq_len[r], 0), room)};
}
constexpr int kListTiles = 512;                  // tiles of one launch

struct TileList {                   // in LDS
    int32_t cu[kListTiles + 1];     // units of the tiles before
    int32_t row[kListTiles];        // the tile's first row of q
    int32_t p[kListTiles];          // that row's position
    int32_t first[kListTiles];      // the first tile of its request, counted over all launches
    uint16_t r[kListTiles];         // its request
    uint8_t tokens[kListTiles];
    int wave_end[kWaves];
    float tokens_all[kWaves], once[kWaves], each[kWaves];
    int found;
};

// Inclusive scans over a workgroup (sums, or maxima of values >= -1), `before` the exclusive one.
template <bool MAX, int CTRL>
__device__ __forceinline__ int scan_step(int v) {
    const int o = __builtin_amdgcn_update_dpp(MAX ? -1 : 0, v, CTRL, 0xf, 0xf, false);
    return MAX ? max(v, o) : v + o;
}
template <bool MAX>
__device__ __forceinline__ int block_scan(int v, int *wave_end, int *before, int *total) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const auto join = [](int x, int y) { return MAX ? max(x, y) : x + y; };
    int x = scan_step<MAX, 0x111>(v);   // row_shr 1, 2, 4, 8
    x = scan_step<MAX, 0x112>(x);
    x = scan_step<MAX, 0x114>(x);
    x = scan_step<MAX, 0x118>(x);
    const int r0 = __builtin_amdgcn_readlane(x, 15);
    const int r1 = join(r0, __builtin_amdgcn_readlane(x, 31));
    const int r2 = join(r1, __builtin_amdgcn_readlane(x, 47));
    const int none = MAX ? -1 : 0;
    x = join(x, lane < 16 ? none : lane < 32 ? r0 : lane < 48 ? r1 : r2);
    if (lane == kWave - 1) wave_end[wave] = x;
    __syncthreads();
    int low = none, all = none;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) low = join(low, wave_end[w]);
        all = join(all, wave_end[w]);
    }
    __syncthreads();
    int prev = __shfl_up(x, 1);
    *before = join(low, lane == 0 ? none : prev);
    *total = all;
    return join(low, x);
}

struct ListArgs {
    const int32_t *cu_new, *seq_len;
    int R, T, room, tile_tokens, first_tile, most_tiles, window, sinks;
};

// Whether tokens are worked on one by one, and tiles first_tile .. first_tile + most_tiles - 1 of
// all requests' tiles, those of a request in a row; returns how many there are.  A few round trips
// to memory and barriers, about 3 us, where a launch of its own that wrote the list for the next
// one took 7.  Loops are kept rolled: a launch this short waits for its instructions as much as
// for its data.
//
// One by one: no more tokens than requests, and what each reads of its context adds up to at most
// twice what the requests' contexts hold.  It is the tokens that count, not the rows of q, most of
// which may be empty.  Single tokens one by one and in tiles of many rows, us (32 requests of up
// to 4000 positions, 32 heads of 128 in 8 groups): bf16 73 and 78, E4M3 46 and 66, fp32 75 and 128,
// fp32 over E4M3 47 and 157; 16 requests of 2 tokens 28 and 30, 8 of 4 25 and 24; one request's 64
// tokens behind 8000 positions among 63 idle ones 166 and 35.
__device__ __forceinline__ int build_list(const ListArgs &a, TileList &s, bool &one_by_one) {
    const int t = threadIdx.x, wave = t / kWave;
    const int per = (a.R + kThreads - 1) / kThreads, r_lo = t * per, r_hi = min(r_lo + per, a.R);
#pragma unroll 1
    for (int i = t; i < kListTiles; i += kThreads) s.first[i] = -1;
    // (in fp32: tokens that lengths count twice pass 32 bits, and what decides is exact below 2^24)
    float tokens_all = 0.f, once = 0.f, each = 0.f;
    int n = 0;   // of a thread that has one request
#pragma unroll 1
    for (int r = r_lo; r < r_hi; ++r) {
        const Request q = request_of(a.cu_new, a.seq_len, r, a.T, a.room);
        n = q.n;
        const unsigned most = a.window > 0 ? unsigned(a.window) + unsigned(a.sinks) : unsigned(INT_MAX);
        const float context = float(min(unsigned(q.seq), most));
        tokens_all += float(n);
        once += n > 0 ? context : 0.f;
        each += float(n) * context;
    }
    tokens_all = apex::ffn::wave_sum(tokens_all);
    once = apex::ffn::wave_sum(once);
    each = apex::ffn::wave_sum(each);
    if (t % kWave == 0) s.tokens_all[wave] = tokens_all, s.once[wave] = once, s.each[wave] = each;
    __syncthreads();
    tokens_all = once = each = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) tokens_all += s.tokens_all[w], once += s.once[w], each += s.each[w];
    one_by_one = uniform(tokens_all <= float(a.R) && each <= 2.f * once);
    const int tile_tokens = one_by_one ? 1 : a.tile_tokens, shift = one_by_one ? kTokenShift : kTileShift;
    const auto tiles_of = [&](int n) { return int(unsigned(n + tile_tokens - 1) / unsigned(tile_tokens)); };
    const auto tokens_of = [&](int r) { return per == 1 ? n : request_of(a.cu_new, a.seq_len, r, a.T, a.room).n; };
    int count = 0;
#pragma unroll 1
    for (int r = r_lo; r < r_hi; ++r) count += tiles_of(tokens_of(r));
    int at, total;
    block_scan<false>(count, s.wave_end, &at, &total);
    // the first tile of each request in the list names it
#pragma unroll 1
    for (int r = r_lo; r < r_hi; ++r) {
        const int n = tiles_of(tokens_of(r));
        if (n > 0 && at + n > a.first_tile && at < a.first_tile + kListTiles) {
            const int i = max(at - a.first_tile, 0);
            s.first[i] = at;
            s.r[i] = uint16_t(r);
        }
        at += n;
    }
    const int tiles = min(max(total - a.first_tile, 0), a.most_tiles);
    __syncthreads();
    // a thread's tiles, in a row; the tiles between two named ones are the first one's
    const int share = (tiles + kThreads - 1) / kThreads, i0 = t * share, i1 = min(i0 + share, tiles);
    int named = -1, before, all;
#pragma unroll 1
    for (int i = i0; i < i1; ++i)
        if (s.first[i] >= 0) named = i;
    block_scan<true>(named, s.wave_end, &before, &all);
    int sum = 0;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
        if (s.first[i] >= 0) before = i;
        const int k = max(before, 0), first = s.first[k], r = s.r[k];
        const Request q = request_of(a.cu_new, a.seq_len, r, a.T, a.room);
        const int q0 = (a.first_tile + i - first) * tile_tokens;
        const int p = q.seq - q.n + q0, tokens = min(tile_tokens, q.n - q0);
        // a tile that sees nothing still has a unit: its rows are written
        sum += max(span_of(p, p + tokens - 1, a.window, a.sinks, shift).units, 1);
        s.cu[i + 1] = sum;
        s.row[i] = q.row0 + q0;
        s.p[i] = p;
        s.tokens[i] = uint8_t(tokens);
        s.r[i] = uint16_t(r);   // (of a named tile, the only ones others read: what it was)
    }
    block_scan<false>(sum, s.wave_end, &before, &all);
    if (t == 0) s.cu[0] = 0;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) s.cu[i + 1] += before;
    __syncthreads();
    return tiles;
}

// The tile of unit z, for all threads.
__device__ __forceinline__ int tile_of(TileList &s, int tiles, int z) {
#pragma unroll 1
    for (int i = threadIdx.x; i < tiles; i += kThreads)
        if (s.cu[i] <= z && z < s.cu[i + 1]) s.found = i;
    __syncthreads();
    return uniform(s.found);
}

// Units 0 .. all - 1 in even shares, workers <= all: none is empty.
struct Shares {
    int each, more;   // units of a share, and how many shares have one more
    __device__ __forceinline__ Shares(int all, int workers) : each(all / workers), more(all % workers) {}
    __device__ __forceinline__ int begin(int w) const { return each * w + min(w, more); }
    __device__ __forceinline__ int worker_of(int unit) const {
        const int wide = more * (each + 1);
        return unit < wide ? unit / (each + 1) : more + (unit - wide) / each;
    }
};

// Where a tile's rows come from, written by the worker whose share it begins in: that worker's
// part `part` and the first parts of the next `more` ones (more = 0: they are written already).
struct Split {
    int row, rows, part, more;      // part: of all [worker][G][2]
};

// -------------------------------------------------------------------------------- device
struct AttendArgs {
    const void *q;
    void *out;
    int64_t q_stride, out_stride;
    const uint8_t *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t *block_table;
    ListArgs list;
    int G, GR, max_blocks, shift, page_size, n_pages;
    int workers, token_workers;   // that share out a head's units: workgroups, or wavefronts
    float scale_log2;      // the softmax scale times log2(e)
    int2 *tiles;           // how many the launch has, and whether of one token
    Split *split;          // [tile][G]
    float *part_o;         // [worker][G][2][rows][hd]
    float2 *part_ml;       // [worker][G][2][rows]: maximum (of scores in powers of two), normaliser
};

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ floatx4 mfma16(uint4 a, uint4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 mfma32(uint4 a, uint4 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

__device__ __forceinline__ float max_xor16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_xor32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ uint32_t pk_bf16(float lo, float hi) {   // rounded to nearest even
    const bf16x2 v = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
    return __builtin_bit_cast(uint32_t, v);
}

// A matrix-core operand of 8 fp32 values in N bf16 pieces, all but the last of which are cut off
// after 8 significant bits and the last rounded: one, two for 16 bits or three for the value.  A
// piece of 0 must not meet an infinite key or value, with which its product is NaN: where the
// other operand `meets` infinities, pieces behind one that holds the value are 2^-40 and 2^-50 of
// it, which no sum in 32 bits shows (from 2^-76 up; those of a smaller value may be 0).  `is`: the
// values may be infinite themselves, all their pieces are then.
enum class Infinity { never, meets, is };
template <int N>
struct Pieces {
    uint4 p[N];
};
template <int N, Infinity INF>
__device__ __forceinline__ Pieces<N> pieces_of(const float (&in)[8]) {
    Pieces<N> r;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = in[e];
#pragma unroll
    for (int q = 0; q < N - 1; ++q) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u0 = __float_as_uint(x[2 * i]), u1 = __float_as_uint(x[2 * i + 1]);
            w[i] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);   // upper halves of u0, u1
            x[2 * i] -= __uint_as_float(u0 & 0xffff0000u);
            x[2 * i + 1] -= __uint_as_float(u1 & 0xffff0000u);
        }
        if constexpr (INF != Infinity::never)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = fmaf(in[e], q == 0 ? 0x1p-40f : 0x1p-50f, x[e]);
        if constexpr (INF == Infinity::is)   // (infinity less itself)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = x[e] == x[e] ? x[e] : in[e];
        r.p[q] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    r.p[N - 1] = make_uint4(pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3]), pk_bf16(x[4], x[5]), pk_bf16(x[6], x[7]));
    return r;
}

// 8 consecutive values of a query row (bf16 or fp32), zeros where !on.
template <bool F32>
__device__ __forceinline__ Pieces<F32 ? 3 : 1> load_q(const void *q, int64_t at, bool on) {
    Pieces<F32 ? 3 : 1> r;
    if constexpr (F32) {
        const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(q) + at);
        const float4 a = p[0], b = p[1];
        const float x[8] = {on ? a.x : 0.f, on ? a.y : 0.f, on ? a.z : 0.f, on ? a.w : 0.f,
                            on ? b.x : 0.f, on ? b.y : 0.f, on ? b.z : 0.f, on ? b.w : 0.f};
        r = pieces_of<3, Infinity::is>(x);
    } else {
        const uint4 v = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(q) + at);
        r.p[0] = make_uint4(on ? v.x : 0u, on ? v.y : 0u, on ? v.z : 0u, on ? v.w : 0u);
    }
    return r;
}

// 8 E4M3 codes as bf16 values (exact).
__device__ __forceinline__ uint4 widen_e4m3(uint2 c) {
    const auto w = [](uint32_t v, bool hi) {
        return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, true)
                                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, false));
    };
    return make_uint4(w(c.x, false), w(c.x, true), w(c.y, false), w(c.y, true));
}

// Whether a position is visible to a query at position p.
__device__ __forceinline__ bool visible(int j, int p, int window, int sinks) {
    return j <= p && (window == 0 || j > p - window || j < sinks);
}

// One page's 16 rows: where they are, how many of them a tile may read, from which on.
// Rows below `from` that are no sinks, rows from `end` on and rows of a bad page read as zeros.
struct Rows16 {
    int64_t row;        // index of the first row in the pool [n_pages, G, page_size]
    int end;            // rows 0..end-1 exist for the tile
    bool ok;            // the page id is in range
};
__device__ __forceinline__ Rows16 rows_of_page(const AttendArgs &a, int page, int g, int j0, int hi) {
    Rows16 r;
    r.ok = page >= 0 && page < a.n_pages && j0 < hi;
    r.row = r.ok ? (int64_t(page) * a.G + g) * a.page_size + (j0 & (a.page_size - 1)) : 0;
    r.end = r.ok ? min(max(hi - j0, 0), 16) : 0;
    return r;
}
__device__ __forceinline__ Rows16 rows16(const AttendArgs &a, const int32_t *table, int g, int j0, int hi) {
    const int b = min(j0 >> a.shift, a.max_blocks - 1);
    return rows_of_page(a, j0 < hi ? scalar_load(table, b) : -1, g, j0, hi);
}

template <int N>
struct Int {
    static constexpr int value = N;
};

constexpr int vmcnt_only(int n) {   // the s_waitcnt operand: at most n vector loads outstanding
    n = n > 63 ? 63 : n;
    return 0x0f70 | (n & 15) | (n >> 4 << 14);
}
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(vmcnt_only(N));
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void lds_barrier() {   // leaves loads from memory in flight
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Rows in LDS are permuted in chunks of 16 bytes (chunk c of row i at c ^ swizzle(i)), by the
// addresses of the loading lanes, so that what a read takes at a time, the same chunk of many
// rows, lies in distinct banks.  RB: bytes of a row.
template <int RB>
struct KSwizzle {   // 16 consecutive rows, one chunk
    static __device__ __forceinline__ int of(int row) {
        return RB == 256 ? row & 15 : RB == 128 ? (row >> 1) & 7 : (row >> 2) & 3;
    }
};
template <int RB, bool F8>
struct TokenVSwizzle {   // bf16: 8 consecutive rows, two chunks; E4M3: rows 0-7 and 16-23, one
    static __device__ __forceinline__ int of(int row) {
        if (!F8) return RB == 256 ? 2 * (row & 7) : 2 * ((row >> 1) & 3);
        return RB == 128 ? ((row >> 1) & 3) | ((row >> 4) & 1) << 2
                         : ((row >> 2) & 1) | ((row >> 4) & 1) << 1;
    }
};
template <int RB>
struct TileVSwizzle {    // 4 consecutive rows, four chunks
    static __device__ __forceinline__ int of(int row) {
        return RB == 256 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
    }
};

// LDS is read at an array's base, an offset held in a register (settled: the compiler takes it as
// it is) and a constant: the compiler follows an address back to its array over few steps only,
// and a read whose array it has lost waits for every load into LDS that is on its way.
__device__ __forceinline__ int settled(int v) {
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ uint4 lds_u4(const uint8_t *p, int at) { return *reinterpret_cast<const uint4 *>(p + at); }
__device__ __forceinline__ uint2 lds_u2(const uint8_t *p, int at) { return *reinterpret_cast<const uint2 *>(p + at); }
// Transposing reads: of the 8 bytes that each of 16 lanes points to, lane i gets the i-th value of
// four rows of 16 bf16 values (a row is four lanes'), or of eight rows of 16 codes (two lanes').
__device__ __forceinline__ uint2 lds_tr16(const uint8_t *p, int at) {
    const shortx4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((APEX_LDS shortx4 *)(p + at));
    return __builtin_bit_cast(uint2, v);
}
__device__ __forceinline__ uint2 lds_tr8(const uint8_t *p, int at) {
    const intx2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((APEX_LDS intx2 *)(p + at));
    return __builtin_bit_cast(uint2, v);
}

// One of two pointers by the lane, chosen here and now (the compiler would rather load it from the
// arguments each time).
typedef const __attribute__((address_space(1))) float *GlobalFloats;   // of memory, not LDS
typedef const __attribute__((address_space(1))) int *GlobalInts;
__device__ __forceinline__ GlobalFloats lane_pointer(const float *p, const float *q, bool second) {
    const uint64_t x = reinterpret_cast<uint64_t>(p), y = reinterpret_cast<uint64_t>(q);
    const int lo = settled(second ? int(y) : int(x)), hi = settled(second ? int(y >> 32) : int(x >> 32));
    return (GlobalFloats)(uint64_t(uint32_t(hi)) << 32 | uint32_t(lo));
}

// Where 16 rows of RB bytes are and how many bytes of them a tile may read, in scalar registers by
// force: a load whose descriptor the compiler does not know to be uniform is wrapped in a loop
// over the lanes' values.
struct Extent {
    uint64_t base;
    uint32_t bytes;
};
template <int RB>
__device__ __forceinline__ Extent extent_of(const uint8_t *pool, const Rows16 &r) {
    const uint64_t base = reinterpret_cast<uint64_t>(pool) + r.row * RB;
    return {uint64_t(uint32_t(uniform(int(base >> 32)))) << 32 | uint32_t(uniform(int(base))),
            uint32_t(uniform(r.end * RB))};
}

// 16 rows of RB bytes, row_of.. of a tile, to LDS.  Rows below `from` and not below `keep` are
// written as zeros, as are those past r.end.
template <int RB, class SW>
__device__ __forceinline__ void load_rows16(const uint8_t *pool, const Rows16 &r, int from, int keep,
                                            uint8_t *lds, int lds_at, int row_of) {
    constexpr int CH = RB / 16, RPI = kWave / CH;   // chunks of a row, rows per load
    const int lane = threadIdx.x % kWave;
    const Extent x = extent_of<RB>(pool, r);
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(x.base), 0, x.bytes, 0x00027000);
#pragma unroll
    for (int i = 0; i < 16 / RPI; ++i) {
        const int row = RPI * i + lane / CH;
        const int chunk = (lane % CH) ^ SW::of(row_of + row);
        const int at = row < from && row >= keep ? 0x40000000 : row * RB + chunk * 16;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (APEX_LDS void *)(lds + (lds_at + RPI * i * RB)), 16, at,
                                                 0, 0, 0);
    }
}

template <bool F32>
__device__ __forceinline__ void store_out(void *out, int64_t at, float v) {
    if constexpr (F32)
        static_cast<float *>(out)[at] = v;
    else
        static_cast<uint16_t *>(out)[at] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// ------------------------------------------------------------------------- one token's tile
// A tile is one token and the query heads of a group: up to 16 rows, columns of the 16x16x32
// products.  Each wavefront is a worker of its own, on units of 32 positions, with stages of its
// own in LDS: behind the list no barrier, only the wavefront's own count of loads.  (Four
// wavefronts on one tile, joined in LDS: 256 requests of 64 to 256 positions 60 us instead of
// 42, where a tile is over before its loads are under way; long contexts the same.)
// Lane (q = lane % 16, lg = lane / 16) holds the scores of row q at positions 16 m + 4 lg + i.
// bf16 weights go through the second product in two pieces, 16 bits: the products wait for memory
// anyway, and rounded to 8 bits they would err as much as the rounding of the result, with E4M3
// scales, which alike rows have alike, up to 1.7 times as much.
// Bound by the stream of keys and values: 64 tokens under a window of 4096 (1.08 GB) 190 us,
// 5.65 TB/s, of 5.8 that a kernel that only reads gets.
constexpr int kMostParts = 512;   // of a launch's tiles, on average: one request of 60000 positions
                                  // in one group 19.5 us (21 when 1024, as many as fitted, took 24, 128 28)
constexpr int kTokenShare = 8;    // units: 256 requests of 64 to 256 positions (5 units a share) 50 us with
                                  // all workers, 47 with half; 31 of up to 4096 (12 units) 71.5 and 79.8

// Stages in LDS, and how many workgroups a CU holds: of tiles of many rows by their registers.
template <int HD, bool F8, bool F32>
struct Shape {
    static constexpr int kPerCu = HD == 128 ? (F32 ? 1 : 2) : (F8 || F32 ? 2 : 3);
    // tiles of many rows: keys and values of a unit, two stages
    static constexpr int kTileStage = 2 * kTileUnit * HD * 2;
    // tiles of one token: the same of 32 positions for each wavefront, a ring of kTokenStages; of
    // what the workgroups of a CU leave room for, or one stage, where keys and values take turns
    static constexpr int kRowBytes = HD * (F8 ? 1 : 2);
    static constexpr int kTokenStage = 2 * kTokenUnit * kRowBytes;
    static constexpr int kRing = 1024 * (kPerCu == 1 ? 128 : kPerCu == 2 ? 64 : 32);
    static constexpr int kTokenStages = kRing / (kWaves * kTokenStage);
    static_assert(kTokenStages == 1 || kTokenStages == 2 || kTokenStages == 4, "a ring");
    static constexpr int kTokenLoads = kTokenStage / 1024 + (F8 ? 1 : 0);
    static constexpr int kTokenArray = kWaves * kTokenStage / (kTokenStages == 1 ? 2 : 1);
    static constexpr int kStage = kTokenArray > kTileStage ? kTokenArray : kTileStage;
    // What parts and their merge cost a call where every workgroup leaves two, about 25 us, in the
    // time of a unit (us, with a CU full of workgroups: 2.1, E4M3 3.1, fp32 2.9; heads of 64
    // 1.5, 2.2 and 1.9).
    static constexpr float kSplitCost = HD == 128 ? (F32 || F8 ? 8.f : 12.f) : (F32 ? 13.f : F8 ? 11.f : 16.f);
};

// LDS of a workgroup.  An array for each stage: the compiler then knows which loads a read of LDS
// has to wait for.
struct Stages {
    uint8_t *st0, *st1, *st2, *st3;
};

template <int HD, bool F8, bool F32>
__device__ __forceinline__ void attend_token(const AttendArgs &a, TileList &list, int tiles, const Stages &lds_stages,
                                             float (*scales)[64]) {
    using S = Shape<HD, F8, F32>;
    constexpr int RB = S::kRowBytes, NS = S::kTokenStages, KS = HD / 32, DT = HD / 16;
    constexpr int NP = F32 ? 3 : 1, NW = F32 ? 3 : 2;   // pieces of a query value and of a weight
    constexpr Infinity kValues = F8 ? Infinity::never : Infinity::meets;   // (no E4M3 code is infinite)
    using KSw = KSwizzle<RB>;
    using VSw = TokenVSwizzle<RB, F8>;
    const int wg = uniform(blockIdx.x / a.G), g = blockIdx.x - wg * a.G;
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int w = wg * kWaves + wave;
    const int n = lane & 15, lg = lane >> 4;
    const int all_units = uniform(list.cu[tiles]);
    // None without a unit; half of them where all would have small shares.
    const bool half = S::kTokenStages == 1 && all_units / kTokenShare < a.token_workers;
    const int workers = min(half ? (a.token_workers + 1) / 2 : a.token_workers, min(all_units, kMostParts * tiles));
    if (w >= workers) return;
    const Shares shares(all_units, workers);
    const int share_lo = uniform(shares.begin(w)), share_hi = uniform(shares.begin(w + 1));
    int tile = 0;
    for (int i0 = 0; i0 < tiles; i0 += kWave) {
        const int i = i0 + lane;
        const unsigned long long here =
            __ballot(i < tiles && list.cu[min(i, tiles - 1)] <= share_lo && share_lo < list.cu[min(i, tiles - 1) + 1]);
        if (here) {
            tile = i0 + __ffsll(static_cast<long long>(here)) - 1;
            break;
        }
    }
    tile = uniform(tile);

    // where this lane reads, in a stage: keys of row n (and n + 16), values of row v_row (and,
    // bf16, v_row + 16); both swizzles are the same 16 rows further.  HALVES: one stage, its keys in
    // the first array and its values in the second.
    constexpr bool HALVES = NS == 1;
    constexpr int kKeys = 32 * RB, kPlace = HALVES ? kKeys : 2 * kKeys, kValuesAt = HALVES ? 0 : kKeys;
    int k_at[KS], v_at[DT];
    const int kv = n >> 1, v_row = F8 ? (kv < 4 ? 4 * lg + kv : 12 + 4 * lg + kv) : 4 * lg + (n >> 2);
#pragma unroll
    for (int u = 0; u < KS; ++u)
        k_at[u] = settled(wave * kPlace + n * RB +
                          (F8 ? 16 * ((2 * u + lg / 2) ^ KSw::of(n)) + 8 * (lg & 1)
                              : 16 * ((4 * u + lg) ^ KSw::of(n))));
#pragma unroll
    for (int d = 0; d < DT; ++d)
        v_at[d] = settled(wave * kPlace + kValuesAt + v_row * RB + 8 * (lane & 1) +
                          16 * ((F8 ? d : 2 * d + ((lane & 3) >> 1)) ^ VSw::of(v_row)));
    const auto stage = [&](auto which) __attribute__((always_inline)) -> uint8_t * {
        constexpr int st = decltype(which)::value;
        if constexpr (st == 0) return lds_stages.st0;
        else if constexpr (st == 1) return lds_stages.st1;
        else if constexpr (st == 2) return lds_stages.st2;
        else return lds_stages.st3;
    };
    const GlobalFloats scale_of = lane_pointer(a.k_scales, a.v_scales, lane >= 32);
    float sc[NS];           // this lane's scale of a stage: keys in lanes 0..31, values behind
    bool ok[NS][2];

    // the share's tiles
#pragma unroll 1
    for (int z = share_lo; z < share_hi; ++tile) {
    const int tile_lo = uniform(list.cu[tile]), tile_hi = uniform(list.cu[tile + 1]);
    const int u_lo = uniform(z - tile_lo), steps = uniform(min(tile_hi, share_hi) - z);
    const int req = uniform(list.r[tile]), p = uniform(list.p[tile]), hi = p + 1;
    const int low = lower_edge(p, a.list.window);
    const Span span = span_of(p, p, a.list.window, a.list.sinks, kTokenShift);
    const int32_t *table = a.block_table + size_t(req) * a.max_blocks;
    const int64_t row = uniform(list.row[tile]);
    const int part = z == tile_lo && tile_hi <= share_hi ? -1 : z == share_lo ? 0 : 1;

    Pieces<NP> qf[KS];
#pragma unroll
    for (int u = 0; u < KS; ++u)
        qf[u] = load_q<F32>(a.q, row * a.q_stride + (g * a.GR + (n < a.GR ? n : 0)) * HD + 32 * u + 8 * lg,
                            n < a.GR);

    // unit i's rows, nothing of which is to be read from the last unit on
    const auto unit_at = [&](int i) { return span.base(u_lo + min(i, steps - 1), kTokenShift); };
    const auto rows_of = [&](int i, Rows16 (&r)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 2; ++m) r[m] = rows16(a, table, g, unit_at(i) + 16 * m, i < steps ? hi : 0);
    };
    const auto load_keys = [&](int i, const Rows16 (&r)[2], uint8_t *at) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int j = unit_at(i) + 16 * m;
            load_rows16<RB, KSw>(a.k_pages, r[m], low - j, a.list.sinks - j, at, wave * kPlace + 16 * m * RB, 16 * m);
        }
    };
    const auto load_values = [&](int i, const Rows16 (&r)[2], uint8_t *at) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int j = unit_at(i) + 16 * m;
            load_rows16<RB, VSw>(a.v_pages, r[m], low - j, a.list.sinks - j, at, wave * kPlace + kValuesAt + 16 * m * RB,
                                 16 * m);
        }
    };
    const auto issue = [&](auto which, int i) __attribute__((always_inline)) {
        constexpr int st = decltype(which)::value;
        Rows16 r[2];
        rows_of(i, r);
        ok[st][0] = r[0].ok;
        ok[st][1] = r[1].ok;
        if constexpr (F8) {
            const int64_t at = lane & 16 ? r[1].row : r[0].row;
            const int last = max((lane & 16 ? r[1].end : r[0].end) - 1, 0);
            sc[st] = scale_of[at + min(n, last)];
        }
        load_keys(i, r, stage(which));
        load_values(i, r, stage(which));
        __builtin_amdgcn_sched_barrier(0);
    };

    float mx = -INFINITY, l = 0.f;    // l: of the lane's own positions
    floatx4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = floatx4{0.f, 0.f, 0.f, 0.f};
    const auto products = [&](const uint8_t *lds, float (&s)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            floatx4 big = floatx4{0.f, 0.f, 0.f, 0.f}, small = big;
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                uint4 k;
                if constexpr (F8)
                    k = widen_e4m3(lds_u2(lds, k_at[u] + 16 * m * RB));
                else
                    k = lds_u4(lds, k_at[u] + 16 * m * RB);
#pragma unroll
                for (int q = NP - 1; q > 0; --q) small = mfma16(k, qf[u].p[q], small);
                big = mfma16(k, qf[u].p[0], big);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * m + e] = F32 ? big[e] + small[e] : big[e];
        }
        if constexpr (HALVES) {   // all reads of LDS first: left to itself, each product waits for its own
            __builtin_amdgcn_sched_group_barrier(0x100, 2 * KS, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 2 * KS * NP, 0);
        }
    };
    // scores to weights (times the values' scales vs) of unit i, whose pages are ok
    const auto weights = [&](int i, bool ok0, bool ok1, float (&s)[8], float (&vs)[8])
                             __attribute__((always_inline)) {
        const int j0 = unit_at(i);
        const bool whole = j0 + 31 < hi && (j0 >= low || j0 + 31 < a.list.sinks) && ok0 && ok1;
        if (!whole) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + 16 * m + 4 * lg + e;
                    const bool on = j < hi && (j >= low || j < a.list.sinks) && (m ? ok1 : ok0);
                    s[4 * m + e] = on ? s[4 * m + e] : -INFINITY;
                    if constexpr (F8) vs[4 * m + e] = on ? vs[4 * m + e] : 0.f;
                }
        }
        float top = s[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
        top = max_xor32(max_xor16(top)) * a.scale_log2;
        if (__ballot(top > mx + kSlack)) {
            const float now = fmaxf(mx, top);
            const float c = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mx - now);
            mx = now;
            l *= c;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= c;
        }
        const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, -ref));
            l += s[e];
            if constexpr (F8) s[e] *= vs[e];
        }
        return pieces_of<NW, kValues>(s);
    };
    const auto accumulate = [&](const uint8_t *lds, const Pieces<NW> &pf) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            uint4 v;
            if constexpr (F8) {
                v = widen_e4m3(lds_tr8(lds, v_at[d]));
            } else {
                const uint2 v0 = lds_tr16(lds, v_at[d]), v1 = lds_tr16(lds, v_at[d] + 16 * RB);
                v = make_uint4(v0.x, v0.y, v1.x, v1.y);
            }
#pragma unroll
            for (int q = NW - 1; q >= 0; --q) o[d] = mfma16(v, pf.p[q], o[d]);
        }
        if constexpr (HALVES) {
            __builtin_amdgcn_sched_group_barrier(0x100, 2 * DT, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, DT * NW, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto step = [&](auto which, int i) __attribute__((always_inline)) {
        constexpr int st = decltype(which)::value;
        constexpr int ahead = (st + NS - 1) % NS;
        issue(Int<ahead>{}, i + NS - 1);
        wait_loads<S::kTokenLoads *(NS - 1)>();
        float s[8], ks[8], vs[8];
        if constexpr (F8) {
            scales[wave][lane] = sc[st];
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ks[4 * m + e] = scales[wave][16 * m + 4 * lg + e];
                    vs[4 * m + e] = scales[wave][32 + 16 * m + 4 * lg + e];
                }
        }
        products(stage(which), s);
        if constexpr (F8)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] *= ks[e];
        accumulate(stage(which), weights(i, ok[st][0], ok[st][1], s, vs));
    };
    if constexpr (HALVES) {
        // The next unit's keys are loaded once the keys are multiplied, its values once these are:
        // a half is always on its way, and a CU has twice the wavefronts that whole stages would
        // leave room for.
        Rows16 r[2], next[2];
        rows_of(0, r);
        load_keys(0, r, stage(Int<0>{}));
        load_values(0, r, stage(Int<1>{}));
        __builtin_amdgcn_sched_barrier(0);
        for (int i = 0; i < steps; ++i) {
            float s[8], vs[8];
            rows_of(i + 1, next);
            wait_loads<S::kTokenLoads / 2>();
            products(stage(Int<0>{}), s);
            __builtin_amdgcn_sched_barrier(0);
            load_keys(i + 1, next, stage(Int<0>{}));
            __builtin_amdgcn_sched_barrier(0);
            const Pieces<NW> pf = weights(i, r[0].ok, r[1].ok, s, vs);
            wait_loads<S::kTokenLoads / 2>();
            accumulate(stage(Int<1>{}), pf);
            load_values(i + 1, next, stage(Int<1>{}));
            __builtin_amdgcn_sched_barrier(0);
            r[0] = next[0];
            r[1] = next[1];
        }
    } else {
        issue(Int<0>{}, 0);
        if constexpr (NS == 4) {
            issue(Int<1>{}, 1);
            issue(Int<2>{}, 2);
        }
        int i = 0;
        while (true) {
            step(Int<0>{}, i);
            if (++i == steps) break;
            step(Int<1>{}, i);
            if (++i == steps) break;
            if constexpr (NS == 4) {
                step(Int<2>{}, i);
                if (++i == steps) break;
                step(Int<3>{}, i);
                if (++i == steps) break;
            }
        }
    }
    l = sum_xor32(sum_xor16(l));
    if (n < a.GR) {
        const size_t at = unsigned((2 * (w * a.G + g) + max(part, 0)) * a.GR + n);
        const int64_t out = row * a.out_stride + (g * a.GR + n) * HD;
        const float inv = 1.f / l;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int dim = 16 * d + 4 * lg;
            if (part >= 0) {
                *reinterpret_cast<floatx4 *>(a.part_o + at * HD + dim) = o[d];
                continue;
            }
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = l == 0.f ? 0.f : o[d][e] * inv;
            if constexpr (F32)
                *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + out + dim) =
                    make_float4(v[0], v[1], v[2], v[3]);
            else
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + out + dim) =
                    make_uint2(pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3]));
        }
        if (part >= 0 && lg == 0) a.part_ml[at] = make_float2(mx, l);
    }
    if (z == tile_lo && lane == 0)
        a.split[size_t(tile) * a.G + g] = {int(row), a.GR, 2 * (w * a.G + g) + part,
                                           part < 0 ? 0 : shares.worker_of(tile_hi - 1) - w};
    z += steps;
    }
    wait_loads<0>();   // no load into LDS outlives the workgroup
}

// ---------------------------------------------------------------------- tiles of many rows
// A tile is up to 128 rows: 128 / GR consecutive tokens of a request with the GR query heads of a
// group, row = token * GR + head.  Each of four wavefronts owns 32 rows, columns of the 32x32x16
// products; units of 64 positions are staged in LDS for all four, the next one in flight while
// one is multiplied (one barrier per unit).  Lane (q = lane % 32, h = lane / 32) holds the
// scores of row q at positions 32 m + 8 (i / 4) + 4 h + i % 4.
// Bound by the matrix cores and what they wait for: 4096 tokens of 32 heads of 128 behind 12288
// positions (962 GFLOP) 900-930 us, 1030-1070 TFLOP/s, where a library's product of 8192^3 gets 1198 and
// both are held back by the card's power (clocks of 1.9 and 1.8 GHz).  Of a unit's 4400 cycles
// (two workgroups on a CU) the products take half; the rest are the softmax's 32 maxima and
// exponentials a lane, which the other workgroup's products overlap, and the wait for the loads.
// E4M3 codes are widened once for the four wavefronts (by each where it reads them: half as long
// again).  Their weights, times the values' scales, go through the second product in two bf16
// pieces, 16 bits: the same chunk 1330-1360 us.  One piece, 1090, errs up to 1.8 times as much as the
// rounding of the result, as alike rows have alike scales; one of fp16, 1140-1160, loses what is 25
// powers of two below a row's largest product but in its normaliser, and with it outputs that such
// positions make up.  fp32 in three pieces: 370-380 TFLOP/s without counting them three times.
constexpr int kTileRows = 128;
// Units of a share at least: a part is 64 KB.  64 tokens behind 1000 positions, heads of 128: 22.0
// us with 2 (and with 1), 25.1 with 4, 34.2 with 16; 64 tokens behind 8000: 36.0, with 4 34.0.
constexpr int kMinShare = 2;
constexpr int kBadPage = 1, kOdd = 2;

struct TileScratch {                // in LDS
    float scales[2][2][kTileUnit];      // keys' times scale_log2; values'
    uint8_t group_flags[2][4];          // of a unit's 16 rows each: kBadPage, kOdd
    int wave_odd[kWaves];
};

template <int HD, bool F8, bool F32>
__device__ __forceinline__ void attend_tile(const AttendArgs &a, TileList &list, int tiles, const Stages &lds_stages,
                                            TileScratch &scratch) {
    constexpr int RB = HD * 2, KS = HD / 16, DT = HD / 32;
    constexpr int NP = F32 ? 3 : 1, NW = F32 ? 3 : F8 ? 2 : 1;   // pieces of a query value and of a weight
    constexpr Infinity kValues = F8 ? Infinity::never : Infinity::meets;   // (no E4M3 code is infinite)
    using KSw = KSwizzle<RB>;
    using VSw = TileVSwizzle<RB>;
    uint8_t *const st0 = lds_stages.st0, *const st1 = lds_stages.st1;   // keys, values
    float (&scales)[2][2][kTileUnit] = scratch.scales;
    uint8_t (&group_flags)[2][4] = scratch.group_flags;
    int (&wave_odd)[kWaves] = scratch.wave_odd;
    const int w = uniform(blockIdx.x / a.G), g = blockIdx.x - w * a.G;
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int n = lane & 31, h = lane >> 5;
    const int all_units = uniform(list.cu[tiles]);
    // Whole tiles, the last ones (of a request: the longest) first, or even shares of the units.
    // In units: even shares take all / workers and kSplitCost for as many parts as they leave;
    // whole tiles as long as the longest one (which runs faster towards the end, alone on its
    // CU), or all / workers and what the last round, the first `rest` tiles, leaves idle.
    // Whole and even, us: a prompt of 2048 tokens 59 and 88, eight E4M3 chunks of 700 tokens behind
    // up to 3500 positions 181 and 182 (bf16 119 and 135), 4096 tokens behind 12288 897 and 964;
    // 512 tokens behind 4096 94 and 64, eight requests of 4 tokens 47 and 25, 2048 fp32 tokens of
    // heads of 64 behind 6144 304 and 276.
    const int workers = max(min(a.workers, all_units / kMinShare), 1);
    const int rest = tiles % a.workers;
    const float even = float(all_units) / workers, parts = float(workers + min(tiles, workers)) / (2 * a.workers);
    float longest = 0.f;
    for (int i = threadIdx.x; i < tiles; i += kThreads) longest = fmaxf(longest, float(list.cu[i + 1] - list.cu[i]));
    longest = max_xor32(max_xor16(apex::ffn::row_max(longest)));
    if (lane == 0) list.wave_end[wave] = int(longest);
    __syncthreads();
    longest = float(max(max(list.wave_end[0], list.wave_end[1]), max(list.wave_end[2], list.wave_end[3])));
    const float idle = rest ? (1.f - float(rest) / a.workers) * list.cu[rest] / rest : 0.f;
    const float whole = fmaxf((Shape<HD, F8, F32>::kPerCu == 2 ? 0.75f : 1.f) * longest,
                              float(all_units) / a.workers + idle);
    const bool whole_tiles = uniform(whole <= even + parts * Shape<HD, F8, F32>::kSplitCost);
    const Shares shares(all_units, workers);
    // Whole tiles in turns of all workgroups.  (One round: workgroup i + 256 comes to workgroup i's
    // CU, so that a long one meets a short one.)
    const int groups = gridDim.x / a.G;
    const auto whole_tile = [&](int turn) {
        return Shape<HD, F8, F32>::kPerCu == 2 && tiles <= a.workers && turn >= a.workers / 2 ? turn - a.workers / 2
                                                                                             : tiles - 1 - turn;
    };
    if (w >= (whole_tiles ? tiles : workers)) return;
    int turn = w, tile = whole_tiles ? whole_tile(w) : tile_of(list, tiles, shares.begin(w));
    int share_lo = uniform(whole_tiles ? list.cu[tile] : shares.begin(w));
    int share_hi = uniform(whole_tiles ? list.cu[tile + 1] : shares.begin(w + 1));
    const int m_row = 32 * wave + n, tok = m_row / a.GR, head = m_row - tok * a.GR;
    // where this lane reads, in a stage: keys of row n (and n + 32), values of rows v_row and
    // v_row + 8 of 16; the swizzles are the same 8, 16 and 32 rows further
    int k_at[KS], v_at[DT];
    constexpr int kV = kTileUnit * RB;   // the values' place
    const int v_row = 4 * h + ((lane & 15) >> 2);
#pragma unroll
    for (int u = 0; u < KS; ++u) k_at[u] = settled(n * RB + 16 * ((2 * u + h) ^ KSw::of(n)));
#pragma unroll
    for (int d = 0; d < DT; ++d)
        v_at[d] = settled(kV + v_row * RB + 8 * (lane & 1) +
                          16 * ((4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ VSw::of(v_row)));
    const GlobalFloats scale_of = lane_pointer(a.k_scales, a.v_scales, lane & 16);

    // the share's tiles
#pragma unroll 1
    for (int z = share_lo; z < share_hi; ++tile) {
    const int tile_lo = uniform(list.cu[tile]), tile_hi = uniform(list.cu[tile + 1]);
    const int u_lo = uniform(z - tile_lo), steps = uniform(min(tile_hi, share_hi) - z);
    const int req = uniform(list.r[tile]), tokens = uniform(list.tokens[tile]);
    const int row0 = uniform(list.row[tile]);
    const int p_first = uniform(list.p[tile]), p_last = p_first + tokens - 1, hi = p_last + 1;
    const int low = lower_edge(p_first, a.list.window);
    const Span span = span_of(p_first, p_last, a.list.window, a.list.sinks, kTileShift);
    const int32_t *table = a.block_table + size_t(req) * a.max_blocks;
    const int part = z == tile_lo && tile_hi <= share_hi ? -1 : z == share_lo ? 0 : 1;
    const bool row_on = tok < tokens;
    const bool wave_on = 32 * wave < tokens * a.GR;
    const float slack = tokens * a.GR <= kExactRows ? 0.f : kSlack;
    const int p = row_on ? p_first + tok : -1;
    const int64_t row = row0 + (row_on ? tok : 0);
    const int col = (g * a.GR + (row_on ? head : 0)) * HD;

    Pieces<NP> qf[KS];
#pragma unroll
    for (int u = 0; u < KS; ++u)
        qf[u] = load_q<F32>(a.q, row * a.q_stride + col + 16 * u + 8 * h, row_on);

    // This wavefront's 16 rows of unit i: bf16 straight to LDS; codes by way of registers, widened
    // to bf16 once for the four wavefronts (each lane 16 codes of CPL chunks).
    constexpr int CPL = F8 ? HD / 64 : 1, CRPI = kWave * 16 / HD;   // code loads, rows of a load
    float sc = 0.f;
    bool sc_on = false, rows_ok = false;
    uint4 codes[2][CPL];
    // A unit's page id is loaded a unit ahead, as a vector load: a scalar one would be waited for
    // with the reads of LDS.
    int page = -1;
    const auto rows_at = [&](int i) { return span.base(u_lo + min(i, steps - 1), kTileShift) + 16 * wave; };
    const auto load_page = [&](int i) {
        page = ((GlobalInts)(table))[min(rows_at(i) >> a.shift, a.max_blocks - 1)];
    };
    const auto issue = [&](auto which, int i) __attribute__((always_inline)) {
        uint8_t *lds = decltype(which)::value ? st1 : st0;
        const int at = 16 * wave * RB;
        const int j = rows_at(i);
        const Rows16 r = rows_of_page(a, uniform(page), g, j, i < steps ? hi : 0);
        load_page(i + 1);
        const int from = low - j, keep = a.list.sinks - j;
        rows_ok = r.ok;
        if constexpr (F8) {
            const int x = lane & 15;   // the scales of rows that are not read are 0
            sc = scale_of[r.row + min(x, max(r.end - 1, 0))];
            sc_on = x < r.end && (x >= from || x < keep);   // (looked at where the load has been waited for)
            const Extent kx = extent_of<HD>(a.k_pages, r), vx = extent_of<HD>(a.v_pages, r);
            const auto kr = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(kx.base), 0, kx.bytes, 0x00027000);
            const auto vr = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(vx.base), 0, vx.bytes, 0x00027000);
#pragma unroll
            for (int c = 0; c < CPL; ++c) {
                const int rr = CRPI * c + lane / (HD / 16);
                const int off = rr < from && rr >= keep ? 0x40000000 : CRPI * HD * c + 16 * lane;
                codes[0][c] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(kr, off, 0, 0));
                codes[1][c] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(vr, off, 0, 0));
            }
        } else {
            load_rows16<RB, KSw>(a.k_pages, r, from, keep, lds, at, 16 * wave);
            load_rows16<RB, VSw>(a.v_pages, r, from, keep, lds, kV + at, 16 * wave);
        }
    };
    constexpr int kIssued = F8 ? 2 * CPL + 2 : RB / 32 + 1;   // loads of an issue
    // Chunk ch of row rr is 16 codes, two chunks of values: the second is at the first's place ^ 16
    // (bytes); 8 rows further a key's is at ^ 128, a value's at the same.  Places are computed
    // from one register each time: kept, they would be eight.
    const int code_row = 16 * wave + lane / (HD / 16), code_ch = 2 * (lane % (HD / 16));
    const int put_k = code_row * RB + 16 * (code_ch ^ KSw::of(code_row));
    const int put_v = kV + code_row * RB + 16 * (code_ch ^ VSw::of(code_row));
    const auto commit = [&](auto which) __attribute__((always_inline)) {
        if constexpr (F8) {
            static_assert(CPL <= 2 && (CPL == 1 || CRPI == 8), "places of the second load");
            uint8_t *lds = decltype(which)::value ? st1 : st0;
            const int pk = settled(put_k), pv = settled(put_v);
#pragma unroll
            for (int c = 0; c < CPL; ++c) {
                const uint4 k = codes[0][c], v = codes[1][c];
                *reinterpret_cast<uint4 *>(lds + ((pk ^ 128 * c) + 8 * RB * c)) = widen_e4m3(make_uint2(k.x, k.y));
                *reinterpret_cast<uint4 *>(lds + ((pk ^ 128 * c ^ 16) + 8 * RB * c)) = widen_e4m3(make_uint2(k.z, k.w));
                const uint2 v0 = make_uint2(v.x, v.y), v1 = make_uint2(v.z, v.w);
                *reinterpret_cast<uint4 *>(lds + (pv + 8 * RB * c)) = widen_e4m3(v0);
                *reinterpret_cast<uint4 *>(lds + ((pv ^ 16) + 8 * RB * c)) = widen_e4m3(v1);
            }
        }
    };

    float mx, l;    // l: of the lane's own positions
    floatx16 o[DT];

    // CAREFUL: see below
    bool met_odd = false;
    const auto step = [&](auto which, auto careful, int i) __attribute__((always_inline)) {
        constexpr int buf = decltype(which)::value;
        constexpr bool CAREFUL = decltype(careful)::value;
        if constexpr (F8) sc = sc_on ? sc : 0.f;
        if constexpr (F8)
            if (lane < 32) scales[buf][lane >> 4][16 * wave + (lane & 15)] = lane < 16 ? sc * a.scale_log2 : sc;
        wait_loads<0>();
        const int j0 = span.base(u_lo + i, kTileShift);
        const uint8_t *lds = buf ? st1 : st0;
        // whether all rows see all positions (but for bad pages)
        const bool even = j0 + kTileUnit - 1 <= p_first &&
                          (a.list.window == 0 || j0 > p_last - a.list.window || j0 + kTileUnit - 1 < a.list.sinks);
        int flags = rows_ok ? 0 : kBadPage;
        if (!even) {   // any value that is no finite number?
            uint32_t odd = 0;
#pragma unroll
            for (int c = 0; c < RB / 64; ++c) {
                const uint4 v = lds_u4(lds, kV + 16 * wave * RB + 16 * lane + 1024 * c);
                const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)   // exponents of all ones carry into the sign's place
                    odd |= ((x[e] & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
            }
            if constexpr (F8) odd |= (__float_as_uint(sc) & 0x7f800000u) == 0x7f800000u;
            if (__ballot(odd)) flags |= kOdd;
        }
        if (lane == 0) group_flags[buf][wave] = uint8_t(flags);
        lds_barrier();
        if (!wave_on) {
            issue(Int<1 - buf>{}, i + 1);
            return;
        }
        const int flags_read = *reinterpret_cast<const int *>(group_flags[buf]);
        // Keys are read AHEAD products before their own; the next unit's loads go out between the
        // products (all at once, the four wavefronts' queue up at the CU's address unit: 800 cycles).
        issue(Int<1 - buf>{}, i + 1);
        constexpr int NK = 2 * KS, AHEAD = 4;
        const auto load_k = [&](int x) { return lds_u4(lds, k_at[x % KS] + 32 * (x / KS) * RB); };
        uint4 kf[AHEAD];
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) kf[x] = load_k(x);
        float s[2][16];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            floatx16 big, small;
#pragma unroll
            for (int e = 0; e < 16; ++e) big[e] = small[e] = 0.f;
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                const int x = m * KS + u;
                const uint4 k = kf[x % AHEAD];
                if (x + AHEAD < NK) kf[x % AHEAD] = load_k(x + AHEAD);
#pragma unroll
                for (int q = NP - 1; q > 0; --q) small = mfma32(k, qf[u].p[q], small);
                big = mfma32(k, qf[u].p[0], big);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) s[m][e] = F32 ? big[e] + small[e] : big[e];
        }
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);   // LDS reads
#pragma unroll
        for (int x = 0; x < NK; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, NP, 0);  // matrix products
            if (x + AHEAD < NK) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if (x < kIssued) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);   // loads
        }
        __builtin_amdgcn_sched_barrier(0);
        const int all_flags = uniform(flags_read);
        if constexpr (F8)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[m][e] *= scales[buf][0][32 * m + 8 * (e / 4) + 4 * h + e % 4];
        const bool whole = even && !(all_flags & 0x01010101 * kBadPage);
        if (!whole) {
            // from the lane's first position on, where the others are at constants (as indices of
            // their own they would be kept in 28 registers)
            const int at = settled(j0 + 4 * h), last = p - at, first = lower_edge(p, a.list.window) - at;
            const int sinks = a.list.sinks - at;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int c = 32 * m + 8 * (e / 4) + e % 4;
                    const bool on = c <= last && (c >= first || c < sinks) && !(all_flags & kBadPage << 8 * (c / 16));
                    s[m][e] = on ? s[m][e] : -INFINITY;
                }
        }
        float top = -INFINITY;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[m][e]);
        top = F8 ? max_xor32(top) : max_xor32(top) * a.scale_log2;   // (E4M3 scores are in powers of two already)
        if (__ballot(top > mx + slack)) {
            const float now = fmaxf(mx, top);
            const float c = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mx - now);
            mx = now;
            l *= c;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= c;
        }
        const float ref = mx == -INFINITY ? 0.f : mx;
        // the weights of step u, 16 positions (8 of this lane's row)
        const auto weights = [&](int u, float (&w)[8]) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = 8 * (u & 1) + e;
                w[e] = __builtin_amdgcn_exp2f(F8 ? s[u / 2][i] - ref : fmaf(s[u / 2][i], a.scale_log2, -ref));
                l += w[e];
            }
            if constexpr (F8) {
                const float4 a4 = *reinterpret_cast<const float4 *>(&scales[buf][1][16 * u + 4 * h]);
                const float4 b4 = *reinterpret_cast<const float4 *>(&scales[buf][1][16 * u + 8 + 4 * h]);
                const float f[8] = {a4.x, a4.y, a4.z, a4.w, b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] *= f[e];
            }
        };
        // Where rows see different positions, a value that is no finite number must not meet the
        // zero weights of the rows that do not see it.  A tile that meets such a unit is worked
        // on again, carefully: that unit's products then go one by one, for the rows that see the
        // position, whatever its weight: 0 times infinity is NaN there as in any other unit.
        // (Done at once, in this loop, the compiler moves all of o between registers three times
        // a unit.)
        const bool odd = all_flags & 0x01010101 * kOdd;
        met_odd = met_odd || odd;
        if (CAREFUL && odd) {
            float all_w[4][8];
#pragma unroll
            for (int u = 0; u < 4; ++u) weights(u, all_w[u]);
#pragma unroll 1
            for (int j = 0; j < kTileUnit; ++j) {
                float w = 0.f;
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (16 * u + 8 * (e / 4) + e % 4 == (j & ~4)) w = all_w[u][e];
                const float other = __shfl_xor(w, 32);
                w = ((j >> 2) & 1) == h ? w : other;
                const bool on = visible(j0 + j, p, a.list.window, a.list.sinks);   // (rows of bad pages are 0)
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e4 = 0; e4 < 4; ++e4) {
                        const uint2 c = lds_u2(lds, kV + j * RB + 16 * ((4 * d + e4) ^ VSw::of(j)) + 8 * h);
                        const float v[4] = {apex::ffn::bf_lo(c.x), apex::ffn::bf_hi(c.x), apex::ffn::bf_lo(c.y),
                                            apex::ffn::bf_hi(c.y)};
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[d][4 * e4 + e] = on ? fmaf(w, v[e], o[d][4 * e4 + e]) : o[d][4 * e4 + e];
                    }
            }
            return;
        }
        // The products of a step run while the next one's values are read and its weights computed.
        const auto load_v = [&](int u, int d) {
            const uint2 v0 = lds_tr16(lds, v_at[d] + 16 * u * RB);
            const uint2 v1 = lds_tr16(lds, v_at[d] + (16 * u + 8) * RB);
            return make_uint4(v0.x, v0.y, v1.x, v1.y);
        };
        __builtin_amdgcn_sched_barrier(0);
        uint4 vf[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) vf[d] = load_v(0, d);
        float w[8];
        weights(0, w);
        Pieces<NW> pf = pieces_of<NW, kValues>(w);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            uint4 vn[DT];
            Pieces<NW> pn;
            if (u < 3) {
#pragma unroll
                for (int d = 0; d < DT; ++d) vn[d] = load_v(u + 1, d);
                weights(u + 1, w);
                pn = pieces_of<NW, kValues>(w);
            }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int q = NW - 1; q >= 0; --q) o[d] = mfma32(vf[d], pf.p[q], o[d]);
            if (u < 3) {
#pragma unroll
                for (int x = 0; x < DT * NW; ++x) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);              // a product
                    if (x < DT) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);   // values of the next step
                    __builtin_amdgcn_sched_group_barrier(0x002, F32 ? 9 : NW == 2 ? 32 / DT : 28 / DT, 0);
                    __builtin_amdgcn_sched_group_barrier(0x400, 8 / DT, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int d = 0; d < DT; ++d) vf[d] = vn[d];
                pf = pn;
            }
        }
    };
    const auto clear = [&] {
        mx = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    };
    const auto work = [&](auto careful) __attribute__((always_inline)) {
        clear();
        commit(Int<0>{});
        for (int i = 0; i < steps; i += 2) {
            step(Int<0>{}, careful, i);
            commit(Int<1>{});
            if (i + 1 < steps) {
                step(Int<1>{}, careful, i + 1);
                commit(Int<0>{});
            }
        }
    };
    load_page(0);
    issue(Int<0>{}, 0);
    work(Int<0>{});
    if (lane == 0) wave_odd[wave] = met_odd;
    wait_loads<0>();
    __syncthreads();
    if (wave_odd[0] | wave_odd[1] | wave_odd[2] | wave_odd[3]) {
        load_page(0);
        issue(Int<0>{}, 0);
        work(Int<1>{});
    }
    wait_loads<0>();
    l = sum_xor32(l);
    if (!row_on) {
        // no row of the tile
    } else if (part < 0) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const int64_t at = row * a.out_stride + col + 32 * d + 8 * e4 + 4 * h;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = l == 0.f ? 0.f : o[d][4 * e4 + e] * inv;
                if constexpr (F32)
                    *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) =
                        make_float4(v[0], v[1], v[2], v[3]);
                else
                    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) =
                        make_uint2(pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3]));
            }
    } else {
        const size_t at = unsigned((2 * (w * a.G + g) + part) * kTileRows + settled(m_row));
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                *reinterpret_cast<float4 *>(a.part_o + at * HD + 32 * d + 8 * e4 + 4 * h) =
                    make_float4(o[d][4 * e4], o[d][4 * e4 + 1], o[d][4 * e4 + 2], o[d][4 * e4 + 3]);
        if (h == 0) a.part_ml[at] = make_float2(mx, l);
    }
    if (z == tile_lo && threadIdx.x == 0)
        a.split[size_t(tile) * a.G + g] = {row0, tokens * a.GR, 2 * (w * a.G + g) + part,
                                           part < 0 ? 0 : shares.worker_of(tile_hi - 1) - w};
    z += steps;
    if (whole_tiles && (turn += groups) < tiles) {
        tile = whole_tile(turn) - 1;
        z = share_lo = uniform(list.cu[tile + 1]);
        share_hi = uniform(list.cu[tile + 2]);
    }
    if (z < share_hi) __syncthreads();   // the stages are free again
    }
}

template <int HD, bool F8, bool F32>
__global__ __launch_bounds__(kThreads, (Shape<HD, F8, F32>::kPerCu)) void attend(AttendArgs a) {
    using S = Shape<HD, F8, F32>;
    constexpr bool FOUR = S::kTokenStages == 4;
    __shared__ __align__(1024) uint8_t st0[S::kStage], st1[S::kStage];
    __shared__ __align__(1024) uint8_t st2[FOUR ? S::kStage : 16], st3[FOUR ? S::kStage : 16];
    __shared__ __align__(16) float token_scales[kWaves][64];
    __shared__ __align__(16) TileScratch scratch;
    __shared__ TileList list;
    bool one_by_one;
    const int tiles = build_list(a.list, list, one_by_one);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.tiles = make_int2(tiles, one_by_one);
    if (tiles == 0) return;
    const Stages stages{st0, st1, st2, st3};
    if (one_by_one)
        attend_token<HD, F8, F32>(a, list, tiles, stages, token_scales);
    else
        attend_tile<HD, F8, F32>(a, list, tiles, stages, scratch);
}

// --------------------------------------------------------------------------------- merge
struct MergeArgs {         // small: a launch this short waits for its arguments
    void *out;
    int64_t out_stride;
    const Split *split;
    const int2 *tiles;
    const float *part_o;
    const float2 *part_ml;
    int G, GR;
};

// Part s of a split tile: the first worker's, then the next ones' first parts (even ones).
__device__ __forceinline__ size_t part_of(const Split &sp, int G, int s) {
    return s == 0 ? size_t(sp.part) : size_t(sp.part & ~1) + size_t(s) * 2 * G;
}

// Tiles of one token: workgroup (tile * G + g, h) of N threads takes a row.  The parts fall into 4096
// / HD sums, part s into sum s mod these, each taken by HD / 4 threads; they meet in LDS.  (As many
// sums whatever N, which goes by T: empty rows of q change no bit of the others.)
template <int HD, bool F32, int N>
__device__ __forceinline__ void merge_token(const MergeArgs &a, const Split &sp) {
    constexpr int LPR = HD / 4, SUMS = 1024 / LPR, WAVES = N / kWave;
    __shared__ float red_m[WAVES], red_d[SUMS];
    __shared__ __align__(16) float red[SUMS][HD];
    const int t = threadIdx.x, wave = t / kWave, lane = t % kWave, at4 = t % LPR;
    const int g = blockIdx.x % a.G, h = blockIdx.y;
    if (h >= a.GR) return;
    float top = -INFINITY;
    for (int s = t; s <= sp.more; s += N)
        top = fmaxf(top, a.part_ml[part_of(sp, a.G, s) * a.GR + h].x);
    top = max_xor32(max_xor16(apex::ffn::row_max(top)));
    if (lane == 0) red_m[wave] = top;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < WAVES; ++v) top = fmaxf(top, red_m[v]);
    const int sums = min(SUMS, sp.more + 1);
#pragma unroll 1
    for (int q = t / LPR; q < sums; q += N / LPR) {
        float den = 0.f;
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4   // (8 take more registers than leave a CU full, which the merge of tiles shares)
        for (int s = q; s <= sp.more; s += SUMS) {
            const size_t at = part_of(sp, a.G, s) * a.GR + h;
            const float2 ml = a.part_ml[at];
            const float4 o = reinterpret_cast<const float4 *>(a.part_o + at * HD)[at4];
            const float c = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
            den = fmaf(ml.y, c, den);
            num.x = fmaf(o.x, c, num.x);
            num.y = fmaf(o.y, c, num.y);
            num.z = fmaf(o.z, c, num.z);
            num.w = fmaf(o.w, c, num.w);
        }
        *reinterpret_cast<float4 *>(&red[q][4 * at4]) = num;
        if (at4 == 0) red_d[q] = den;
    }
    __syncthreads();
    if (t < HD) {
        float d = 0.f, v = 0.f;
#pragma unroll 4
        for (int q = 0; q < sums; ++q) {
            d += red_d[q];
            v += red[q][t];
        }
        store_out<F32>(a.out, sp.row * a.out_stride + (g * a.GR + h) * HD + t, d == 0.f ? 0.f : v / d);
    }
}

// Tiles of many rows: workgroups (tile * G + g, y) of kThreads at work, HD / 4 lanes per row (more
// threads on fewer rows' parts: 64 tokens behind 8000 positions 12.9 us instead of 8.6).  Bound by
// the parts it reads, 64 KB each: 33 MB 10.5 us behind the launch before; 5 where no tile was split.
template <int HD, bool F32>
__device__ __forceinline__ void merge_tile(const MergeArgs &a, const Split &sp) {
    constexpr int LPR = HD / 4, PER = kThreads / LPR;   // rows at a time
    if (threadIdx.x >= kThreads) return;
    const int at4 = threadIdx.x % LPR, g = blockIdx.x % a.G;
    for (int m = blockIdx.y * PER + threadIdx.x / LPR; m < sp.rows; m += gridDim.y * PER) {
        float top = -INFINITY;
#pragma unroll 8
        for (int s = 0; s <= sp.more; ++s) top = fmaxf(top, a.part_ml[part_of(sp, a.G, s) * kTileRows + m].x);
        float den = 0.f;
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int s = 0; s <= sp.more; ++s) {
            const size_t at = part_of(sp, a.G, s) * kTileRows + m;
            const float2 ml = a.part_ml[at];
            const float4 o = reinterpret_cast<const float4 *>(a.part_o + at * HD)[at4];
            const float c = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
            den = fmaf(ml.y, c, den);
            num.x = fmaf(o.x, c, num.x);
            num.y = fmaf(o.y, c, num.y);
            num.z = fmaf(o.z, c, num.z);
            num.w = fmaf(o.w, c, num.w);
        }
        const int tok = m / a.GR, head = m - tok * a.GR;
        const int64_t at = (int64_t(sp.row) + tok) * a.out_stride + (g * a.GR + head) * HD + 4 * at4;
        const float v[4] = {num.x, num.y, num.z, num.w};
        float r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = den == 0.f ? 0.f : v[e] / den;
        if constexpr (F32)
            *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = make_float4(r[0], r[1], r[2], r[3]);
        else
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) =
                make_uint2(pk_bf16(r[0], r[1]), pk_bf16(r[2], r[3]));
    }
}

template <int HD, bool F32, int N>
__global__ __launch_bounds__(N) void merge(MergeArgs a) {
    const Split sp = a.split[blockIdx.x];
    const int2 tiles = *a.tiles;
    // what is needed behind the branch is loaded before it, in one round trip
    asm volatile("" ::"s"(a.part_o), "s"(a.part_ml), "s"(a.GR), "s"(tiles.x), "s"(tiles.y));
    if (int(blockIdx.x) >= tiles.x * a.G || sp.more <= 0) return;
    if (tiles.y)
        merge_token<HD, F32, N>(a, sp);
    else
        merge_tile<HD, F32>(a, sp);
}

// ---------------------------------------------------------------------------------- host
// What a call's workspace holds, whichever kind of tiles its lengths take: room for the most
// workers that a CU may hold, whatever the types.
struct Plan {
    bool tiles;                     // of many rows, perhaps: one row of q has one token
    bool likely_tokens;             // one by one: no more rows than requests
    int GR, tile_tokens, max_tiles;
    size_t at_ml, at_o, bytes;
};
Plan plan_of(int T, int R, int H, int G, int hd) {
    Plan p;
    p.GR = H / G;
    p.tiles = T > 1;
    p.likely_tokens = T <= R;
    p.tile_tokens = kTileRows / p.GR;
    // the sum of ceil(n / tile_tokens) over min(T, R) requests that have any of T tokens; as many
    // as there are tokens where these are no more than the requests
    p.max_tiles = int(std::min((T + int64_t(p.tile_tokens - 1) * std::min(T, R)) / p.tile_tokens,
                               int64_t(INT_MAX)));
    const int most = std::max(1, (hd == 128 ? 2 : 3) * kCus / G);   // workgroups that share out a head's units
    const int token_workers = kWaves * most, workers = p.tiles ? most : 0;
    const auto up = [](size_t v) { return apex::align_up(v, 256); };
    const size_t rows = 2 * size_t(G) * std::max(size_t(token_workers) * p.GR, size_t(workers) * kTileRows);
    p.at_ml = 256 + up(size_t(std::min(p.max_tiles, kListTiles)) * G * sizeof(Split));
    p.at_o = p.at_ml + up(rows * sizeof(float2));
    p.bytes = p.at_o + up(rows * hd * sizeof(float));
    return p;
}

template <int HD, bool F8, bool F32>
apex_status launch_attention(const Plan &p, hipStream_t st, AttendArgs a) {
    using S = Shape<HD, F8, F32>;
    a.workers = std::max(1, kCus * S::kPerCu / a.G);
    a.token_workers = a.workers * kWaves;
    const MergeArgs m{a.out, a.out_stride, a.split, a.tiles, a.part_o, a.part_ml, a.G, a.GR};
    // a launch's units are counted in 32 bits
    const int at_once = std::min(kListTiles, INT_MAX / (a.list.room / kTokenUnit + 2));
    for (int f = 0; f < p.max_tiles; f += at_once) {
        const int tiles = std::min(p.max_tiles - f, at_once), x = tiles * a.G;
        a.list.first_tile = f;
        a.list.most_tiles = tiles;
        // no more workers than there can be shares
        const auto held = [&](int workers, int64_t units) { return int(std::min(int64_t(workers), tiles * units + 1)); };
        int groups = (held(a.token_workers, a.list.room / kTokenUnit + 1) + kWaves - 1) / kWaves;
        if (p.tiles) groups = std::max(groups, held(a.workers, (a.list.room / kTileUnit + 1) / kMinShare + 1));
        // A workgroup for each tile, so that the GPU hands them out as they end, unless there are
        // likely to be none (each of them would list the launch's tiles: 1024 single tokens 360 us
        // instead of 305).
        if (!p.likely_tokens) groups = std::max(groups, tiles);
        hipLaunchKernelGGL((attend<HD, F8, F32>), dim3(groups * a.G), dim3(kThreads), 0, st, a);
        // Few tokens have many parts: 4 requests of up to 131072 positions in 8 groups 4.8 us with 1024
        // threads, 6.1 with 512; 256 requests' tiles of a few parts each 5.5 with 256, 18.9 with 1024.
        const int n = p.likely_tokens && x <= 64 ? 1024 : 256, turns = kTileRows / (kThreads / (HD / 4));
        const dim3 grid(x, std::max(a.GR, p.tiles ? std::min(8192 / x, turns) : 1));
        if (n == 1024)
            hipLaunchKernelGGL((merge<HD, F32, 1024>), grid, dim3(1024), 0, st, m);
        else
            hipLaunchKernelGGL((merge<HD, F32, 256>), grid, dim3(256), 0, st, m);
        APEX_HIP(hipGetLastError());
    }
    return APEX_OK;
}

template <int HD>
apex_status launch_attention(const Plan &p, bool f8, bool f32, hipStream_t st, const AttendArgs &a) {
    return f8 ? (f32 ? launch_attention<HD, true, true>(p, st, a) : launch_attention<HD, true, false>(p, st, a))
              : (f32 ? launch_attention<HD, false, true>(p, st, a) : launch_attention<HD, false, false>(p, st, a));
}

}  // namespace

extern "C" size_t apex_attention_paged_workspace_bytes(int T, int R, int H, int G, int hd) {
    if (T <= 0 || R <= 0 || G <= 0 || H < G || H / G > kMaxGroup || hd <= 0) return 256;
    return plan_of(T, R, H, G, hd).bytes;
}

extern "C" apex_status apex_attention_paged(const apex_paged_cache *cache, const void *q, int dtype,
                                            int T, int R, int H, int64_t q_stride,
                                            const int32_t *cu_new, const int32_t *seq_len,
                                            const int32_t *block_table, int max_blocks, int window,
                                            int sinks, float scale, void *out, int64_t out_stride,
                                            void *workspace, size_t workspace_bytes,
                                            hipStream_t stream) {
    const char *fn = "apex_attention_paged";
    APEX_REQUIRE(T >= 0 && R >= 0, "%s: T=%d and R=%d must be >= 0", fn, T, R);
    if (T > APEX_MAX_STEP_TOKENS)
        return apex::fail(APEX_E_UNSUPPORTED, "%s: T=%d exceeds %d", fn, T, APEX_MAX_STEP_TOKENS);
    apex_status st = apex::check_paged_cache(fn, cache, T > 0 && R > 0);
    if (st != APEX_OK) return st;
    const int G = cache->G, hd = cache->hd, page_size = cache->page_size;
    APEX_REQUIRE(dtype == APEX_TYPE_FP32 || dtype == APEX_TYPE_BF16, "%s: unknown type %d", fn, dtype);
    APEX_REQUIRE(H >= G && H % G == 0, "%s: H=%d must be a multiple of G=%d", fn, H, G);
    if (H / G > kMaxGroup)
        return apex::fail(APEX_E_UNSUPPORTED, "%s: %d query heads per group exceed %d", fn, H / G,
                          kMaxGroup);
    if (R > APEX_MAX_REQUESTS)
        return apex::fail(APEX_E_UNSUPPORTED, "%s: R=%d exceeds %d", fn, R, APEX_MAX_REQUESTS);
    APEX_REQUIRE(max_blocks >= 1, "%s: max_blocks=%d must be >= 1", fn, max_blocks);
    if (int64_t(max_blocks) * page_size >= (int64_t(1) << 31))
        return apex::fail(APEX_E_UNSUPPORTED, "%s: table rows of %d pages of %d positions: 2^31 or more",
                          fn, max_blocks, page_size);
    APEX_REQUIRE(window >= 0 && sinks >= 0, "%s: window=%d and sinks=%d must be >= 0", fn, window, sinks);
    APEX_REQUIRE(scale > 0.f && scale * kLog2e < INFINITY,   // (what scores are multiplied by)
                 "%s: scale=%g must be positive and below 2.3e38", fn, double(scale));
    if ((st = apex::check_rows(fn, "q", dtype, q_stride, int64_t(H) * hd)) != APEX_OK) return st;
    if ((st = apex::check_rows(fn, "out", dtype, out_stride, int64_t(H) * hd)) != APEX_OK) return st;
    if (T == 0 || R == 0) return APEX_OK;
    APEX_REQUIRE(q && cu_new && seq_len && block_table && out && workspace, "%s: NULL pointer", fn);
    APEX_REQUIRE(apex::aligned16(q) && apex::aligned16(out) && apex::aligned16(workspace),
                 "%s: q, out and workspace must be 16-byte aligned", fn);
    APEX_REQUIRE(reinterpret_cast<uintptr_t>(cu_new) % 4 == 0 &&
                     reinterpret_cast<uintptr_t>(seq_len) % 4 == 0 &&
                     reinterpret_cast<uintptr_t>(block_table) % 4 == 0,
                 "%s: misaligned lengths or table", fn);
    const Plan p = plan_of(T, R, H, G, hd);
    if (workspace_bytes < p.bytes)
        return apex::fail(APEX_E_CAPACITY, "%s: workspace %zu < %zu bytes", fn, workspace_bytes, p.bytes);
    char *ws = static_cast<char *>(workspace);
    AttendArgs a;
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.k_pages = static_cast<const uint8_t *>(cache->k_pages);
    a.v_pages = static_cast<const uint8_t *>(cache->v_pages);
    a.k_scales = cache->k_scales;
    a.v_scales = cache->v_scales;
    a.block_table = block_table;
    a.list = {cu_new, seq_len, R, T, max_blocks * page_size, p.tile_tokens, 0, 0, window, sinks};
    a.G = G;
    a.GR = p.GR;
    a.max_blocks = max_blocks;
    a.shift = apex::log2_of(page_size);
    a.page_size = page_size;
    a.n_pages = cache->n_pages;
    a.scale_log2 = scale * kLog2e;
    a.tiles = reinterpret_cast<int2 *>(ws);
    a.split = reinterpret_cast<Split *>(ws + 256);
    a.part_ml = reinterpret_cast<float2 *>(ws + p.at_ml);
    a.part_o = reinterpret_cast<float *>(ws + p.at_o);
    const bool f32 = dtype == APEX_TYPE_FP32, f8 = cache->format == APEX_KV_FP8_E4M3;
    return hd == 64 ? launch_attention<64>(p, f8, f32, stream, a) : launch_attention<128>(p, f8, f32, stream, a);
}
