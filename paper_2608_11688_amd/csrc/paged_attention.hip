// Attention of new tokens over a paged cache (apex_attention_paged).
//
// Launches of a call:
//   schedule  one workgroup: the query tiles of all requests, the key/value units each of them
//             sees, and the items (tile, range of units) that the next launch works on.
//   attend    grid (G, items), one workgroup per item and key/value head.  Tiles of one token
//             (attend_token) or of up to 128 query rows, heads of one group and consecutive
//             tokens (attend_tile).  A tile that is one item writes its rows; the items of one
//             that is split write weighted sums, maxima and normalisers to the workspace.
//   merge     the items of split tiles joined by the log-sum-exp rule.
//
// Both kernels compute S^T = K Q^T and O^T = V^T P^T on the matrix cores: a lane then holds the
// scores of one query row in its registers, so that maxima, sums and rescaling are a lane's own
// (but for one or two exchanges between lanes of a row), and the scores' registers are the
// second product's operand as they stand.  The order of the positions within a step, which the
// first product's registers give, is taken over by the loads of V^T (transposing reads of LDS).
// Keys and values go from memory to LDS directly, by buffer loads whose descriptor is a page's
// 16 rows: rows past the last position, under the window or of a bad page lie past the
// descriptor's end and are written as zeros, so nothing that is not visible to a tile is read.
#include <hip/hip_runtime.h>

#include <algorithm>
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

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMaxGroup = 16;      // query heads per key/value head
constexpr float kLog2e = 1.4426950408889634f;
// Weights are 2^(score - m) for a reference m that is raised to the running maximum only when
// that is more than kSlack above it: they stay below 2^kSlack, where sums in 32 bits and
// roundings, which are relative, are as good, and rescaling is rare.
constexpr float kSlack = 8.f;

// ------------------------------------------------------------------------------ schedule
struct Item {
    int r, q0;          // request, first token of the tile (from the request's first new one)
    int u_lo, u_hi;     // its units, of those the tile sees
    int part;           // where its partial results go, or -1: it is the whole tile
    int pad[3];
};
struct SplitTile {
    int r, q0, part, n;   // the tile's first partial result and their number
};
struct Header {
    int n_items, n_split, pad[2];
};

// The positions a tile of tokens [q0, q1) of a request sees: sink units from 0 up, then the
// units from `first` up to the last token's position.  UP: positions of a unit.
struct Span {
    int sinks, first, units;
    __device__ __forceinline__ int base(int u, int UP) const {
        return (u < sinks ? u : first + u - sinks) * UP;
    }
};
template <int UP>
__device__ __forceinline__ Span span_of(int p_first, int p_last, int window, int sinks) {
    Span s;
    const int low = window > 0 ? max(0, p_first - window + 1) : 0;
    s.first = low / UP;
    s.sinks = window > 0 ? min((min(sinks, p_last + 1) + UP - 1) / UP, s.first) : 0;
    s.units = p_last < 0 ? 0 : p_last / UP + 1 - s.first + s.sinks;
    return s;
}

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
__device__ __forceinline__ Request scalar_request(const int32_t *cu_new, const int32_t *seq_len, int r,
                                                  int T, int room) {
    const int a = min(max(scalar_load(cu_new, r), 0), T);
    const int b = min(max(scalar_load(cu_new, r + 1), a), T);
    return {a, b - a, min(max(scalar_load(seq_len, r), 0), room)};
}
__device__ __forceinline__ Item scalar_item(const Item *items, int i) {
    const int *p = reinterpret_cast<const int *>(items + i);
    return {scalar_load(p, 0), scalar_load(p, 1), scalar_load(p, 2), scalar_load(p, 3), scalar_load(p, 4), {}};
}

struct ScheduleArgs {
    const int32_t *cu_new, *seq_len;
    int R, T, room, tile_tokens, max_tiles, window, sinks, target, G, max_items, max_split;
    Header *head;
    Item *items;
    SplitTile *split;
};

constexpr int kSchedThreads = 1024;

__device__ __forceinline__ int block_scan(int v, int *total, int *buf) {   // exclusive
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    int x = v;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int o = __shfl_up(x, d);
        if (lane >= d) x += o;
    }
    __syncthreads();
    if (lane == kWave - 1) buf[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kSchedThreads / kWave; ++w) {
        if (w < wave) before += buf[w];
        all += buf[w];
    }
    *total = all;
    return before + x - v;
}

// Tiles in descending order (a request's last tile sees most).  Every tile is cut into items of
// at most s units, s chosen so that all items together, times G, come to about `target`.
template <int UP>
__global__ __launch_bounds__(kSchedThreads) void schedule(ScheduleArgs a) {
    __shared__ int32_t cu_tiles[APEX_MAX_REQUESTS + 1];
    __shared__ int buf[kSchedThreads / kWave];
    __shared__ long long unit_sum;
    const int t = threadIdx.x;
    if (t == 0) {
        unit_sum = 0;
        cu_tiles[0] = 0;
    }
    int tiles = 0;
    for (int r0 = 0; r0 < a.R; r0 += kSchedThreads) {
        const int r = r0 + t;
        int n = 0, all;
        if (r < a.R) {
            const Request q = request_of(a.cu_new, a.seq_len, r, a.T, a.room);
            n = (q.n + a.tile_tokens - 1) / a.tile_tokens;
        }
        const int at = tiles + block_scan(n, &all, buf);
        // more than max_tiles only where cu_new is no ascending list
        if (r < a.R) cu_tiles[r + 1] = min(at + n, a.max_tiles);
        tiles = min(tiles + all, a.max_tiles);
    }
    __syncthreads();
    struct Tile {
        int r, q0, units;
    };
    const auto tile_at = [&](int i) {
        const int k = tiles - 1 - i;
        int lo = 0, hi = a.R;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cu_tiles[mid] <= k)
                lo = mid;
            else
                hi = mid;
        }
        const Request q = request_of(a.cu_new, a.seq_len, lo, a.T, a.room);
        const int q0 = (k - cu_tiles[lo]) * a.tile_tokens, q1 = min(q0 + a.tile_tokens, q.n);
        const int base = q.seq - q.n;
        return Tile{lo, q0, span_of<UP>(max(base + q0, 0), base + q1 - 1, a.window, a.sinks).units};
    };
    long long sum = 0;
    for (int i = t; i < tiles; i += kSchedThreads) sum += tile_at(i).units;
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) sum += __shfl_xor(sum, d);
    if (t % kWave == 0) atomicAdd(reinterpret_cast<unsigned long long *>(&unit_sum), sum);
    __syncthreads();
    const long long want = (unit_sum * a.G + a.target - 1) / a.target;
    const int s = int(max(want, 1ll));
    int items = 0, parts = 0, splits = 0;
    for (int i0 = 0; i0 < tiles; i0 += kSchedThreads) {
        const int i = i0 + t;
        Tile tile{0, 0, 0};
        int n = 0;
        if (i < tiles) {
            tile = tile_at(i);
            n = max(1, (tile.units + s - 1) / s);
        }
        int all_items, all_parts, all_splits;
        const int at = items + block_scan(n, &all_items, buf);
        const int part = parts + block_scan(n > 1 ? n : 0, &all_parts, buf);
        const int sp = splits + block_scan(n > 1 ? 1 : 0, &all_splits, buf);
        for (int j = 0; j < n && at + j < a.max_items; ++j) {
            Item &it = a.items[at + j];
            it.r = tile.r;
            it.q0 = tile.q0;
            it.u_lo = int((long long)tile.units * j / n);
            it.u_hi = int((long long)tile.units * (j + 1) / n);
            it.part = n > 1 ? part + j : -1;
        }
        if (n > 1 && sp < a.max_split) a.split[sp] = {tile.r, tile.q0, part, n};
        items += all_items;
        parts += all_parts;
        splits += all_splits;
    }
    if (t == 0) {
        a.head->n_items = min(items, a.max_items);
        a.head->n_split = min(splits, a.max_split);
    }
}

// -------------------------------------------------------------------------------- device
struct AttendArgs {
    const void *q;
    void *out;
    int64_t q_stride, out_stride;
    const uint8_t *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t *cu_new, *seq_len, *block_table;
    int T, H, G, GR, tile_tokens, max_blocks, shift, page_size, n_pages, room, window, sinks;
    float scale_log2;      // the softmax scale times log2(e)
    const Header *head;
    const Item *items;
    const SplitTile *split;
    float *part_o;         // [part][G][rows][hd]
    float2 *part_ml;       // [part][G][rows]: maximum (of scores in powers of two), normaliser
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

// A matrix-core operand of 8 fp32 values: one bf16 piece each (rounded), or the three pieces of
// 8 significant bits that add up to the value exactly.
template <bool F32>
struct Pieces {
    static constexpr int N = F32 ? 3 : 1;
    uint4 p[N];
};
template <bool F32>
__device__ __forceinline__ Pieces<F32> pieces_of(const float (&in)[8]) {
    Pieces<F32> r;
    if constexpr (!F32) {
        r.p[0] = make_uint4(pk_bf16(in[0], in[1]), pk_bf16(in[2], in[3]), pk_bf16(in[4], in[5]),
                            pk_bf16(in[6], in[7]));
    } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = in[e];
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t u0 = __float_as_uint(x[2 * i]), u1 = __float_as_uint(x[2 * i + 1]);
                w[i] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);   // upper halves of u0, u1
                x[2 * i] -= __uint_as_float(u0 & 0xffff0000u);
                x[2 * i + 1] -= __uint_as_float(u1 & 0xffff0000u);
            }
            r.p[q] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    return r;
}

// 8 consecutive values of a query row (bf16 or fp32), zeros where !on.
template <bool F32>
__device__ __forceinline__ Pieces<F32> load_q(const void *q, int64_t at, bool on) {
    Pieces<F32> r;
    if constexpr (F32) {
        const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(q) + at);
        const float4 a = p[0], b = p[1];
        const float x[8] = {on ? a.x : 0.f, on ? a.y : 0.f, on ? a.z : 0.f, on ? a.w : 0.f,
                            on ? b.x : 0.f, on ? b.y : 0.f, on ? b.z : 0.f, on ? b.w : 0.f};
        r = pieces_of<true>(x);
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
__device__ __forceinline__ Rows16 rows16(const AttendArgs &a, const int32_t *table, int g, int j0,
                                         int hi) {
    Rows16 r;
    const int b = min(j0 >> a.shift, a.max_blocks - 1);
    const int page = j0 < hi ? scalar_load(table, b) : -1;
    r.ok = page >= 0 && page < a.n_pages;
    r.row = r.ok ? (int64_t(page) * a.G + g) * a.page_size + (j0 & (a.page_size - 1)) : 0;
    r.end = r.ok ? min(max(hi - j0, 0), 16) : 0;
    return r;
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
template <int RB, bool F8>
struct TileVSwizzle {    // bf16: 4 consecutive rows, four chunks; E4M3: rows 0-3 and 8-11, two
    static __device__ __forceinline__ int of(int row) {
        if (!F8) return RB == 256 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
        return RB == 128 ? 2 * (((row >> 1) & 1) | ((row >> 3) & 1) << 1) : 2 * ((row >> 3) & 1);
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
__device__ __forceinline__ GlobalFloats lane_pointer(const float *p, const float *q, bool second) {
    const uint64_t x = reinterpret_cast<uint64_t>(p), y = reinterpret_cast<uint64_t>(q);
    const int lo = settled(second ? int(y) : int(x)), hi = settled(second ? int(y >> 32) : int(x >> 32));
    return (GlobalFloats)(uint64_t(uint32_t(hi)) << 32 | uint32_t(lo));
}

// 16 rows of RB bytes, row_of.. of a tile, to LDS.  Rows below `from` and not below `keep` are
// written as zeros, as are those past r.end.
template <int RB, class SW>
__device__ __forceinline__ void load_rows16(const uint8_t *pool, const Rows16 &r, int from, int keep,
                                            uint8_t *lds, int lds_at, int row_of) {
    constexpr int CH = RB / 16, RPI = kWave / CH;   // chunks of a row, rows per load
    const int lane = threadIdx.x % kWave;
    // in scalar registers by force: a load whose descriptor the compiler does not know to be
    // uniform is wrapped in a loop over the lanes' values
    const uint64_t base = reinterpret_cast<uint64_t>(pool) + r.row * RB;
    const uint64_t at0 = uint64_t(uint32_t(uniform(int(base >> 32)))) << 32 | uint32_t(uniform(int(base)));
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(at0), 0,
                                                        uint32_t(uniform(r.end * RB)), 0x00027000);
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
// products.  Each of four wavefronts takes 32 of a unit's 128 positions, with a ring of stages
// of its own in LDS: no barrier stands in the loop, only the wavefront's own count of loads.
// Lane (q = lane % 16, lg = lane / 16) holds the scores of row q at positions 16 m + 4 lg + i.
constexpr int kTokenUnit = 128;
constexpr int kTokenRows = 16;
constexpr int kTokenTarget = 1024;   // items, all heads

template <int HD, bool F8, bool F32>
struct TokenShape {
    static constexpr int RB = HD * (F8 ? 1 : 2);
    static constexpr int kStage = 2 * 32 * RB;              // keys and values of 32 positions
    static constexpr int NS = kStage >= 16384 ? 2 : 4;      // stages
    static constexpr int kLoads = kStage / 1024 + (F8 ? 1 : 0);
};

template <int HD, bool F8, bool F32>
__global__ __launch_bounds__(kThreads) void attend_token(AttendArgs a) {
    using S = TokenShape<HD, F8, F32>;
    constexpr int RB = S::RB, NS = S::NS, KS = HD / 32, DT = HD / 16, NP = Pieces<F32>::N;
    using KSw = KSwizzle<RB>;
    using VSw = TokenVSwizzle<RB, F8>;
    // an array for each stage: the compiler then knows which loads a read of LDS has to wait for
    __shared__ __align__(1024) uint8_t st0[kWaves][S::kStage], st1[kWaves][S::kStage];
    __shared__ __align__(1024) uint8_t st2[NS > 2 ? kWaves : 1][NS > 2 ? S::kStage : 16];
    __shared__ __align__(1024) uint8_t st3[NS > 2 ? kWaves : 1][NS > 2 ? S::kStage : 16];
    __shared__ __align__(16) float scales[kWaves][64];
    __shared__ float red_m[kWaves][kTokenRows], red_l[kWaves][kTokenRows];
    static_assert(sizeof(st0) >= kWaves * kTokenRows * HD * sizeof(float), "merge room");
    const int item = uniform(blockIdx.x / a.G), g = blockIdx.x - item * a.G;
    if (item >= scalar_load(&a.head->n_items, 0)) return;
    const Item it = scalar_item(a.items, item);
    const Request rq = scalar_request(a.cu_new, a.seq_len, it.r, a.T, a.room);
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int n = lane & 15, lg = lane >> 4;
    const int p = uniform(rq.seq - rq.n + it.q0), hi = p + 1;
    const int low = a.window > 0 ? max(0, p - a.window + 1) : 0;
    const Span span = span_of<kTokenUnit>(max(p, 0), p, a.window, a.sinks);
    const int32_t *table = a.block_table + size_t(it.r) * a.max_blocks;
    const int64_t row = rq.row0 + it.q0;
    const int steps = it.u_hi - it.u_lo;

    Pieces<F32> qf[KS];
#pragma unroll
    for (int u = 0; u < KS; ++u)
        qf[u] = load_q<F32>(a.q, row * a.q_stride + (g * a.GR + (n < a.GR ? n : 0)) * HD + 32 * u + 8 * lg,
                            n < a.GR);

    // where this lane reads, in a stage: keys of row n (and n + 16), values of row v_row (and,
    // bf16, v_row + 16); both swizzles are the same 16 rows further
    int k_at[KS], v_at[DT];
    const int kv = n >> 1, v_row = F8 ? (kv < 4 ? 4 * lg + kv : 12 + 4 * lg + kv) : 4 * lg + (n >> 2);
#pragma unroll
    for (int u = 0; u < KS; ++u)
        k_at[u] = settled(wave * S::kStage + n * RB +
                          (F8 ? 16 * ((2 * u + lg / 2) ^ KSw::of(n)) + 8 * (lg & 1)
                              : 16 * ((4 * u + lg) ^ KSw::of(n))));
#pragma unroll
    for (int d = 0; d < DT; ++d)
        v_at[d] = settled(wave * S::kStage + (32 + v_row) * RB + 8 * (lane & 1) +
                          16 * ((F8 ? d : 2 * d + ((lane & 3) >> 1)) ^ VSw::of(v_row)));
    const auto stage = [&](auto which) __attribute__((always_inline)) -> uint8_t * {
        constexpr int st = decltype(which)::value;
        if constexpr (st == 0) return st0[0];
        else if constexpr (st == 1) return st1[0];
        else if constexpr (st == 2) return st2[0];
        else return st3[0];
    };
    const GlobalFloats scale_of = lane_pointer(a.k_scales, a.v_scales, lane >= 32);
    float sc[NS];           // this lane's scale of a stage: keys in lanes 0..31, values behind
    bool ok[NS][2];
    const auto issue = [&](auto which, int i) __attribute__((always_inline)) {
        constexpr int st = decltype(which)::value;
        const int j0 = span.base(it.u_lo + min(i, steps - 1), kTokenUnit) + 32 * wave;
        const int end = i < steps ? hi : 0;
        Rows16 r[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            r[m] = rows16(a, table, g, j0 + 16 * m, end);
            ok[st][m] = r[m].ok;
        }
        if constexpr (F8) {
            const int64_t at = lane & 16 ? r[1].row : r[0].row;
            const int last = max((lane & 16 ? r[1].end : r[0].end) - 1, 0);
            sc[st] = scale_of[at + min(n, last)];
        }
        uint8_t *at = stage(which);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int j = j0 + 16 * m;
            load_rows16<RB, KSw>(a.k_pages, r[m], low - j, a.sinks - j, at, wave * S::kStage + 16 * m * RB, 16 * m);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int j = j0 + 16 * m;
            load_rows16<RB, VSw>(a.v_pages, r[m], low - j, a.sinks - j, at, wave * S::kStage + (32 + 16 * m) * RB, 16 * m);
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    float mx = -INFINITY, l = 0.f;    // l: of the lane's own positions
    floatx4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = floatx4{0.f, 0.f, 0.f, 0.f};
    const auto step = [&](auto which, int i) __attribute__((always_inline)) {
        constexpr int st = decltype(which)::value;
        constexpr int ahead = (st + NS - 1) % NS;
        issue(Int<ahead>{}, i + NS - 1);
        wait_loads<S::kLoads *(NS - 1)>();
        const int j0 = span.base(it.u_lo + i, kTokenUnit) + 32 * wave;
        const uint8_t *lds = stage(which);
        float ks[8], vs[8];
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
        float s[8];
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
            for (int e = 0; e < 4; ++e) {
                s[4 * m + e] = F32 ? big[e] + small[e] : big[e];
                if constexpr (F8) s[4 * m + e] *= ks[4 * m + e];
            }
        }
        const bool whole = j0 + 31 < hi && (j0 >= low || j0 + 31 < a.sinks) && ok[st][0] && ok[st][1];
        if (!whole) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + 16 * m + 4 * lg + e;
                    const bool on = j < hi && (j >= low || j < a.sinks) && ok[st][m];
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
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, -ref));
            l += w[e];
            if constexpr (F8) w[e] *= vs[e];
        }
        const Pieces<F32> pf = pieces_of<F32>(w);
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
            for (int q = NP - 1; q >= 0; --q) o[d] = mfma16(v, pf.p[q], o[d]);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    if (steps > 0) {
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
    // the wavefronts' shares joined in LDS, over the first stage
    wait_loads<0>();
    __syncthreads();
    float(*red)[kTokenRows][HD] = reinterpret_cast<float(*)[kTokenRows][HD]>(&st0[0][0]);
    l = sum_xor32(sum_xor16(l));
    if (lg == 0) {
        red_m[wave][n] = mx;
        red_l[wave][n] = l;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
        *reinterpret_cast<floatx4 *>(&red[wave][n][16 * d + 4 * lg]) = o[d];
    __syncthreads();
    for (int idx = threadIdx.x; idx < a.GR * HD; idx += kThreads) {
        const int h = idx / HD, dim = idx % HD;
        float m = red_m[0][h];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, red_m[w][h]);
        float den = 0.f, num = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float c = red_m[w][h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(red_m[w][h] - m);
            den = fmaf(red_l[w][h], c, den);
            num = fmaf(red[w][h][dim], c, num);
        }
        if (it.part < 0) {
            store_out<F32>(a.out, row * a.out_stride + (g * a.GR + h) * HD + dim, den == 0.f ? 0.f : num / den);
        } else {
            const size_t at = (size_t(it.part) * a.G + g) * kTokenRows + h;
            a.part_o[at * HD + dim] = num;
            if (dim == 0) a.part_ml[at] = make_float2(m, den);
        }
    }
}

// ---------------------------------------------------------------------- tiles of many rows
// A tile is up to 128 rows: 128 / GR consecutive tokens of a request with the GR query heads of a
// group, row = token * GR + head.  Each of four wavefronts owns 32 rows, columns of the 32x32x16
// products; units of 64 positions are staged in LDS for all four, the next one in flight while
// one is multiplied (one barrier per unit).  Lane (q = lane % 32, h = lane / 32) holds the
// scores of row q at positions 32 m + 8 (i / 4) + 4 h + i % 4.
constexpr int kTileUnit = 64;
constexpr int kTileRows = 128;
constexpr int kTileTarget = 512;     // items, all heads

template <int HD, bool F8, bool F32>
__global__ __launch_bounds__(kThreads, F32 ? 1 : 2) void attend_tile(AttendArgs a) {
    constexpr int RB = HD * (F8 ? 1 : 2), KS = HD / 16, DT = HD / 32, NP = Pieces<F32>::N;
    using KSw = KSwizzle<RB>;
    using VSw = TileVSwizzle<RB, F8>;
    __shared__ __align__(1024) uint8_t st0[2 * kTileUnit * RB], st1[2 * kTileUnit * RB];   // keys, values
    __shared__ __align__(16) float scales[2][2][kTileUnit];
    __shared__ __align__(16) int group_ok[2][4];
    __shared__ int wave_odd[kWaves];
    const int item = uniform(blockIdx.x / a.G), g = blockIdx.x - item * a.G;
    if (item >= scalar_load(&a.head->n_items, 0)) return;
    const Item it = scalar_item(a.items, item);
    const Request rq = scalar_request(a.cu_new, a.seq_len, it.r, a.T, a.room);
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int n = lane & 31, h = lane >> 5;
    const int q1 = min(it.q0 + a.tile_tokens, rq.n), tokens = q1 - it.q0;
    const int p_first = uniform(rq.seq - rq.n + it.q0), p_last = p_first + tokens - 1, hi = p_last + 1;
    const int low = a.window > 0 ? max(0, p_first - a.window + 1) : 0;
    const Span span = span_of<kTileUnit>(max(p_first, 0), p_last, a.window, a.sinks);
    const int32_t *table = a.block_table + size_t(it.r) * a.max_blocks;
    const int steps = it.u_hi - it.u_lo;
    const int m_row = 32 * wave + n, tok = m_row / a.GR, head = m_row - tok * a.GR;
    const bool row_on = tok < tokens;
    const bool wave_on = 32 * wave < tokens * a.GR;
    const int p = row_on ? p_first + tok : -1;
    const int64_t row = rq.row0 + it.q0 + (row_on ? tok : 0);
    const int col = (g * a.GR + (row_on ? head : 0)) * HD;

    Pieces<F32> qf[KS];
#pragma unroll
    for (int u = 0; u < KS; ++u)
        qf[u] = load_q<F32>(a.q, row * a.q_stride + col + 16 * u + 8 * h, row_on);

    // where this lane reads, in a stage: keys of row n (and n + 32), values of row v_row and (bf16)
    // v_row + 8, of 16 rows at a time; the swizzles are the same 8 (bf16), 16 and 32 rows further
    int k_at[KS], v_at[DT];
    constexpr int kV = kTileUnit * RB;   // the values' place
    const int kv = (lane & 15) >> 1, half = (lane >> 4) & 1;
    const int v_row = F8 ? 4 * h + (kv < 4 ? kv : kv + 4) : 4 * h + ((lane & 15) >> 2);
#pragma unroll
    for (int u = 0; u < KS; ++u)
        k_at[u] = settled(n * RB + (F8 ? 16 * (u ^ KSw::of(n)) + 8 * h : 16 * ((2 * u + h) ^ KSw::of(n))));
#pragma unroll
    for (int d = 0; d < DT; ++d)
        v_at[d] = settled(kV + v_row * RB + 8 * (lane & 1) +
                          16 * ((F8 ? 2 * d + half : 4 * d + 2 * half + ((lane & 3) >> 1)) ^ VSw::of(v_row)));
    const GlobalFloats scale_of = lane_pointer(a.k_scales, a.v_scales, lane & 16);
    float sc = 0.f;
    bool rows_ok = false;
    // this wavefront's 16 rows of unit i
    const auto issue = [&](auto which, int i) __attribute__((always_inline)) {
        uint8_t *lds = decltype(which)::value ? st1 : st0;
        const int at = 16 * wave * RB;
        const int j = span.base(it.u_lo + min(i, steps - 1), kTileUnit) + 16 * wave;
        const Rows16 r = rows16(a, table, g, j, i < steps ? hi : 0);
        rows_ok = r.ok;
        if constexpr (F8)
            sc = scale_of[r.row + min(lane & 15, max(r.end - 1, 0))];
        load_rows16<RB, KSw>(a.k_pages, r, low - j, a.sinks - j, lds, at, 16 * wave);
        load_rows16<RB, VSw>(a.v_pages, r, low - j, a.sinks - j, lds, kV + at, 16 * wave);
        __builtin_amdgcn_sched_barrier(0);
    };

    float mx, l;    // l: of the lane's own positions
    floatx16 o[DT];

    // CAREFUL: see below
    bool met_odd = false;
    const auto step = [&](auto which, auto careful, int i) __attribute__((always_inline)) {
        constexpr int buf = decltype(which)::value;
        constexpr bool CAREFUL = decltype(careful)::value;
        wait_loads<0>();
        if constexpr (F8)
            if (lane < 32) scales[buf][lane >> 4][16 * wave + (lane & 15)] = sc;
        if (lane == 0) group_ok[buf][wave] = rows_ok;
        lds_barrier();
        issue(Int<1 - buf>{}, i + 1);
        if (!wave_on) return;
        const int j0 = span.base(it.u_lo + i, kTileUnit);
        const uint8_t *lds = buf ? st1 : st0;
        const int4 gok = *reinterpret_cast<const int4 *>(group_ok[buf]);
        const int oks = uniform((gok.x & 1) | (gok.y & 1) << 1 | (gok.z & 1) << 2 | (gok.w & 1) << 3);
        float s[2][16];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            floatx16 big, small;
#pragma unroll
            for (int e = 0; e < 16; ++e) big[e] = small[e] = 0.f;
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                uint4 k;
                if constexpr (F8)
                    k = widen_e4m3(lds_u2(lds, k_at[u] + 32 * m * RB));
                else
                    k = lds_u4(lds, k_at[u] + 32 * m * RB);
#pragma unroll
                for (int q = NP - 1; q > 0; --q) small = mfma32(k, qf[u].p[q], small);
                big = mfma32(k, qf[u].p[0], big);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[m][e] = F32 ? big[e] + small[e] : big[e];
                if constexpr (F8) s[m][e] *= scales[buf][0][32 * m + 8 * (e / 4) + 4 * h + e % 4];
            }
        }
        const bool whole = j0 + kTileUnit - 1 <= p_first && oks == 15 &&
                           (a.window == 0 || j0 > p_last - a.window || j0 + kTileUnit - 1 < a.sinks);
        if (!whole) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int jj = 32 * m + 8 * (e / 4) + 4 * h + e % 4;
                    const bool on = visible(j0 + jj, p, a.window, a.sinks) && (oks >> (jj / 16) & 1);
                    s[m][e] = on ? s[m][e] : -INFINITY;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[m][e]);
        top = max_xor32(top) * a.scale_log2;
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
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float w = __builtin_amdgcn_exp2f(fmaf(s[m][e], a.scale_log2, -ref));
                l += w;
                if constexpr (F8)   // a scale that the row does not see may be anything
                    s[m][e] = w == 0.f ? 0.f : w * scales[buf][1][32 * m + 8 * (e / 4) + 4 * h + e % 4];
                else
                    s[m][e] = w;
            }
        // Where rows see different positions, a value that is no finite number must not meet the
        // zero weights of the rows that do not see it.  A tile that meets such a unit is worked
        // on again, carefully: that unit's products then go one by one.  (Done at once, in this
        // loop, the compiler moves all of o between registers three times a unit.)
        bool odd = false;
        if (!whole) {
#pragma unroll 1
            for (int c = lane; c < kTileUnit * RB / 16; c += kWave) {
                const uint4 v = lds_u4(lds, kV + 16 * c);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if constexpr (F8) {
                        const uint32_t y = (w[x] & 0x7f7f7f7fu) ^ 0x7f7f7f7fu;   // 0: a NaN code
                        odd = odd || ((y - 0x01010101u) & ~y & 0x80808080u);
                    } else {
                        odd = odd || (w[x] & 0x7f80u) == 0x7f80u || (w[x] & 0x7f800000u) == 0x7f800000u;
                    }
                }
            }
            odd = __ballot(odd) != 0;
            met_odd = met_odd || odd;
        }
        if (CAREFUL && odd) {
#pragma unroll 1
            for (int j = 0; j < kTileUnit; ++j) {
                float w = 0.f;
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (32 * m + 8 * (e / 4) + e % 4 == (j & ~4)) w = s[m][e];
                const float other = __shfl_xor(w, 32);
                w = ((j >> 2) & 1) == h ? w : other;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e4 = 0; e4 < 4; ++e4) {
                        float v[4];
                        if constexpr (F8) {
                            const uint32_t c = *reinterpret_cast<const uint32_t *>(
                                lds + (kV + j * RB + 16 * ((2 * d + e4 / 2) ^ VSw::of(j)) + 8 * (e4 & 1) + 4 * h));
                            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(c), false);
                            const auto up = __builtin_amdgcn_cvt_pk_f32_fp8(int(c), true);
                            v[0] = lo[0], v[1] = lo[1], v[2] = up[0], v[3] = up[1];
                        } else {
                            const uint2 c = lds_u2(lds, kV + j * RB + 16 * ((4 * d + e4) ^ VSw::of(j)) + 8 * h);
                            v[0] = apex::ffn::bf_lo(c.x), v[1] = apex::ffn::bf_hi(c.x);
                            v[2] = apex::ffn::bf_lo(c.y), v[3] = apex::ffn::bf_hi(c.y);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[d][4 * e4 + e] = w == 0.f ? o[d][4 * e4 + e] : fmaf(w, v[e], o[d][4 * e4 + e]);
                    }
            }
            return;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = s[u / 2][8 * (u & 1) + e];
            const Pieces<F32> pf = pieces_of<F32>(w);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                uint4 v;
                if constexpr (F8) {
                    v = widen_e4m3(lds_tr8(lds, v_at[d] + 16 * u * RB));
                } else {
                    const uint2 v0 = lds_tr16(lds, v_at[d] + 16 * u * RB);
                    const uint2 v1 = lds_tr16(lds, v_at[d] + (16 * u + 8) * RB);
                    v = make_uint4(v0.x, v0.y, v1.x, v1.y);
                }
#pragma unroll
                for (int q = NP - 1; q >= 0; --q) o[d] = mfma32(v, pf.p[q], o[d]);
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
    const auto all_units = [&](auto careful) __attribute__((always_inline)) {
        clear();
        if (steps > 0) issue(Int<0>{}, 0);
        for (int i = 0; i < steps; i += 2) {
            step(Int<0>{}, careful, i);
            if (i + 1 < steps) step(Int<1>{}, careful, i + 1);
        }
    };
    all_units(Int<0>{});
    if (lane == 0) wave_odd[wave] = met_odd;
    wait_loads<0>();
    __syncthreads();
    if (wave_odd[0] | wave_odd[1] | wave_odd[2] | wave_odd[3]) all_units(Int<1>{});
    wait_loads<0>();
    if (!row_on) return;
    l = sum_xor32(l);
    if (it.part < 0) {
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
        const size_t at = (size_t(it.part) * a.G + g) * kTileRows + m_row;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                *reinterpret_cast<float4 *>(a.part_o + at * HD + 32 * d + 8 * e4 + 4 * h) =
                    make_float4(o[d][4 * e4], o[d][4 * e4 + 1], o[d][4 * e4 + 2], o[d][4 * e4 + 3]);
        if (h == 0) a.part_ml[at] = make_float2(mx, l);
    }
}

// --------------------------------------------------------------------------------- merge
// One wavefront per row of a split tile, HD / 64 dimensions per lane.
constexpr int kMergeBlocks = 512;

template <int HD, bool F32>
__global__ __launch_bounds__(kThreads) void merge_parts(AttendArgs a, int rows) {
    constexpr int PER = HD / kWave;
    const int lane = threadIdx.x % kWave;
    const int per_tile = a.tile_tokens * a.GR * a.G;
    const int64_t total = int64_t(a.head->n_split) * per_tile;
    for (int64_t e = int64_t(blockIdx.x) * kWaves + threadIdx.x / kWave; e < total;
         e += int64_t(gridDim.x) * kWaves) {
        const int tile = uniform(int(e / per_tile)), rest = uniform(int(e - int64_t(tile) * per_tile));
        const int m = rest / a.G, g = rest - m * a.G, tok = m / a.GR, head = m - tok * a.GR;
        const SplitTile sp = a.split[tile];
        const Request rq = request_of(a.cu_new, a.seq_len, sp.r, a.T, a.room);
        if (sp.q0 + tok >= rq.n) continue;
        const size_t step = size_t(a.G) * rows;
        const size_t at = (size_t(sp.part) * a.G + g) * rows + m;
        float top = -INFINITY;
        for (int s = lane; s < sp.n; s += kWave) top = fmaxf(top, a.part_ml[at + s * step].x);
#pragma unroll
        for (int d = kWave / 2; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
        float den = 0.f, num[PER];
#pragma unroll
        for (int x = 0; x < PER; ++x) num[x] = 0.f;
#pragma unroll 4
        for (int s = 0; s < sp.n; ++s) {
            const float2 ml = a.part_ml[at + s * step];
            const float c = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
            const float *o = a.part_o + (at + s * step) * HD + lane * PER;
            den = fmaf(ml.y, c, den);
#pragma unroll
            for (int x = 0; x < PER; ++x) num[x] = fmaf(o[x], c, num[x]);
        }
        const int64_t out = (int64_t(rq.row0) + sp.q0 + tok) * a.out_stride + (g * a.GR + head) * HD + lane * PER;
#pragma unroll
        for (int x = 0; x < PER; ++x) store_out<F32>(a.out, out + x, den == 0.f ? 0.f : num[x] / den);
    }
}

// ---------------------------------------------------------------------------------- host
// Which kernel a call takes and what its workspace holds.
struct Plan {
    bool token;
    int GR, tile_tokens, max_tiles, target, rows;
    int max_split, max_parts, max_items;     // per key/value head
    size_t at_items, at_split, at_ml, at_o, bytes;
};
Plan plan_of(int T, int R, int H, int G, int hd) {
    Plan p;
    p.GR = H / G;
    // no more rows than requests: single tokens, as a rule; a request that has more of them
    // is worked on token by token
    p.token = T <= R;
    p.tile_tokens = p.token ? 1 : kTileRows / p.GR;
    p.rows = p.token ? kTokenRows : kTileRows;
    p.target = p.token ? kTokenTarget : kTileTarget;
    p.max_tiles = T / p.tile_tokens + std::min(T, R);
    // s units an item, s >= U G / target: fewer than target / G tiles have more than s of them,
    // and their items are fewer than their units / s, target / G at most, and one for each
    const int per_head = p.target / G + 1;
    p.max_split = per_head;
    p.max_parts = 2 * per_head;
    p.max_items = p.max_tiles + per_head;
    const auto up = [](size_t v) { return apex::align_up(v, 256); };
    p.at_items = 256;
    p.at_split = p.at_items + up(size_t(p.max_items) * sizeof(Item));
    p.at_ml = p.at_split + up(size_t(p.max_split) * sizeof(SplitTile));
    const size_t parts = size_t(p.max_parts) * G * p.rows;
    p.at_o = p.at_ml + up(parts * sizeof(float2));
    p.bytes = p.at_o + up(parts * hd * sizeof(float));
    return p;
}

template <int HD, bool F32>
void launch_attention(const Plan &p, bool f8, int G, hipStream_t st, const AttendArgs &a) {
    const dim3 grid(unsigned(p.max_items) * unsigned(G));
    const auto f = p.token ? (f8 ? attend_token<HD, true, F32> : attend_token<HD, false, F32>)
                           : (f8 ? attend_tile<HD, true, F32> : attend_tile<HD, false, F32>);
    hipLaunchKernelGGL(f, grid, dim3(kThreads), 0, st, a);
    hipLaunchKernelGGL((merge_parts<HD, F32>), dim3(kMergeBlocks), dim3(kThreads), 0, st, a, p.rows);
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
    APEX_REQUIRE(scale > 0.f && scale < INFINITY, "%s: scale=%g must be positive and finite", fn,
                 double(scale));
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
    if (int64_t(p.max_items) * G > (int64_t(1) << 31) - 1)
        return apex::fail(APEX_E_UNSUPPORTED, "%s: T=%d rows of %d heads are too many", fn, T, H);
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
    a.cu_new = cu_new;
    a.seq_len = seq_len;
    a.block_table = block_table;
    a.T = T;
    a.H = H;
    a.G = G;
    a.GR = p.GR;
    a.tile_tokens = p.tile_tokens;
    a.max_blocks = max_blocks;
    a.shift = apex::log2_of(page_size);
    a.page_size = page_size;
    a.n_pages = cache->n_pages;
    a.room = max_blocks * page_size;
    a.window = window;
    a.sinks = sinks;
    a.scale_log2 = scale * kLog2e;
    a.head = reinterpret_cast<const Header *>(ws);
    a.items = reinterpret_cast<const Item *>(ws + p.at_items);
    a.split = reinterpret_cast<const SplitTile *>(ws + p.at_split);
    a.part_ml = reinterpret_cast<float2 *>(ws + p.at_ml);
    a.part_o = reinterpret_cast<float *>(ws + p.at_o);
    const ScheduleArgs sa{cu_new, seq_len, R, T, a.room, p.tile_tokens, p.max_tiles, window, sinks,
                          p.target, G, p.max_items, p.max_split,
                          reinterpret_cast<Header *>(ws), reinterpret_cast<Item *>(ws + p.at_items),
                          reinterpret_cast<SplitTile *>(ws + p.at_split)};
    if (p.token)
        hipLaunchKernelGGL(schedule<kTokenUnit>, dim3(1), dim3(kSchedThreads), 0, stream, sa);
    else
        hipLaunchKernelGGL(schedule<kTileUnit>, dim3(1), dim3(kSchedThreads), 0, stream, sa);
    APEX_HIP(hipGetLastError());
    const bool f32 = dtype == APEX_TYPE_FP32, f8 = cache->format == APEX_KV_FP8_E4M3;
    if (hd == 64)
        f32 ? launch_attention<64, true>(p, f8, G, stream, a) : launch_attention<64, false>(p, f8, G, stream, a);
    else
        f32 ? launch_attention<128, true>(p, f8, G, stream, a) : launch_attention<128, false>(p, f8, G, stream, a);
    APEX_HIP(hipGetLastError());
    return APEX_OK;
}
