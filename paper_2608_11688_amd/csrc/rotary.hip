// Rotary positions (apex_rotary) and the store of turned keys, with their values, into the paged cache
// (apex_paged_store_rotary).
//
// A workgroup takes a token.  Its threads first fill a table in LDS with the cosines and sines of
// the token's angles, one angle each, in 64 bits and rounded once.  Then lane l of a head's hd / 8
// holds 8 values: four pairs of the table where l < dim / 8, else 8 values that stay as they are.
// Every head of a token uses the same table, so an angle costs its share of H + G heads; what remains
// is one read and one write of every value, 4.8 to 5.2 TB/s of both from memory: 8192 rows of 32
// heads of 64 in fp32 or of 128 in bf16, 134 MB, 27.5 us; 8192 of 32 + 2 x 8 heads of 128 in fp32
// with E4M3 pages, 353 MB, 67.5, in bf16 with bf16 pages, 201 MB, 39.  Two and four tokens a
// workgroup, their tables side by side, took 29.8 and 32.2 for the 27.5, 71 and 74 for the 67.5 and
// 47 and 46 for the 39.  With few heads, whose lanes leave most of a workgroup idle, they would
// be faster: 8192 bf16 rows of 3 heads of 64 7.1 us, 5.6 and 4.8; stored, of 4 + 2 x 1 heads of 128 9.8,
// 9.5 and 8.8.  Loads and stores past the caches take 27.1 where rows come from memory, but 26.3
// instead of 20.7 where a projection has just written them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "common.h"
#include "ffn_device.h"
#include "paged_internal.h"
#include "paged_store.h"

namespace {

using apex::ffn::bf_hi;
using apex::ffn::bf_lo;
using apex::paged::e4m3_row;
using apex::paged::pack_bf16;

constexpr int kThreads = 256;
constexpr int kMaxHd = 1024;

struct Turn {
    const double *freq;
    const int32_t *positions;
    float amplitude;
    int dim, T;
};

// cos and sin (times the amplitude) of the angles of position p, dim / 2 of them.  An angle is turns = p f / (2 pi), as the
// sum of two 64-bit numbers whose rounding errors are carried along, less its nearest quarter: at most an eighth of a
// turn, where the series end with x^11 and x^12 (the next terms are below 2^-36), times the amplitude, and rounded to 32 bits at
// the very end.
__device__ __forceinline__ void fill_table(const Turn &a, int p, float2 *table) {
#pragma clang fp contract(off)      // `turns` is a rounded product: made one with the difference from `whole`, its error counts twice
    constexpr double kHi = 0x1.45f306dc9c883p-3, kLo = -0x1.6b01ec5417056p-57;       // 1 / (2 pi)
    for (int i = threadIdx.x; i < a.dim / 2; i += kThreads) {
        const double f = a.freq[i], angle = p * f, turns = angle * kHi;
        const double low = fma(angle, kLo, fma(fma(double(p), f, -angle), kHi, fma(angle, kHi, -turns)));
        const double whole = rint(turns), quarter = rint(4.0 * (turns - whole));
        const double x = (fma(quarter, -0.25, turns - whole) + low) * 6.28318530717958647693, xx = x * x;
        double s = fma(xx, -1.0 / 39916800, 1.0 / 362880), c = fma(xx, 1.0 / 479001600, -1.0 / 3628800);
        s = fma(xx, s, -1.0 / 5040), c = fma(xx, c, 1.0 / 40320);
        s = fma(xx, s, 1.0 / 120), c = fma(xx, c, -1.0 / 720);
        s = fma(xx, s, -1.0 / 6), c = fma(xx, c, 1.0 / 24);
        s = fma(xx * x, s, x), c = fma(xx, fma(xx, c, -0.5), 1.0);
        const int q = int(quarter);                    // -2 to 2
        const double cq = q & 1 ? s : c, sq = q & 1 ? c : s;       // a quarter on: cos -> -sin, sin -> cos
        const double m = a.amplitude;
        table[i] = make_float2(float((q + 1) & 2 ? -m * cq : m * cq), float(q & 2 ? -m * sq : m * sq));
    }
    __syncthreads();
}

// The two places in a head where lane l's 8 values stand, four each: of the turned part and of the rest both halves
// are in the order of the lanes, so that neighbours' 16 (or 8) bytes are side by side.
struct Places {
    int first, second;
    bool turned;
};
__device__ __forceinline__ Places places(int l, int dim, int hd) {
    const bool turned = l < dim / 8;
    const int base = turned ? 0 : dim, half = (turned ? dim : hd - dim) / 2, at = base + 4 * (turned ? l : l - dim / 8);
    return {at, at + half, turned};
}

// Four values as they stand in memory.
template <bool F32>
struct Four {
    using Raw = uint2;
};
template <>
struct Four<true> {
    using Raw = float4;
};
template <bool F32>
__device__ __forceinline__ typename Four<F32>::Raw &four(void *row, int at) {
    return *reinterpret_cast<typename Four<F32>::Raw *>(static_cast<char *>(row) + at * (F32 ? 4 : 2));
}
__device__ __forceinline__ void widen(float4 v, float *x) { x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w; }
__device__ __forceinline__ void widen(uint2 v, float *x) {
    x[0] = bf_lo(v.x), x[1] = bf_hi(v.x), x[2] = bf_lo(v.y), x[3] = bf_hi(v.y);
}
template <bool F32>
__device__ __forceinline__ typename Four<F32>::Raw narrow(const float *x) {
    if constexpr (F32)
        return make_float4(x[0], x[1], x[2], x[3]);
    else
        return make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
}

// Lane l's four pairs: x[i] with x[4 + i], or neighbours.
template <bool INTER>
__device__ __forceinline__ void turn(float (&x)[8], const float2 *table, int l, int dim) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 cs = table[INTER ? (i < 2 ? 2 * l + i : dim / 4 + 2 * l + i - 2) : 4 * l + i];
        float &a = x[INTER ? 2 * i : i], &b = x[INTER ? 2 * i + 1 : 4 + i];
        const float u = a, v = b;
        a = fmaf(u, cs.x, -(v * cs.y));
        b = fmaf(u, cs.y, v * cs.x);
    }
}

struct RotaryArgs {
    Turn turn;
    void *x, *out;       // x is read only
    int64_t x_stride, out_stride;
    int heads, hd;
};

template <bool F32, bool INTER>
__global__ __launch_bounds__(kThreads) void rotary(RotaryArgs a) {
    __shared__ float2 table[kMaxHd / 2];
    constexpr int size = F32 ? 4 : 2;
    const int64_t t = blockIdx.x;
    const int p = a.turn.positions[t];
    if (p < 0) return;
    fill_table(a.turn, p, table);
    const int lanes = a.hd / 8, rows = kThreads / lanes;      // of a head; heads at a time
    const int l = threadIdx.x % lanes, first = threadIdx.x / lanes;
    if (first >= rows) return;
    const Places at = places(l, a.turn.dim, a.hd);
    for (int h = blockIdx.y * rows + first; h < a.heads; h += rows * gridDim.y) {
        char *src = static_cast<char *>(a.x) + (t * a.x_stride + int64_t(h) * a.hd) * size;
        char *dst = static_cast<char *>(a.out) + (t * a.out_stride + int64_t(h) * a.hd) * size;
        auto u = four<F32>(src, at.first), v = four<F32>(src, at.second);
        if (at.turned) {
            float x[8];
            widen(u, x);
            widen(v, x + 4);
            turn<INTER>(x, table, l, a.turn.dim);
            u = narrow<F32>(x);
            v = narrow<F32>(x + 4);
        }
        four<F32>(dst, at.first) = u;
        four<F32>(dst, at.second) = v;
    }
}

struct StoreArgs {
    Turn turn;
    void *q, *k, *v;     // read only
    void *q_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    const int32_t *slot_map;
    void *k_pages, *v_pages;
    float *k_scales, *v_scales;
    int H, G, page_size, shift, n_slots;
};

template <int HD, bool F32, bool F8, bool INTER>
__global__ __launch_bounds__(kThreads) void store_rotary(StoreArgs a) {
    __shared__ float2 table[HD / 2];
    constexpr int size = F32 ? 4 : 2, lanes = HD / 8, rows = kThreads / lanes;
    const int64_t t = blockIdx.x;
    const int p = a.turn.positions[t], slot = a.slot_map[t];
    if (p < 0) return;
    fill_table(a.turn, p, table);
    const bool stored = slot >= 0 && slot < a.n_slots;
    const int l = threadIdx.x % lanes, first = threadIdx.x / lanes;
    const Places at = places(l, a.turn.dim, HD);
    for (int h = blockIdx.y * rows + first; h < a.H + 2 * a.G; h += rows * gridDim.y) {
        const bool is_q = h < a.H, is_v = h >= a.H + a.G;
        if (!is_q && !stored) continue;          // a head's lanes take the same way
        const int g = is_q ? h : is_v ? h - a.H - a.G : h - a.H;
        const int64_t stride = is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride;
        char *src = static_cast<char *>(is_q ? a.q : is_v ? a.v : a.k) + (t * stride + int64_t(g) * HD) * size;
        auto u = four<F32>(src, at.first), v = four<F32>(src, at.second);
        float x[8];
        widen(u, x);
        widen(v, x + 4);
        if (at.turned && !is_v) {
            turn<INTER>(x, table, l, a.turn.dim);
            u = narrow<F32>(x);
            v = narrow<F32>(x + 4);
        }
        if (is_q) {
            char *dst = static_cast<char *>(a.q_out) + (t * a.q_out_stride + int64_t(g) * HD) * size;
            four<F32>(dst, at.first) = u;
            four<F32>(dst, at.second) = v;
            continue;
        }
        const size_t row = (size_t(slot >> a.shift) * a.G + g) * a.page_size + (slot & (a.page_size - 1));
        char *dst = static_cast<char *>(is_v ? a.v_pages : a.k_pages) + row * HD * (F8 ? 1 : 2);
        if constexpr (F8) {
            uint32_t code[2];
            const float s = e4m3_row<lanes>(x, code);
            *reinterpret_cast<uint32_t *>(dst + at.first) = code[0];
            *reinterpret_cast<uint32_t *>(dst + at.second) = code[1];
            if (l == 0) (is_v ? a.v_scales : a.k_scales)[row] = s;
        } else if constexpr (F32) {
            four<false>(dst, at.first) = narrow<false>(x);
            four<false>(dst, at.second) = narrow<false>(x + 4);
        } else {
            four<false>(dst, at.first) = u;
            four<false>(dst, at.second) = v;
        }
    }
}

apex_status check_rotation(const char *fn, const apex_rotation *r, int hd, bool pointers) {
    APEX_REQUIRE(r, "%s: NULL rotation", fn);
    APEX_REQUIRE(r->layout == APEX_ROPE_HALF || r->layout == APEX_ROPE_INTERLEAVED, "%s: unknown layout %d", fn,
                 r->layout);
    APEX_REQUIRE(r->dim >= 16 && r->dim % 16 == 0 && r->dim <= hd,
                 "%s: dim=%d must be a multiple of 16 and at most the head size %d", fn, r->dim, hd);
    APEX_REQUIRE(std::isfinite(r->amplitude), "%s: the amplitude must be finite", fn);
    APEX_REQUIRE(!pointers || (r->freq && apex::aligned16(r->freq)), "%s: NULL or misaligned frequencies", fn);
    return APEX_OK;
}

// A workgroup a token; of few tokens the heads over several, up to 512 workgroups in all: 32 rows of 40 heads of 128 take
// 2.9 us with any number from 256 to 4096, 3.4 with a workgroup a token.
dim3 grid_of(int T, int heads, int rows) {
    return dim3(unsigned(T), unsigned(std::min((heads + rows - 1) / rows, std::max(1, 512 / T))));
}

template <bool F32, bool INTER>
void launch_rotary(const RotaryArgs &a, hipStream_t st) {
    hipLaunchKernelGGL((rotary<F32, INTER>), grid_of(a.turn.T, a.heads, kThreads / (a.hd / 8)), dim3(kThreads), 0, st, a);
}

template <int HD, bool F32, bool F8, bool INTER>
void launch_store(const StoreArgs &a, hipStream_t st) {
    hipLaunchKernelGGL((store_rotary<HD, F32, F8, INTER>), grid_of(a.turn.T, a.H + 2 * a.G, kThreads / (HD / 8)),
                       dim3(kThreads), 0, st, a);
}

template <int HD>
void launch_store(bool f32, bool f8, bool inter, const StoreArgs &a, hipStream_t st) {
    using F = void (*)(const StoreArgs &, hipStream_t);
    static const F table[8] = {launch_store<HD, false, false, false>, launch_store<HD, false, false, true>,
                               launch_store<HD, false, true, false>, launch_store<HD, false, true, true>,
                               launch_store<HD, true, false, false>, launch_store<HD, true, false, true>,
                               launch_store<HD, true, true, false>, launch_store<HD, true, true, true>};
    table[4 * f32 + 2 * f8 + inter](a, st);
}

apex_status check_tokens(const char *fn, int T) {
    APEX_REQUIRE(T >= 0, "%s: T=%d must be >= 0", fn, T);
    if (T > APEX_MAX_STEP_TOKENS)
        return apex::fail(APEX_E_UNSUPPORTED, "%s: T=%d exceeds %d", fn, T, APEX_MAX_STEP_TOKENS);
    return APEX_OK;
}

bool aligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

}  // namespace

extern "C" apex_status apex_rotary(const apex_rotation *rotation, const void *x, int dtype, int T, int heads,
                                   int hd, int64_t x_stride, const int32_t *positions, void *out,
                                   int64_t out_stride, hipStream_t stream) {
    const char *fn = "apex_rotary";
    apex_status st = check_tokens(fn, T);
    if (st != APEX_OK) return st;
    APEX_REQUIRE(dtype == APEX_TYPE_FP32 || dtype == APEX_TYPE_BF16, "%s: unknown type %d", fn, dtype);
    APEX_REQUIRE(heads >= 1, "%s: heads=%d must be >= 1", fn, heads);
    if (heads > (1 << 20)) return apex::fail(APEX_E_UNSUPPORTED, "%s: heads=%d exceeds 2^20", fn, heads);
    APEX_REQUIRE(hd >= 16 && hd % 8 == 0, "%s: head size %d must be a multiple of 8, 16 or more", fn, hd);
    if (hd > kMaxHd) return apex::fail(APEX_E_UNSUPPORTED, "%s: head size %d exceeds %d", fn, hd, kMaxHd);
    if ((st = check_rotation(fn, rotation, hd, T > 0)) != APEX_OK) return st;
    if ((st = apex::check_rows(fn, "x", dtype, x_stride, int64_t(heads) * hd)) != APEX_OK) return st;
    if ((st = apex::check_rows(fn, "out", dtype, out_stride, int64_t(heads) * hd)) != APEX_OK) return st;
    if (T == 0) return APEX_OK;
    APEX_REQUIRE(x && positions && out, "%s: NULL pointer", fn);
    APEX_REQUIRE(apex::aligned16(x) && apex::aligned16(out) && aligned4(positions), "%s: misaligned pointer", fn);
    APEX_REQUIRE(x != out || x_stride == out_stride, "%s: out is x with another stride", fn);
    const int64_t size = dtype == APEX_TYPE_FP32 ? 4 : 2, row = int64_t(heads) * hd * size;
    APEX_REQUIRE(x == out || !apex::rows_overlap({x, x_stride * size, row}, {out, out_stride * size, row}, T),
                 "%s: rows of out overlap others of x", fn);
    const RotaryArgs a{{rotation->freq, positions, rotation->amplitude, rotation->dim, T}, const_cast<void *>(x),
                       out, x_stride, out_stride, heads, hd};
    const bool inter = rotation->layout == APEX_ROPE_INTERLEAVED;
    if (dtype == APEX_TYPE_FP32)
        inter ? launch_rotary<true, true>(a, stream) : launch_rotary<true, false>(a, stream);
    else
        inter ? launch_rotary<false, true>(a, stream) : launch_rotary<false, false>(a, stream);
    APEX_HIP(hipGetLastError());
    return APEX_OK;
}

extern "C" apex_status apex_paged_store_rotary(const apex_paged_cache *cache, const apex_rotation *rotation,
                                               const void *q, const void *k, const void *v, int dtype, int T,
                                               int H, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                               const int32_t *slot_map, const int32_t *positions, void *q_out,
                                               int64_t q_out_stride, hipStream_t stream) {
    const char *fn = "apex_paged_store_rotary";
    apex_status st = check_tokens(fn, T);
    if (st != APEX_OK) return st;
    if ((st = apex::check_paged_cache(fn, cache, T > 0)) != APEX_OK) return st;
    if ((st = check_rotation(fn, rotation, cache->hd, T > 0)) != APEX_OK) return st;
    APEX_REQUIRE(dtype == APEX_TYPE_FP32 || dtype == APEX_TYPE_BF16, "%s: unknown type %d", fn, dtype);
    const int G = cache->G, hd = cache->hd;
    APEX_REQUIRE(H >= 0, "%s: H=%d must be >= 0", fn, H);
    if (H > (1 << 20)) return apex::fail(APEX_E_UNSUPPORTED, "%s: H=%d exceeds 2^20", fn, H);
    if (H > 0) {
        if ((st = apex::check_rows(fn, "q", dtype, q_stride, int64_t(H) * hd)) != APEX_OK) return st;
        if ((st = apex::check_rows(fn, "q_out", dtype, q_out_stride, int64_t(H) * hd)) != APEX_OK) return st;
    }
    if ((st = apex::check_rows(fn, "k", dtype, k_stride, int64_t(G) * hd)) != APEX_OK) return st;
    if ((st = apex::check_rows(fn, "v", dtype, v_stride, int64_t(G) * hd)) != APEX_OK) return st;
    if (T == 0) return APEX_OK;
    APEX_REQUIRE(k && v && slot_map && positions && (H == 0 || (q && q_out)), "%s: NULL pointer", fn);
    APEX_REQUIRE(apex::aligned16(k) && apex::aligned16(v) && aligned4(slot_map) && aligned4(positions) &&
                     (H == 0 || (apex::aligned16(q) && apex::aligned16(q_out))),
                 "%s: misaligned pointer", fn);
    APEX_REQUIRE(H == 0 || q != q_out || q_stride == q_out_stride, "%s: q_out is q with another stride", fn);
    if (H > 0) {
        const int64_t size = dtype == APEX_TYPE_FP32 ? 4 : 2, q_row = int64_t(H) * hd * size, row = int64_t(G) * hd * size;
        const apex::Rows out{q_out, q_out_stride * size, q_row};
        APEX_REQUIRE(q == q_out || !apex::rows_overlap(out, {q, q_stride * size, q_row}, T),
                     "%s: rows of q_out overlap others of q", fn);
        APEX_REQUIRE(!apex::rows_overlap(out, {k, k_stride * size, row}, T) && !apex::rows_overlap(out, {v, v_stride * size, row}, T),
                     "%s: rows of q_out overlap rows of k or v", fn);
    }
    const StoreArgs a{{rotation->freq, positions, rotation->amplitude, rotation->dim, T}, const_cast<void *>(q),
                      const_cast<void *>(k), const_cast<void *>(v), q_out,
                      q_stride, k_stride, v_stride, q_out_stride, slot_map, cache->k_pages, cache->v_pages,
                      cache->k_scales, cache->v_scales, H, G, cache->page_size, apex::log2_of(cache->page_size),
                      cache->n_pages * cache->page_size};
    const bool f32 = dtype == APEX_TYPE_FP32, f8 = cache->format == APEX_KV_FP8_E4M3;
    const bool inter = rotation->layout == APEX_ROPE_INTERLEAVED;
    if (hd == 64)
        launch_store<64>(f32, f8, inter, a, stream);
    else
        launch_store<128>(f32, f8, inter, a, stream);
    APEX_HIP(hipGetLastError());
    return APEX_OK;
}
