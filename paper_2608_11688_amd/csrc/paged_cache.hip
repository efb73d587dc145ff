// Paged key/value cache: the plan of pages and slots (apex_paged_plan) and the store of new keys
// and values (apex_paged_store).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "common.h"
#include "ffn_device.h"
#include "paged_internal.h"

namespace {

using apex::ffn::kWave;

// ---------------------------------------------------------------------------------- plan
constexpr int kPlanBlocks = 64;   // workgroups at most

struct PlanArgs {
    const int32_t *cached, *n_new;
    int R, page_size, shift, n_pages, max_blocks, T;
    int32_t *free_pages;
    const int32_t *free_count;
    int32_t *block_table, *seq_len, *cu_new, *slot_map, *positions, *free_count_out, *status;
};

// Sums that stand still at 2^32 - 1: lengths are any 32-bit numbers, and what is compared with
// such a sum (pages, rows) is smaller.
__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }

struct Sums {
    uint32_t given, need, want;   // pages given back, pages wanted, tokens wanted
    __device__ __forceinline__ void add(const Sums &o) {
        given = add_sat(given, o.given);
        need = add_sat(need, o.need);
        want = add_sat(want, o.want);
    }
};

template <int CTRL>
__device__ __forceinline__ uint32_t lane_back(uint32_t v) {   // 0 before the row's first lane
    return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x, int lane) {   // inclusive
    x = add_sat(x, lane_back<0x111>(x));   // row_shr 1, 2, 4, 8
    x = add_sat(x, lane_back<0x112>(x));
    x = add_sat(x, lane_back<0x114>(x));
    x = add_sat(x, lane_back<0x118>(x));
    const uint32_t a = __builtin_amdgcn_readlane(x, 15);
    const uint32_t b = add_sat(a, __builtin_amdgcn_readlane(x, 31));
    const uint32_t c = add_sat(b, __builtin_amdgcn_readlane(x, 47));
    return add_sat(x, lane < 16 ? 0u : lane < 32 ? a : lane < 48 ? b : c);
}

__device__ __forceinline__ int wave_scan_max(int x, int lane) {   // of values >= 0; the last lane's is all's
    x = max(x, int(lane_back<0x111>(uint32_t(x))));
    x = max(x, int(lane_back<0x112>(uint32_t(x))));
    x = max(x, int(lane_back<0x114>(uint32_t(x))));
    x = max(x, int(lane_back<0x118>(uint32_t(x))));
    const int a = __builtin_amdgcn_readlane(x, 15), b = max(a, __builtin_amdgcn_readlane(x, 31));
    const int c = max(b, __builtin_amdgcn_readlane(x, 47));
    return max(x, lane < 16 ? 0 : lane < 32 ? a : lane < 48 ? b : c);
}

// The last r in [0, R) with cu[r] <= k, for cu[0] = 0 <= k < cu[R]: the request of entry k.
__device__ __forceinline__ int owner(const int32_t *cu, int R, int k) {
    int lo = 0, hi = R;   // cu[lo] <= k < cu[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= k)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int clamped(uint32_t v) { return int(min(v, uint32_t(INT_MAX))); }

// One launch: every workgroup takes the sums over all requests for itself, keeps them in LDS and
// then writes its share of the outputs, finding the request of a slot, a taken page or a returned
// page by bisection.  Pages taken in this step may be ones given back in it: entry k of the
// returned pages is read from its owner's table row, which nobody writes, not from the stack.
// A chain of round trips (lengths, sums, bisection, table) and the fetch of its instructions, not
// bytes, are what bounds it.  N threads: 256 up to as many requests, where a thread has one,
// else 1024.  32 requests 3.5 us, 1024 requests with 17000 tokens 8.3.
template <int N>
__global__ __launch_bounds__(N) void paged_plan(PlanArgs a) {
    constexpr int WAVES = N / kWave, R_MAX = N == 256 ? 256 : APEX_MAX_REQUESTS;
    __shared__ int32_t cu_given[R_MAX + 1], cu_need[R_MAX + 1], cu_tok[R_MAX + 1];
    __shared__ Sums wave_sums[WAVES];
    __shared__ int32_t wave_need[WAVES], wave_tok[WAVES];
    const int t = threadIdx.x, wave = t / kWave, lane = t % kWave;
    const int per = (a.R + N - 1) / N, r0 = min(t * per, a.R), r1 = min(r0 + per, a.R);
    const int fc = min(max(a.free_count[0], 0), a.n_pages);
    const uint32_t room = uint32_t(a.max_blocks) << a.shift;   // < 2^31
    const auto blocks = [&](uint32_t n) { return (n + a.page_size - 1) >> a.shift; };
    struct Request {
        int cached, state;
        Sums sums;
    };
    const auto request = [&](int r) {
        const int c = a.cached[r], n = a.n_new[r];
        Request q{c, APEX_REQ_SERVED, {0u, 0u, 0u}};
        if (c < 0 || n < -1 || uint32_t(c) + uint32_t(max(n, 0)) > room) {
            q.state = APEX_REQ_INVALID;
        } else if (n == -1) {
            q.state = APEX_REQ_ENDED;
            q.sums.given = blocks(c);
        } else if (n > 0) {
            q.sums.want = n;
            q.sums.need = blocks(c + n) - blocks(c);
        }
        return q;
    };
    Sums sum = {0u, 0u, 0u};
    Request mine;   // of a thread that has one
#pragma unroll 1
    for (int r = r0; r < r1; ++r) {
        mine = request(r);
        sum.add(mine.sums);
    }
    // sums up to this thread's requests
    Sums upto = {wave_scan(sum.given, lane), wave_scan(sum.need, lane), wave_scan(sum.want, lane)};
    if (lane == kWave - 1) wave_sums[wave] = upto;
    __syncthreads();
    Sums at = {0u, 0u, 0u}, all = at;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const Sums o = wave_sums[w];
        if (w < wave) at.add(o);
        all.add(o);
    }
    const Sums before = {lane_back<0x138>(upto.given), lane_back<0x138>(upto.need), lane_back<0x138>(upto.want)};
    at.add(before);   // (wave_shr 1)
    const int top = int(min(uint64_t(fc) + all.given, uint64_t(a.n_pages)));
    // requests are served up to the first that does not fit: from there on the sums stand still
    int last_need = 0, last_tok = 0;
#pragma unroll 1
    for (int r = r0; r < r1; ++r) {
        if (per > 1) mine = request(r);
        at.add(mine.sums);
        const bool fits = at.need <= uint32_t(top) && at.want <= uint32_t(a.T);
        cu_given[r + 1] = clamped(at.given);
        cu_need[r + 1] = fits ? int(at.need) : -1;
        cu_tok[r + 1] = fits ? int(at.want) : -1;
        if (fits) {
            last_need = int(at.need);
            last_tok = int(at.want);
        }
    }
    if (t == 0) cu_given[0] = cu_need[0] = cu_tok[0] = 0;
    // (of sums that fit, the last is the largest)
    last_need = __builtin_amdgcn_readlane(int(wave_scan_max(last_need, lane)), 63);
    last_tok = __builtin_amdgcn_readlane(int(wave_scan_max(last_tok, lane)), 63);
    if (lane == 0) {
        wave_need[wave] = last_need;
        wave_tok[wave] = last_tok;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        last_need = max(last_need, wave_need[w]);
        last_tok = max(last_tok, wave_tok[w]);
    }
#pragma unroll 1
    for (int r = r0; r < r1; ++r)
        if (cu_need[r + 1] < 0) {
            cu_need[r + 1] = last_need;
            cu_tok[r + 1] = last_tok;
        }
    __syncthreads();

    // the page at position k of the returned ones, and the j-th page taken
    const auto returned = [&](int k) {
        const int r = owner(cu_given, a.R, k);
        return a.block_table[size_t(r) * a.max_blocks + (k - cu_given[r])];
    };
    const auto taken = [&](int j) {
        const int pos = top - 1 - j;
        return pos < fc ? a.free_pages[pos] : returned(pos - fc);
    };
    if (blockIdx.x == 0) {
#pragma unroll 1
        for (int r = r0; r < r1; ++r) {
            if (per > 1) mine = request(r);
            const int got = cu_tok[r + 1] - cu_tok[r];
            const int held = int(min(uint32_t(max(mine.cached, 0)), room));
            a.seq_len[r] = mine.state == APEX_REQ_ENDED ? 0 : held + got;
            a.cu_new[r + 1] = cu_tok[r + 1];
            if (a.status)
                a.status[r] = mine.state == APEX_REQ_SERVED && mine.sums.want > 0 && got == 0 ? APEX_REQ_WAITS
                                                                                              : mine.state;
        }
        if (t == 0) {
            a.cu_new[0] = 0;
            a.free_count_out[0] = top - last_need;
        }
    }
    const int first = blockIdx.x * N + t, step = gridDim.x * N;
#pragma unroll 1
    for (unsigned u = first; u < unsigned(a.T); u += step) {   // (T + step may pass 2^31)
        const int s = int(u);
        int slot = -1, p = -1;
        if (s < last_tok) {
            const int r = owner(cu_tok, a.R, s);
            const int c = a.cached[r];
            p = c + (s - cu_tok[r]);
            const int b = p >> a.shift, held = int(blocks(c));
            const int page = b < held ? a.block_table[size_t(r) * a.max_blocks + b]
                                      : taken(cu_need[r] + b - held);
            if (page >= 0 && page < a.n_pages) slot = (page << a.shift) + (p & (a.page_size - 1));
        }
        a.slot_map[s] = slot;
        if (a.positions) a.positions[s] = p;
    }
#pragma unroll 1
    for (int j = first; j < last_need; j += step) {
        const int r = owner(cu_need, a.R, j);
        a.block_table[size_t(r) * a.max_blocks + blocks(a.cached[r]) + (j - cu_need[r])] = taken(j);
    }
#pragma unroll 1
    for (int k = first; k < top - fc; k += step) a.free_pages[fc + k] = returned(k);
}

// --------------------------------------------------------------------------------- store
constexpr int kStoreThreads = 256;

struct StoreArgs {
    const void *src[2];      // k, v
    int64_t stride[2];       // in values
    void *pages[2];
    float *scales[2];
    const int32_t *slot_map;
    int64_t rows;            // T * G
    int G, page_size, shift;
    int n_slots;
};

// 8 consecutive values of a row as fp32.
template <bool F32>
__device__ __forceinline__ void load8(const void *row, int at, float (&x)[8], uint4 &raw) {
    if constexpr (F32) {
        const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(row) + at);
        const float4 a = p[0], b = p[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
        x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        raw = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(row) + at);
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = apex::ffn::bf_lo(w[i]);
            x[2 * i + 1] = apex::ffn::bf_hi(w[i]);
        }
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(lo))) |
           uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(hi))) << 16;
}

// The maximum over the N lanes (8 or 16, aligned) that share a row.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xf, 0xf, false));
}
template <int N>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
    v = max(v, dpp<0xb1>(v));                   // quad_perm 1,0,3,2
    v = max(v, dpp<0x4e>(v));                   // quad_perm 2,3,0,1
    v = max(v, dpp<0x141>(v));                  // row_half_mirror
    if (N == 16) v = max(v, dpp<0x140>(v));     // row_mirror
    return v;
}

// x / s for the conversion to E4M3, near enough to the quotient that the conversion rounds as the
// exact quotient would: x * (1 / s) is off by a few units in the last place, which matters only
// next to a tie (halfway between two codes: of 20 lower bits only the highest set, or an odd
// multiple of 2^-10 below 2^-6).  There the sign of x - tie * s, exact in one fused
// multiply-add, tells the side; a tie stays one.
__device__ __forceinline__ float code_ratio(float x, float s, float inv) {
    const float q = x * inv;
    const float a = fabsf(q);
    float tie;
    if (a >= 0.015625f) {
        const uint32_t u = __float_as_uint(q);
        tie = __uint_as_float((u & 0xfff00000u) | 0x80000u);
    } else {
        tie = copysignf((floorf(a * 512.f) + 0.5f) * (1.f / 512.f), q);
    }
    if (fabsf(q - tie) > a * 0x1p-20f) return q;
    const float d = copysignf(1.f, q) * fmaf(-tie, s, x);   // > 0: beyond the tie
    const int up = d > 0.f ? 1 : d < 0.f ? -1 : 0;
    return __uint_as_float(__float_as_uint(tie) + up);
}

// HD / 8 lanes per row of one token and head, 8 values each; keys and values in turn.
// Bound by memory, each value read and written once: 8192 fp32 rows of 8 heads of 128 into E4M3
// pools (84 MB moved, a fifth of it written) 16.2-17.2 us, 4.9-5.2 TB/s, where a large copy gets 4.9.
// 32 rows of bf16 2.3 us, a launch's time.
template <int HD, bool F32, bool F8>
__global__ __launch_bounds__(kStoreThreads) void paged_store(StoreArgs a) {
    constexpr int LPR = HD / 8;
    const int64_t i = (int64_t(blockIdx.x) * kStoreThreads + threadIdx.x) / LPR;
    const int at = 8 * (threadIdx.x % LPR), kv = blockIdx.y;
    if (i >= a.rows) return;
    const int64_t t = i / a.G;
    const int g = int(i - t * a.G);
    const int slot = a.slot_map[t];
    if (slot < 0 || slot >= a.n_slots) return;
    const size_t row = (size_t(slot >> a.shift) * a.G + g) * a.page_size + (slot & (a.page_size - 1));
    float x[8];
    uint4 raw;
    load8<F32>(static_cast<const char *>(a.src[kv]) +
                   (t * a.stride[kv] + int64_t(g) * HD) * (F32 ? 4 : 2),
               at, x, raw);
    if constexpr (!F8) {
        if constexpr (F32)
            raw = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                             pack_bf16(x[6], x[7]));
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.pages[kv]) + row * HD + at) = raw;
    } else {
        // magnitudes compare as integers, infinity and NaN above every number
        uint32_t peak = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) peak = max(peak, __float_as_uint(x[e]) & 0x7fffffffu);
        peak = lanes_max<LPR>(peak);
        const bool bad = peak >= 0x7f800000u;
        const float s = __uint_as_float(peak) / 448.f;
        uint32_t code[2] = {0u, 0u};
        if (!bad && s > 0.f) {
            // tiny rows: both sides of the quotient scaled alike, away from subnormal numbers
            const float up = s < 0x1p-100f ? 0x1p64f : 1.f, su = s * up, inv = 1.f / su;
            float q[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                q[e] = fminf(fmaxf(code_ratio(x[e] * up, su, inv), -448.f), 448.f);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * w], q[4 * w + 1], 0, false);
                code[w] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * w + 2], q[4 * w + 3], c, true));
            }
        }
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.pages[kv]) + row * HD + at) =
            make_uint2(code[0], code[1]);
        if (at == 0) a.scales[kv][row] = bad ? NAN : s;
    }
}

template <int HD>
void launch_store(bool f32, bool f8, dim3 grid, hipStream_t st, const StoreArgs &a) {
    const auto f = f32 ? (f8 ? paged_store<HD, true, true> : paged_store<HD, true, false>)
                       : (f8 ? paged_store<HD, false, true> : paged_store<HD, false, false>);
    hipLaunchKernelGGL(f, grid, dim3(kStoreThreads), 0, st, a);
}

}  // namespace

extern "C" apex_status apex_paged_plan(const int32_t *cached, const int32_t *n_new, int R,
                                       int page_size, int n_pages, int max_blocks, int T,
                                       int32_t *free_pages, const int32_t *free_count,
                                       int32_t *block_table, int32_t *seq_len, int32_t *cu_new,
                                       int32_t *slot_map, int32_t *positions,
                                       int32_t *free_count_out, int32_t *status,
                                       hipStream_t stream) {
    const char *fn = "apex_paged_plan";
    APEX_REQUIRE(R >= 0, "%s: R=%d must be >= 0", fn, R);
    if (R > APEX_MAX_REQUESTS)
        return apex::fail(APEX_E_UNSUPPORTED, "%s: R=%d exceeds %d", fn, R, APEX_MAX_REQUESTS);
    const apex_status st = apex::check_page_sizes(fn, page_size, n_pages);
    if (st != APEX_OK) return st;
    APEX_REQUIRE(max_blocks >= 1, "%s: max_blocks=%d must be >= 1", fn, max_blocks);
    if (int64_t(max_blocks) * page_size >= (int64_t(1) << 31))
        return apex::fail(APEX_E_UNSUPPORTED, "%s: table rows of %d pages of %d positions: 2^31 or more",
                          fn, max_blocks, page_size);
    APEX_REQUIRE(T >= 0, "%s: T=%d must be >= 0", fn, T);
    APEX_REQUIRE(free_pages && free_count && cu_new && free_count_out, "%s: NULL pointer", fn);
    APEX_REQUIRE(R == 0 || (cached && n_new && block_table && seq_len), "%s: NULL pointer", fn);
    APEX_REQUIRE(T == 0 || slot_map, "%s: NULL slot_map", fn);
    // the inputs first: they may be one buffer, an output may be none of the others
    const void *all[] = {cached, n_new, free_count, free_pages, block_table, seq_len,
                         cu_new, slot_map, positions, free_count_out, status};
    const int n_all = int(sizeof(all) / sizeof(all[0])), n_in = 3;
    for (int i = 0; i < n_all; ++i) {
        APEX_REQUIRE(reinterpret_cast<uintptr_t>(all[i]) % 4 == 0, "%s: misaligned pointer", fn);
        for (int j = 0; i >= n_in && j < i; ++j)
            APEX_REQUIRE(!all[i] || all[i] != all[j], "%s: an output is the buffer of another argument", fn);
    }
    const PlanArgs a{cached, n_new, R, page_size, apex::log2_of(page_size), n_pages, max_blocks, T,
                     free_pages, free_count, block_table, seq_len, cu_new, slot_map, positions,
                     free_count_out, status};
    const int threads = R <= 256 ? 256 : 1024;
    const dim3 grid(std::min(std::max(1, (T - 1) / threads + 1), kPlanBlocks));
    if (threads == 256)
        hipLaunchKernelGGL(paged_plan<256>, grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL(paged_plan<1024>, grid, dim3(1024), 0, stream, a);
    APEX_HIP(hipGetLastError());
    return APEX_OK;
}

extern "C" apex_status apex_paged_store(const apex_paged_cache *cache, const void *k, const void *v,
                                        int dtype, int T, int64_t k_stride, int64_t v_stride,
                                        const int32_t *slot_map, hipStream_t stream) {
    const char *fn = "apex_paged_store";
    APEX_REQUIRE(T >= 0, "%s: T=%d must be >= 0", fn, T);
    apex_status st = apex::check_paged_cache(fn, cache, T > 0);
    if (st != APEX_OK) return st;
    APEX_REQUIRE(dtype == APEX_TYPE_FP32 || dtype == APEX_TYPE_BF16, "%s: unknown type %d", fn, dtype);
    const int G = cache->G, hd = cache->hd;
    if ((st = apex::check_rows(fn, "k", dtype, k_stride, int64_t(G) * hd)) != APEX_OK) return st;
    if ((st = apex::check_rows(fn, "v", dtype, v_stride, int64_t(G) * hd)) != APEX_OK) return st;
    if (T == 0) return APEX_OK;
    APEX_REQUIRE(k && v && slot_map, "%s: NULL pointer", fn);
    APEX_REQUIRE(apex::aligned16(k) && apex::aligned16(v) &&
                     reinterpret_cast<uintptr_t>(slot_map) % 4 == 0,
                 "%s: k and v must be 16-byte aligned", fn);
    const StoreArgs a{{k, v}, {k_stride, v_stride}, {cache->k_pages, cache->v_pages},
                      {cache->k_scales, cache->v_scales}, slot_map, int64_t(T) * G, G,
                      cache->page_size, apex::log2_of(cache->page_size),
                      cache->n_pages * cache->page_size};
    const int64_t blocks = (a.rows * (hd / 8) + kStoreThreads - 1) / kStoreThreads;
    if (blocks > UINT32_MAX / kStoreThreads)   // a grid has fewer than 2^32 threads
        return apex::fail(APEX_E_UNSUPPORTED, "%s: T=%d tokens of %d heads are too many", fn, T, G);
    const dim3 grid(unsigned(blocks), 2);
    const bool f32 = dtype == APEX_TYPE_FP32, f8 = cache->format == APEX_KV_FP8_E4M3;
    if (hd == 64)
        launch_store<64>(f32, f8, grid, stream, a);
    else
        launch_store<128>(f32, f8, grid, stream, a);
    APEX_HIP(hipGetLastError());
    return APEX_OK;
}
