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
#include "ffn_device.h"
#include "paged_store.h"

namespace {

using apex::ffn::ld_stream;
using apex::paged::pack_bf16;

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
    int N, T, blocks, group;        // blocks of kBlock codes in a row
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

__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

template <bool F32>
__device__ __forceinline__ float load_y(const void *p, int64_t i) {
    if constexpr (F32) return static_cast<const float *>(p)[i];
    return __uint_as_float(uint32_t(static_cast<const uint16_t *>(p)[i]) << 16);
}
template <bool F32>
__device__ __forceinline__ void store_y(void *p, int64_t i, float v) {
    if constexpr (F32)
        static_cast<float *>(p)[i] = v;
    else
        static_cast<uint16_t *>(p)[i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// Rows: a workgroup takes 16 R rows of the weights and 16 TT tokens; its wavefronts take blocks of 128
// codes along K in turn and join their sums in LDS in a fixed order.
template <int P, int R, int TT, int WAVES, bool Y32>
__global__ __launch_bounds__(64 * WAVES) void linear_rows(LinearArgs a) {
    __shared__ floatx4 part[WAVES][R][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, quarter = lane >> 4;
    const int n0 = blockIdx.x * 16 * R, t0 = blockIdx.y * 16 * TT;
    const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
    const int per_block = kBlock / a.group, steps = a.group / 32;
    floatx4 sum[R][TT] = {};
    for (int b = wave; b < a.blocks; b += WAVES) {
        uint4 code[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = min(n0 + 16 * r + col, a.N - 1);
            code[r] = ld_stream(reinterpret_cast<const uint4 *>(a.codes + (int64_t(n) * a.blocks + b) * 64 + 16 * quarter));
        }
        floatx4 prod[R][TT] = {}, total[TT] = {};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = b * kBlock + 32 * j + 8 * quarter;
            bf16x8 x[P][TT];
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) {
                const int t = min(t0 + 16 * tt + col, a.T - 1);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (k < a.x_cols) v = *reinterpret_cast<const uint4 *>(a.x + p * a.x_piece + t * a.x_stride + k);
                    x[p][tt] = __builtin_bit_cast(bf16x8, v);
                    total[tt] = mfma(x[p][tt], ones, total[tt]);
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const uint32_t w = j == 0 ? code[r].x : j == 1 ? code[r].y : j == 2 ? code[r].z : code[r].w;
                const bf16x8 q = widen(w);
#pragma unroll
                for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                    for (int p = 0; p < P; ++p) prod[r][tt] = mfma(x[p][tt], q, prod[r][tt]);
            }
            if ((j + 1) % steps == 0) {      // a group ends
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int n = min(n0 + 16 * r + col, a.N - 1);
                    const uint32_t word = a.words[int64_t(b * per_block + j / steps) * a.N + n];
                    const float s = __uint_as_float(word & 0xffff0000u), z = 16.f + __uint_as_float(word << 16);
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            sum[r][tt][i] = fmaf(s, fmaf(-z, total[tt][i], prod[r][tt][i]), sum[r][tt][i]);
                        prod[r][tt] = floatx4{};
                    }
                }
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) total[tt] = floatx4{};
            }
        }
    }
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) {
        if (tt) __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) part[wave][r][lane] = sum[r][tt];
        __syncthreads();
        for (int i = threadIdx.x; i < R * 64; i += 64 * WAVES) {
            const int r = i >> 6, at = i & 63;
            floatx4 v = part[0][r][at];
            for (int w = 1; w < WAVES; ++w) v += part[w][r][at];
            const int n = n0 + 16 * r + (at & 15);
            if (n >= a.N) continue;
            const float bias = a.bias ? a.bias[n] : 0.f;
            for (int e = 0; e < 4; ++e) {
                const int64_t t = t0 + 16 * tt + 4 * (at >> 4) + e;
                if (t >= a.T) continue;
                float y = v[e] + bias;
                if (a.residual) y += load_y<Y32>(a.residual, t * a.residual_stride + n);
                store_y<Y32>(a.y, t * a.y_stride + n, y);
            }
        }
    }
}

// Rows of fp32 values as three rows of bf16 pieces whose sum they are, zeros behind K.
__global__ __launch_bounds__(256) void split_x(const float *x, int64_t stride, int T, int K, int Kp, uint16_t *out) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int lanes = Kp / 8;
    const int64_t t = i / lanes;
    const int k = int(i - t * lanes) * 8;
    if (t >= T) return;
    uint32_t p[3][4] = {};
    if (k < K) {
        const float4 *src = reinterpret_cast<const float4 *>(x + t * stride + k);
        const float4 u = src[0], v = src[1];
        const float f[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float rest = f[e];
#pragma unroll
            for (int j = 0; j < 3; ++j) {
                const uint32_t top = __float_as_uint(rest) & 0xffff0000u;
                p[j][e / 2] |= e & 1 ? top : top >> 16;
                rest -= __uint_as_float(top);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 3; ++j)
        *reinterpret_cast<uint4 *>(out + (int64_t(j) * T + t) * Kp + k) = make_uint4(p[j][0], p[j][1], p[j][2], p[j][3]);
}

bool sizes_ok(int N, int K, int group) { return apex_linear_w4_bytes(N, K, group) != 0; }

int padded(int K) { return (K + kBlock - 1) / kBlock * kBlock; }

template <int P, int TT, bool Y32>
void launch_rows(const LinearArgs &a, hipStream_t st) {
    const dim3 grid((a.N + 31) / 32, (a.T + 16 * TT - 1) / (16 * TT));
    hipLaunchKernelGGL((linear_rows<P, 2, TT, 8, Y32>), grid, dim3(512), 0, st, a);
}

template <int P, bool Y32>
void launch(const LinearArgs &a, hipStream_t st) {
    if (a.T <= 16)
        launch_rows<P, 1, Y32>(a, st);
    else if (a.T <= 32)
        launch_rows<P, 2, Y32>(a, st);
    else
        launch_rows<P, 4, Y32>(a, st);
}

bool is_type(int t) { return t == APEX_TYPE_FP32 || t == APEX_TYPE_BF16; }

}  // namespace

extern "C" size_t apex_linear_w4_workspace_bytes(int T, int N, int K, int group, int x_type) {
    if (T < 1 || T > APEX_MAX_STEP_TOKENS || !sizes_ok(N, K, group) || x_type != APEX_TYPE_FP32) return 0;
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
    const int Kp = padded(K);
    LinearArgs a{static_cast<const uint8_t *>(w),
                 reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(w) + size_t(N) * (Kp / 2)),
                 static_cast<const uint16_t *>(x), x_stride, 0, K, bias, residual, y, residual_stride, y_stride, N, T,
                 Kp / kBlock, group};
    if (x_type == APEX_TYPE_FP32) {
        uint16_t *pieces = static_cast<uint16_t *>(workspace);
        const int64_t items = int64_t(T) * (Kp / 8);
        hipLaunchKernelGGL(split_x, dim3(unsigned((items + 255) / 256)), dim3(256), 0, stream,
                           static_cast<const float *>(x), x_stride, T, K, Kp, pieces);
        APEX_HIP(hipGetLastError());
        a.x = pieces;
        a.x_stride = Kp;
        a.x_piece = int64_t(T) * Kp;
        a.x_cols = Kp;
        y_type == APEX_TYPE_FP32 ? launch<3, true>(a, stream) : launch<3, false>(a, stream);
    } else {
        y_type == APEX_TYPE_FP32 ? launch<1, true>(a, stream) : launch<1, false>(a, stream);
    }
    APEX_HIP(hipGetLastError());
    return APEX_OK;
}
