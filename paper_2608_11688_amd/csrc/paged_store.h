// Device helpers of the kernels that write rows of keys and values into pages.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

namespace apex {
namespace paged {

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

// A row's scale and, of the 8 values that each of its LPR lanes (aligned) holds, the E4M3 codes:
// s = max / 448 and codes x / s; codes 0 where s is 0; NaN and codes 0 where a value is not finite.
template <int LPR>
__device__ __forceinline__ float e4m3_row(const float (&x)[8], uint32_t (&code)[2]) {
    // magnitudes compare as integers, infinity and NaN above every number
    uint32_t peak = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) peak = max(peak, __float_as_uint(x[e]) & 0x7fffffffu);
    peak = lanes_max<LPR>(peak);
    const bool bad = peak >= 0x7f800000u;
    const float s = __uint_as_float(peak) / 448.f;
    code[0] = code[1] = 0u;
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
    return bad ? NAN : s;
}

}  // namespace paged
}  // namespace apex
