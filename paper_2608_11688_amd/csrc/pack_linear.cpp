// Packing of projections with 4-bit weights (apex_linear_w4_bytes, apex_pack_linear_w4): a scale and
// a zero point per row and group.  Host code only; the layout is in apex.h.
//
// A row's 64-byte block of 128 codes is one load of 16 bytes for each of four lanes: lane a of them
// holds in word j the 8 codes that the matrix instruction j of the block takes from it (values
// 32 j + 8 a + e), so that every instruction's 32 values are of one group.  Elements 2 i and 2 i + 1
// of a word stand at bits 4 i and 16 + 4 i: one shift and mask yields both, as a pair of 16 bits.
#include <cmath>
#include <cstring>

#include "common.h"

namespace {

double bf16_value(uint16_t bits) {
    const uint32_t u = uint32_t(bits) << 16;
    float f;
    std::memcpy(&f, &u, sizeof f);
    return f;
}

// To nearest even; v is finite or NaN.
uint16_t bf16_bits(float v) {
    if (std::isnan(v)) return 0x7fc0;
    uint32_t u;
    std::memcpy(&u, &v, sizeof u);
    return uint16_t((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

double clamp15(double v) { return std::fmin(std::fmax(v, 0.0), 15.0); }

int padded(int K) { return (K + 127) / 128 * 128; }

bool sizes_ok(int N, int K, int group) {
    return N >= 1 && N <= (1 << 24) && K >= 8 && K % 8 == 0 && K <= (1 << 20) &&
           (group == 32 || group == 64 || group == 128);
}

}  // namespace

extern "C" size_t apex_linear_w4_bytes(int N, int K, int group) {
    if (!sizes_ok(N, K, group)) return 0;
    const size_t Kp = size_t(padded(K));
    return size_t(N) * (Kp / 2 + 4 * (Kp / group));
}

extern "C" apex_status apex_pack_linear_w4(const uint16_t *w, int N, int K, int group, void *out) {
    const char *fn = "apex_pack_linear_w4";
    APEX_REQUIRE(w && out, "%s: NULL pointer", fn);
    APEX_REQUIRE(sizes_ok(N, K, group),
                 "%s: N=%d (1 to 2^24), K=%d (multiple of 8 to 2^20) or group=%d (32, 64, 128) out of range",
                 fn, N, K, group);
    const size_t Kp = size_t(padded(K));
    uint8_t *codes = static_cast<uint8_t *>(out);
    uint8_t *words = codes + size_t(N) * (Kp / 2);
    std::memset(out, 0, apex_linear_w4_bytes(N, K, group));
    for (size_t n = 0; n < size_t(N); ++n) {
        const uint16_t *row = w + n * size_t(K);
        for (int g = 0; g * group < K; ++g) {
            const int first = g * group, last = first + group < K ? first + group : K;
            double lo = 0.0, hi = 0.0;
            bool finite = true;
            for (int k = first; k < last; ++k) {
                const double v = bf16_value(row[k]);
                finite = finite && std::isfinite(v);
                lo = std::fmin(lo, v);
                hi = std::fmax(hi, v);
            }
            uint16_t s_bits = 0x7fc0, z_bits = 0;
            if (finite) {
                s_bits = bf16_bits(float((hi - lo) / 15.0));
                const double s = bf16_value(s_bits);
                if (s > 0.0) {
                    const double z = lo < 0.0 ? clamp15(std::nearbyint(-lo / s)) : 0.0;
                    z_bits = bf16_bits(float(z));
                    for (int k = first; k < last; ++k) {
                        const uint32_t q = uint32_t(clamp15(std::nearbyint(bf16_value(row[k]) / s) + z));
                        const int in = k % 128, j = in / 32, a = in % 32 / 8, e = in % 8;
                        const int bit = 4 * (e / 2) + 16 * (e % 2);
                        uint8_t *p = codes + n * (Kp / 2) + size_t(k / 128) * 64 + (4 * a + j) * 4 + bit / 8;
                        *p = uint8_t(*p | q << (bit % 8));
                    }
                }
            }
            const uint32_t word = uint32_t(s_bits) << 16 | z_bits;
            std::memcpy(words + (size_t(g) * N + n) * 4, &word, 4);
        }
    }
    return APEX_OK;
}
