// Drives the packer of 4-bit projections and the rotary frequencies over random and invalid inputs,
// built with AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_host_sanitized_linear.py:
// every buffer is exactly as large as the declarations in apex.h say, so an access past it, or
// undefined behaviour inside, stops the program.  Prints "ok" when every check passed.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <limits>
#include <random>
#include <vector>

#include "apex.h"

namespace {

int failures = 0;

void check(bool ok, const char *what) {
    if (!ok) {
        std::printf("FAIL: %s\n", what);
        ++failures;
    }
}

float value(uint32_t upper) {
    const uint32_t u = upper << 16;
    float f;
    std::memcpy(&f, &u, sizeof f);
    return f;
}

void packers(std::mt19937 &rng) {
    for (int trial = 0; trial < 300; ++trial) {
        const int N = 1 + int(rng() % 20), K = 8 * (1 + int(rng() % 60)), group = 32 << (rng() % 3);
        const size_t Kp = (size_t(K) + 127) / 128 * 128, bytes = apex_linear_w4_bytes(N, K, group);
        check(bytes == size_t(N) * (Kp / 2 + 4 * (Kp / group)), "size of a packed projection");
        std::vector<uint16_t> w(size_t(N) * K);
        const bool any = trial % 3 == 0;             // any bits, NaN and infinities among them
        for (auto &v : w) v = uint16_t(any ? rng() : (0x3c00 + rng() % 0x400) | (rng() % 2 << 15));
        std::vector<uint8_t> out(bytes);
        check(apex_pack_linear_w4(w.data(), N, K, group, out.data()) == APEX_OK, "pack");
        if (any) continue;
        for (size_t n = 0; n < size_t(N); ++n)
            for (int k = 0; k < K; ++k) {
                const int in = k % 128, e = in % 8, bit = 4 * (e / 2) + 16 * (e % 2);
                uint32_t code, word;
                std::memcpy(&code, &out[n * (Kp / 2) + k / 128 * 64 + (in % 32 / 8 * 4 + in / 32) * 4], 4);
                std::memcpy(&word, &out[N * (Kp / 2) + (size_t(k / group) * N + n) * 4], 4);
                const float s = value(word >> 16), z = value(word & 0xffff);
                const float got = s * (float(code >> bit & 15) - z), want = value(w[n * K + k]);
                // half a step each by the code's and, at the range's ends, the zero point's rounding, and 15 times the
                // scale's, half a step of 2^-8
                check(std::fabs(got - want) <= (1.f + 15.f / 512) * s * 1.001f, "a weight is within a step");
            }
    }
    uint16_t w[8] = {};
    uint8_t out[1024];
    check(apex_pack_linear_w4(nullptr, 1, 8, 32, out) == APEX_E_INVAL, "NULL weights");
    check(apex_pack_linear_w4(w, 1, 8, 32, nullptr) == APEX_E_INVAL, "NULL output");
    check(apex_pack_linear_w4(w, 1, 12, 32, out) == APEX_E_INVAL, "K not a multiple of 8");
    check(apex_pack_linear_w4(w, 0, 8, 32, out) == APEX_E_INVAL, "no rows");
    check(apex_pack_linear_w4(w, 1, 8, 48, out) == APEX_E_INVAL, "group of 48");
    check(apex_linear_w4_bytes(-1, 8, 32) == 0 && apex_linear_w4_bytes(1, 0, 32) == 0 &&
              apex_linear_w4_bytes((1 << 24) + 1, 8, 32) == 0 && apex_linear_w4_bytes(1, 8, 0) == 0,
          "sizes of shapes that are refused");
    check(apex_linear_w4_bytes(1 << 24, 1 << 20, 32) == (size_t(1) << 24) * ((1 << 19) + 4 * (1 << 15)), "largest size");
}

void frequencies(std::mt19937 &rng) {
    const double inf = std::numeric_limits<double>::infinity(), nan = std::nan("");
    for (int trial = 0; trial < 2000; ++trial) {
        const int dim = 16 * (1 + int(rng() % 64)), scaling = int(rng() % 5);
        std::vector<double> f(dim / 2, -1.0);
        const double base = 1.0 + std::pow(10.0, int(rng() % 8) - 1), factor = 1.0 + rng() % 100;
        const double original = 1.0 + rng() % 100000, low = 0.5 + rng() % 4, high = low + 0.5 + rng() % 40;
        check(apex_rotary_frequencies(dim, base, scaling, factor, original, low, high, f.data()) == APEX_OK, "frequencies");
        for (double v : f) check(v > 0.0 && v <= 1.0, "a frequency is in (0, 1]");
    }
    std::vector<double> f(64);
    const double odd[] = {inf, -inf, nan, 0.0, -1.0, std::numeric_limits<double>::max(), std::numeric_limits<double>::denorm_min()};
    for (int scaling = 0; scaling < 5; ++scaling)
        for (double a : odd)
            for (double b : odd) {
                apex_rotary_frequencies(128, a, scaling, b, 4096, 1, 32, f.data());
                apex_rotary_frequencies(128, 1e4, scaling, 4, a, 1, b, f.data());
                apex_rotary_frequencies(128, 1e4, scaling, 4, a, b, 32, f.data());
            }
    check(apex_rotary_frequencies(128, 1e4, 0, 1, 0, 0, 0, nullptr) == APEX_E_INVAL, "NULL output");
    for (int dim : {0, -16, 8, 24, 1040}) check(apex_rotary_frequencies(dim, 1e4, 0, 1, 0, 0, 0, f.data()) == APEX_E_INVAL, "dim");
    check(apex_rotary_frequencies(128, 1e4, 5, 1, 0, 0, 0, f.data()) == APEX_E_INVAL, "scaling");
}

}  // namespace

int main() {
    std::mt19937 rng(20261208);
    packers(rng);
    frequencies(rng);
    if (failures) {
        std::printf("%d failures\n", failures);
        return 1;
    }
    std::printf("ok\n");
    return 0;
}
