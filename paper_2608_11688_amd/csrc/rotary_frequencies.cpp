// Frequencies of rotary positions and their scaling for long contexts (apex_rotary_frequencies).  Host
// code only.
#include <algorithm>
#include <cmath>

#include "common.h"

extern "C" apex_status apex_rotary_frequencies(int dim, double base, int scaling, double factor,
                                               double original, double low, double high, double *freq) {
    const char *fn = "apex_rotary_frequencies";
    const double pi = 3.14159265358979323846;
    APEX_REQUIRE(freq, "%s: NULL pointer", fn);
    APEX_REQUIRE(dim >= 16 && dim <= 1024 && dim % 16 == 0, "%s: dim=%d must be a multiple of 16 up to 1024", fn, dim);
    APEX_REQUIRE(base > 1.0 && std::isfinite(base), "%s: base=%g must be above 1", fn, base);
    APEX_REQUIRE(scaling >= APEX_ROPE_PLAIN && scaling <= APEX_ROPE_INDEX, "%s: unknown scaling %d", fn, scaling);
    if (scaling != APEX_ROPE_PLAIN)
        APEX_REQUIRE(factor >= 1.0 && std::isfinite(factor), "%s: factor=%g must be at least 1", fn, factor);
    const bool ramp = scaling == APEX_ROPE_TURNS || scaling == APEX_ROPE_INDEX;
    if (ramp)
        APEX_REQUIRE(original > 0.0 && std::isfinite(original) && low > 0.0 && low < high && std::isfinite(high),
                     "%s: original=%g, low=%g and high=%g must be 0 < original and 0 < low < high", fn, original,
                     low, high);
    if (scaling == APEX_ROPE_BASE) {
        base *= std::pow(factor, double(dim) / (dim - 2));
        APEX_REQUIRE(std::isfinite(base), "%s: the scaled base is infinite", fn);
    }
    const auto index = [&](double turns) {
        return dim * std::log(original / (2.0 * pi * turns)) / (2.0 * std::log(base));
    };
    const double i0 = ramp ? std::max(std::floor(index(high)), 0.0) : 0.0;
    const double i1 = ramp ? std::min(std::ceil(index(low)), dim - 1.0) : 0.0;
    for (int i = 0; i < dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / dim);
        double r = 1.0;    // how much of f itself
        if (scaling == APEX_ROPE_LINEAR) r = 0.0;
        if (scaling == APEX_ROPE_TURNS) r = (original * f / (2.0 * pi) - low) / (high - low);
        if (scaling == APEX_ROPE_INDEX) r = 1.0 - (i - i0) / std::max(i1 - i0, 0.001);
        r = std::min(std::max(r, 0.0), 1.0);
        freq[i] = r == 1.0 ? f : f * ((1.0 - r) / factor + r);
    }
    return APEX_OK;
}
