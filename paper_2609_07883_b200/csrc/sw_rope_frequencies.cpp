// Frequencies of rotary positions, on the host: turns per position of every pair, with the usual ways to stretch them for long contexts.
#include <algorithm>
#include <cmath>

#include "sw.h"
#include "sw_error.h"

extern "C" sw_status sw_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_len, double low, double high,
                                         double* turns, float* magnitude) {
    if (!turns || !magnitude) return sw_fail(SW_ERR_INVALID_ARG, "sw_rope_frequencies: null argument");
    if (rotary_dim < 16 || rotary_dim % 16 != 0 || rotary_dim > 128)
        return sw_fail(SW_ERR_UNSUPPORTED, "sw_rope_frequencies: rotary_dim %d (multiples of 16 up to 128)", rotary_dim);
    if (scaling < SW_ROPE_PLAIN || scaling > SW_ROPE_RAMP) return sw_fail(SW_ERR_INVALID_ARG, "sw_rope_frequencies: scaling %d", scaling);
    const bool by_wavelength = scaling == SW_ROPE_BANDS || scaling == SW_ROPE_RAMP;
    if (!(base > 1.) || !std::isfinite(base) || (scaling != SW_ROPE_PLAIN && (!(factor >= 1.) || !std::isfinite(factor))))
        return sw_fail(SW_ERR_INVALID_ARG, "sw_rope_frequencies: base %g, factor %g (more than 1, at least 1)", base, factor);
    if (by_wavelength && (!(original_len >= 1.) || !std::isfinite(original_len) || !(low > 0.) || !(high > low) || !std::isfinite(high)))
        return sw_fail(SW_ERR_INVALID_ARG, "sw_rope_frequencies: original_len %g, low %g, high %g", original_len, low, high);
    const double two_pi = 2. * std::acos(-1.);
    const int half = rotary_dim / 2;
    if (scaling == SW_ROPE_BASE) base *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
    // SW_ROPE_RAMP: the pair that turns t times over the original length
    auto pair_of = [&](double t) { return half * std::log(original_len / (t * two_pi)) / std::log(base); };
    const double first = by_wavelength ? std::max(std::floor(pair_of(high)), 0.) : 0.;
    const double last = by_wavelength ? std::min(std::ceil(pair_of(low)), (double)rotary_dim - 1.) : 0.;
    for (int i = 0; i < half; ++i) {
        const double w = std::pow(base, -(double)i / half) / two_pi;
        double kept = 1.;   // share of the frequency that is not stretched
        if (scaling == SW_ROPE_LINEAR) kept = 0.;
        if (scaling == SW_ROPE_BANDS) kept = std::min(std::max((original_len * w - low) / (high - low), 0.), 1.);
        if (scaling == SW_ROPE_RAMP) kept = 1. - std::min(std::max((i - first) / std::max(last - first, 1e-3), 0.), 1.);
        turns[i] = kept == 1. ? w : w * (kept + (1. - kept) / factor);
    }
    *magnitude = scaling == SW_ROPE_RAMP ? (float)(0.1 * std::log(factor) + 1.) : 1.f;
    return SW_OK;
}
