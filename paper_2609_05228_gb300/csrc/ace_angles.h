// ace_angles.h — the frequencies of rotary positions as fractions of a turn.
#pragma once

#include <math.h>

#include <cstdint>

#include "ace.h"

namespace ace {

// f_i in turns a position, off by (3 + ln base) 2^-53 of itself at most: the exponent -2 i / rot_dim is off by 2^-54, pow, pi and
// the products by little. BY_TURNS, between its ends: by factor * high / (high - low) times that, as the number of turns is a difference.
inline double rope_frequency(const ace_rope_desc& D, int i) {
    constexpr double kTwoPi = 6.283185307179586476925;
    const double t = pow(D.base, -2.0 * i / D.rot_dim) / kTwoPi;
    double keep = 1.0;
    if (D.scaling == ACE_ROPE_LINEAR) {
        keep = 0.0;
    } else if (D.scaling == ACE_ROPE_BY_TURNS) {
        keep = (D.original_len * t - D.low) / (D.high - D.low);
    } else if (D.scaling == ACE_ROPE_BY_INDEX) {
        auto index_of = [&](double turns) { return D.rot_dim * log(D.original_len / (turns * kTwoPi)) / (2.0 * log(D.base)); };
        const double lo = fmax(floor(index_of(D.high)), 0.0), hi = fmin(ceil(index_of(D.low)), D.rot_dim - 1.0);
        keep = 1.0 - (i - lo) / ((hi == lo ? lo + 0.001 : hi) - lo);
    }
    keep = fmin(fmax(keep, 0.0), 1.0);
    return D.scaling == ACE_ROPE_NONE ? t : t * (keep + (1.0 - keep) / D.factor);
}

// f (>= 0, finite) without its whole turns in units of 2^-64 of a turn, to nearest. (No carry: the fraction is a double below 1, so
// 2^64 times it is 2^64 - 2^11 at most, and whole from 2^53 on.)
inline uint64_t rope_turn(double f) { return (uint64_t)rint(ldexp(f - floor(f), 64)); }

}  // namespace ace
