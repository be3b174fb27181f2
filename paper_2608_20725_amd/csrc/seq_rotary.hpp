// Internal definitions of rotary positions: what their host side
// (seq_cache_api.cpp) passes to the launch.
#pragma once

#include "seq.hpp"

namespace im2win {

// Turns (mod 1) a position of each pair, as fractions of 2^64.  They travel as a
// kernel argument, most calls' in half of it: a launch with 1 KB of arguments
// takes 3.9 us, with 300 bytes 3.4.
constexpr int kMaxPairs = 128, kUsualPairs = 64;
template <int PAIRS>
struct TurnsOf {
    uint64_t turn[PAIRS];
};
typedef TurnsOf<kMaxPairs> Turns;

struct RotaryArgs {
    const char *x;
    char *y;
    const int32_t *pos;                        // by token, by sequence, or null: 0, 1, ..
    int64_t x_sb, x_st, x_sh, y_sb, y_st, y_sh;  // bytes between sequences, tokens, heads
    FastDiv units, groups, len;                // units of a head, groups of heads, tokens of a sequence
    uint32_t lanes;
    int32_t H, D, rot, pair_units, by_token, few, in_place;
    float amplitude, sin_amplitude;
};

// Fills the launch's shape in; false where it would need 2^32 lanes or more.
bool plan_rotary(RotaryArgs &a, int64_t B, int64_t L, bool paired, bool in_place, int dt);
hipError_t launch_rotary(const RotaryArgs &a, const Turns &f, bool paired, int dt, hipStream_t st);

}  // namespace im2win
