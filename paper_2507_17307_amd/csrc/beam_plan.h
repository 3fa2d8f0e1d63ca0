// How rs_beam_select deals a row's vocabulary to workgroups.  Plain C++ without HIP types, so that it can also be compiled and checked on a CPU.
#pragma once

#include "attn_plan.h"

namespace rs {

constexpr int BEAM_MAX = 64;                                       // beams of a group, and candidates
constexpr int BEAM_WAVES = 4, BEAM_THREADS = 64 * BEAM_WAVES;
constexpr int BEAM_BATCH = 1024;                                   // values a wave looks at together, 16 a lane
constexpr int BEAM_PARTS = 64;                                     // workgroups of a row, at most
constexpr int BEAM_KEYS = 4096;                                    // keys of a group's parts, at most: what the join of a group holds

struct BeamPlan { int parts, batches; };                           // workgroups of a row; batches that each wave of one takes

// The parts with the least of rounds * (batches + BEAM_START): `slots` workgroups run at once, and one costs as much as three batches before its first and behind its
// last one.  us of k_beam_scan, 152064 fp32 logits a row, of 24 x 16 rows with 32 candidates in 3 / 4 / 5 / 8 parts 75 / 71 / 71 / 83 (the rule takes 2 of
// 19 batches or 5 of 8, which cost the same by it), of 32 x 4 with 4 in 4 / 8 / 10 / 13 / 19 parts 25.7 / 24.5 / 26.7 / 27.3 / 29.3.
constexpr int BEAM_START = 3;
RS_HD BeamPlan beam_plan(int rows, int n_beams, int vocab, int n_out, int slots) {
    const long long all = ((long long)vocab + BEAM_BATCH * BEAM_WAVES - 1) / (BEAM_BATCH * BEAM_WAVES);      // parts of one batch a wave
    int most = BEAM_KEYS / (n_beams * n_out);
    if (most > BEAM_PARTS) most = BEAM_PARTS;
    BeamPlan best{0, 0};
    long long least = 0;
    for (int n = most; n >= 1; --n) {
        const long long each = (all + n - 1) / n, parts = (all + each - 1) / each, cost = (((long long)rows * parts + slots - 1) / slots) * (each + BEAM_START);
        if (!best.parts || cost < least) { best = {(int)parts, (int)each}; least = cost; }
    }
    return best;
}

}  // namespace rs
