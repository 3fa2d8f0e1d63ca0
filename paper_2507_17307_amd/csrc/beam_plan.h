// How rs_beam_select deals a row's vocabulary to workgroups.  Plain C++ without HIP types, so that it can also be compiled and checked on a CPU.
#pragma once

#include "attn_plan.h"

namespace rs {

constexpr int BEAM_MAX = 64;                                       // beams of a group, and candidates
constexpr int BEAM_WAVES = 4, BEAM_THREADS = 64 * BEAM_WAVES;
constexpr int BEAM_BATCH = 1024;                                   // values a wave looks at together, 16 a lane
constexpr int BEAM_PARTS = 64;                                     // workgroups of a row, at most
constexpr int BEAM_KEYS = 4096;                                    // keys of a group's parts, at most: what the join of a group holds

struct BeamPlan { int parts, batches; };                           // workgroups of a row; batches of each wave of one by which it was chosen (beam_share deals them out)

// The parts with the least of rounds * (batches + BEAM_START): `slots` workgroups run at once, and one costs as much as three batches before its first and behind its
// last one.  us of a call, 152064 fp32 logits a row: 24 x 16 rows with 32 candidates in 2 / 3 / 4 / 5 / 8 parts 64 / 70 / 69 / 72 / 76 (2 of 19 batches
// and 5 of 8 cost the same by the rule, which takes the 5), 32 x 4 with 4 in 4 / 8 / 10 / 13 / 19 parts 30.4 / 30.4 / 32.5 / 33.0 / 35.2 (it takes 8).
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

// What a wave of a part takes of a row: pieces of 16 bytes unit_0 .. unit_end - 1, counted from the row's value `before`, the first on a 16-byte border, and
// `ends` single values: the `head` first of the row, then its last ones from `tail` on.  The pieces are shared evenly by as many waves as they fill (a wave
// with a few of them would have no border); the values before them are the first part's, those behind them the last one's, of its first wave.
struct BeamShare { int before, unit_0, unit_end, head, ends, tail; };
RS_HD BeamShare beam_share(int address_mod_16, int value_bytes, int vocab, int parts, int part, int wave) {
    const int unit = 16 / value_bytes, to_border = (16 - address_mod_16) % 16 / value_bytes, before = vocab < to_border ? vocab : to_border;
    const int pieces = (vocab - before) / unit, behind = vocab - before - pieces * unit, wave_units = BEAM_BATCH / unit;
    const int filled = (pieces + wave_units - 1) / wave_units, most = parts * BEAM_WAVES, waves = filled > most ? most : filled < 1 ? 1 : filled;
    const int own = (pieces + waves - 1) / waves, from = (part * BEAM_WAVES + wave) * own;
    BeamShare s{};
    s.before = before;
    s.unit_0 = pieces < from ? pieces : from;
    s.unit_end = pieces < s.unit_0 + own ? pieces : s.unit_0 + own;
    s.head = part == 0 ? before : 0;
    s.ends = wave == 0 ? s.head + (part == parts - 1 ? behind : 0) : 0;
    s.tail = vocab - behind;
    return s;
}
RS_HD int beam_end_token(const BeamShare &s, int i) { return i < s.head ? i : s.tail + (i - s.head); }      // of end i < ends

}  // namespace rs
