// How the attention's passes are launched, of sizes that the host knows.  Host code without a GPU's headers.
#pragma once

#include <stdint.h>

#include <initializer_list>

#include "harp.h"

namespace harp {
namespace attention {

constexpr int kKeys = 64;            // keys of a tile in LDS, where rows stay
constexpr int kBack = 32;            // rows of one, where keys stay
constexpr int kJoinRows = 8;         // rows of a workgroup that joins shares
constexpr int kDies = 8;
constexpr int64_t kMostThreads = (int64_t(1) << 32) - 1;       // of a launch
constexpr int64_t kMostJoins = (int64_t(1) << 23) - 1;         // workgroups of one that joins two results

inline bool sizes_fit(const harp_attention *g) {
    const int64_t most = (int64_t(1) << 30) - 1;
    return g->tokens_q >= 0 && g->tokens_k >= 0 && g->tokens_q <= most && g->tokens_k <= most && g->batch >= 1 && g->batch <= 1 << 20 &&
           g->heads >= 1 && g->heads <= 1 << 14 && g->kv_heads >= 1 && g->heads % g->kv_heads == 0 && g->head >= 8 && g->head % 8 == 0 &&
           g->head <= HARP_ATTENTION_MAX_HEAD && g->tokens_q * (g->heads / g->kv_heads) <= most;
}

// With begins on the device a pass has room for a partial tile of every sequence.
struct Plan {
    int waves;                       // of a workgroup
    int64_t tiles;                   // of rows, or of keys
    int shares;                      // of what a tile goes through
    bool paired;                     // a workgroup takes two tiles
    int64_t places() const { return paired ? (tiles + 1) / 2 : tiles; }
    // Kv heads that fit one launch, at most `heads`: whole rounds of the dies where there are so many.  One does always: a kv head has less
    // than 2^30 rows and 2^20 sequences, 2^23 + 2^20 tiles of 128 or 2^22 + 2^20 of 256.
    int64_t heads_of_a_launch(int64_t heads) const {
        const int64_t each = places() * shares * waves * 64, fit = each > 0 ? kMostThreads / each : heads;
        return fit >= heads ? heads : fit >= kDies ? fit / kDies * kDies : fit;
    }
};
inline int64_t tiles_of(int64_t tokens, int64_t times, int batch, int side) {
    const int64_t whole = tokens * times / side, each = (tokens / batch * times + side - 1) / side * batch;
    // equal lengths need `each`; begins on the device at most this
    return whole + batch > each ? whole + batch : each;
}
// Microseconds by what was measured: `step` for a tile of 256 by the 64 (32) rows that go through LDS at a time with 128 channels, 6
// around them.  Tiles of 128 are two to a compute unit, at the same pace where both are there.  `bytes` that a share's sums take
// are written and read by a launch more, of `joins` workgroups.  The `through` rows are shared out where tiles are few, or, under the
// causal order, differ.
inline Plan plan_for(int n_cu, int64_t tokens, int64_t times, int batch, int kv_heads, int64_t through, int unit, double step, int head,
                     double bytes, int64_t joins, bool causal, bool may_pair) {
    Plan best = {};
    double least = 1e300;
    const double channels = head <= 64 ? 0.5 : head <= 96 ? 0.75 : 1.0;
    const int64_t rows = tokens * times / batch;
    for (int waves = 8; waves >= 4; waves -= 4) {
        const int64_t side = 32 * waves, slots = int64_t(n_cu) * 8 / waves;
        const int64_t busy = (rows > side ? (rows + side - 1) / side : 1) * batch * kv_heads;       // tiles that have something to do
        for (int shares : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (shares > 1 && (through < int64_t(shares) * unit || joins > kMostJoins)) break;
            const int64_t items = busy * shares;
            const double steps = double((through + unit - 1) / unit) / shares;
            const double each = step * channels * (waves == 4 && items <= n_cu ? 0.6 : 1.0);
            const int64_t rounds = (items + slots - 1) / slots, pairs = (items + 1) / 2, pair_rounds = (pairs + slots - 1) / slots;
            const double alone = steps * each + 6;
            double us = double(rounds) * alone;
            bool paired = false;
            if (causal) {
                // heavy tiles first; workgroups are handed to shader engines in turn and wait for their own, so that they do not
                // even out.  A heavy and a light one in one workgroup are alike.
                const double spread = 1.25 * double(items) / double(slots) * (steps * each / 2 + 6);
                us = alone > spread ? alone : spread;
                const double both = double(pair_rounds) * (steps * each + 12);
                if (may_pair && both < us) us = both, paired = true;
            }
            if (shares > 1) us += 8 + shares * bytes * 2 / 4e6;
            if (waves == 4) us *= 1.1;                           // keys are read twice as often
            const Plan plan = {waves, tiles_of(tokens, times, batch, int(side)), shares, paired};
            if (us < least && plan.heads_of_a_launch(1) >= 1) least = us, best = plan;
        }
    }
    return best;
}
inline int64_t query_joins(const harp_attention *g) {
    return tiles_of(g->tokens_q, g->heads / g->kv_heads, g->batch, kJoinRows) * g->kv_heads;
}
inline Plan plan_queries(int n_cu, const harp_attention *g, bool causal) {
    const int group = g->heads / g->kv_heads;
    return plan_for(n_cu, g->tokens_q, group, g->batch, g->kv_heads, g->tokens_k / g->batch, kKeys, 2.4, g->head,
                    double(g->tokens_q) * g->heads * g->head * 4, query_joins(g), causal, true);
}
inline Plan plan_keys(int n_cu, const harp_attention *g, bool causal) {
    return plan_for(n_cu, g->tokens_k, 1, g->batch, g->kv_heads, g->tokens_q / g->batch * (g->heads / g->kv_heads), kBack, 2.4, g->head,
                    double(g->tokens_k) * g->kv_heads * g->head * 8, tiles_of(g->tokens_k, g->kv_heads, g->batch, kJoinRows), causal, false);
}

}  // namespace attention
}  // namespace harp
