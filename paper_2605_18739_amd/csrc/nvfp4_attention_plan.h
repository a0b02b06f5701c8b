// Which attention kernel a call takes and into how many pieces it cuts the cached tokens: plain C++ without HIP types.
#ifndef NVFP4_ATTENTION_PLAN_H
#define NVFP4_ATTENTION_PLAN_H

#include <algorithm>
#include <cstdint>

namespace nvfp4 {

constexpr int kRows16Step = 32, kTileStep = 64;       // cached tokens of a step of either kernel
// rows16: heads of a workgroup at most, workgroups that the chip holds at once, steps of a piece at least
constexpr int kRows16Heads = 4, kRows16Slots = 512, kRows16MinSteps = 4;

struct AttentionPlan {
    bool rows16;            // at most 16 (query, head) rows a cached head: a wave per cached head and piece
    int waves;              // waves of a workgroup
    int groups;             // rows16: workgroups that a token's heads take; otherwise: blocks of rows of a cached head
    int pieces;             // rows16: of all sequences together, about; otherwise of each.  1: no partial results
    int piece_steps;        // steps of a piece (rows16: at least so many; the lengths, which the device knows, decide)
    int64_t part_rows;      // (query, head) rows of partial results
};

// max_kv: tokens of the longest cache; a window (with its sink tokens) leaves max_q queries at most so many of them to read
inline AttentionPlan attention_plan(int64_t total_q, int64_t Hq, int64_t H, int64_t d, int64_t max_kv, int64_t B, int64_t max_q, int64_t window,
                                    int64_t sink)
{
    AttentionPlan p{};
    if (window > 0) max_kv = std::min(max_kv, window + max_q + std::min(sink, max_kv) + 2 * kTileStep);
    const int64_t rows = max_q * (Hq / H);
    p.rows16 = rows <= 16;
    if (p.rows16) {
        p.groups = (int)((H + kRows16Heads - 1) / kRows16Heads);
        p.waves = (int)((H + p.groups - 1) / p.groups);
        const int64_t steps = std::max<int64_t>(1, (max_kv + kRows16Step - 1) / kRows16Step);
        p.piece_steps = kRows16MinSteps;
        // as many pieces as the chip holds at once (one that waits for another to end doubles the time of a short call): the
        // sequences are cut to a common length, so every one of them may add a shorter piece to those of full length
        const int64_t most = B * ((steps + kRows16MinSteps - 1) / kRows16MinSteps);
        p.pieces = (int)std::min(std::max<int64_t>(kRows16Slots / p.groups - B, std::min<int64_t>(B, 64)), most);
        if (steps <= kRows16MinSteps) p.pieces = 1;
        p.part_rows = p.pieces <= 1 ? 0 : (p.pieces + B) * max_q * Hq;
    } else {
        p.waves = d > 64 && d <= 128 && rows > 128 ? 8 : 4;
        p.groups = (int)((rows + 32 * p.waves - 1) / (32 * p.waves));
        const int64_t steps = std::max<int64_t>(1, (max_kv + kTileStep - 1) / kTileStep);
        const int64_t items = B * H * p.groups, slots = p.waves == 8 || d > 128 ? 256 : 512;
        // as many pieces as make whole waves of workgroups (a piece more costs a pass over the partial results), with at
        // least 8 steps each
        int best = 1;
        double best_cost = 1e30;
        for (int n = 1; n <= 64 && (n == 1 || steps / n >= 8); ++n) {
            const double rounds = (double)((items * n + slots - 1) / slots), cost = rounds / n * (1.0 + 0.02 * (n > 1 ? n : 0));
            if (cost < best_cost * 0.999) best = n, best_cost = cost;
        }
        p.piece_steps = (int)((steps + best - 1) / best);
        p.pieces = (int)((steps + p.piece_steps - 1) / p.piece_steps);
        p.part_rows = p.pieces <= 1 ? 0 : p.pieces * total_q * Hq;
    }
    return p;
}

inline size_t attention_workspace_bytes(const AttentionPlan &p, int64_t d) { return (size_t)p.part_rows * ((size_t)d * 4 + 8); }

}  // namespace nvfp4
#endif
