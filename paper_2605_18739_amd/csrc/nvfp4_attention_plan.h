// Which attention kernel a call takes and into how many pieces it cuts the cached tokens: plain C++ without HIP types.
#ifndef NVFP4_ATTENTION_PLAN_H
#define NVFP4_ATTENTION_PLAN_H

#include <algorithm>
#include <cstdint>

namespace nvfp4 {

constexpr int kRows16Step = 32, kTileStep = 64;       // cached tokens of a step of either kernel

struct AttentionPlan {
    bool rows16;            // at most 16 (query, head) rows a cached head: a wave per cached head and piece
    int waves;              // waves of a workgroup
    int groups;             // rows16: workgroups that a token's heads take; otherwise: blocks of rows of a cached head
    int pieces;             // of the cached tokens, at most; 1: no partial results
    int piece_steps;        // steps of a piece
};

// max_kv: tokens of the longest cache; a window (with its sink tokens) leaves max_q queries at most so many of them to read
inline AttentionPlan attention_plan(int64_t Hq, int64_t H, int64_t d, int64_t max_kv, int64_t B, int64_t max_q, int64_t window, int64_t sink)
{
    AttentionPlan p{};
    if (window > 0) max_kv = std::min(max_kv, window + max_q + std::min(sink, max_kv) + 2 * kTileStep);
    const int64_t rows = max_q * (Hq / H);
    p.rows16 = rows <= 16;
    if (p.rows16) {
        p.groups = (int)((H + 7) / 8);
        p.waves = (int)((H + p.groups - 1) / p.groups);
        const int64_t steps = std::max<int64_t>(1, (max_kv + kRows16Step - 1) / kRows16Step);
        // 4096 waves or more where the cache is long enough for pieces of 128 tokens
        const int64_t want = std::max<int64_t>(1, 4096 / (B * H));
        p.piece_steps = (int)std::max<int64_t>((steps + want - 1) / want, 4);
        p.pieces = (int)((steps + p.piece_steps - 1) / p.piece_steps);
    } else {
        p.waves = d <= 128 && rows > 128 ? 8 : 4;
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
    }
    return p;
}

// rows of a call's partial results
inline size_t attention_workspace_bytes(const AttentionPlan &p, int64_t total_q, int64_t Hq, int64_t d)
{
    return p.pieces <= 1 ? 0 : (size_t)p.pieces * (size_t)(total_q * Hq) * ((size_t)d * 4 + 8);
}

}  // namespace nvfp4
#endif
