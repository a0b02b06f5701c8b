// Which attention kernel a call takes and into how many pieces it cuts the cached tokens: plain C++ without HIP types.
#ifndef NVFP4_ATTENTION_PLAN_H
#define NVFP4_ATTENTION_PLAN_H

#include <algorithm>
#include <cstdint>

namespace nvfp4 {

constexpr int kRows16Step = 32, kTileStep = 64;       // cached tokens of a step of either kernel
// rows16: heads of a workgroup at most, workgroups of a call, and steps of a piece at least.  Two workgroups to a compute unit up to
// d = 128 and one above (whose registers leave room for one): eight caches of up to 16384 tokens, d = 64 / 128 / 256: 512
// workgroups take 17.0 / 20.4 / 40.9 us, 256 18.6 / 21.2 / 33.4.
// Steps of a piece: a step of a wave that has its SIMD alone takes 0.8 us, a partial result more next to nothing (five caches of up
// to 704 tokens, d = 64: pieces of four steps 9.0 + 5.2 us, of two 7.2 + 5.5).
constexpr int kRows16Heads = 4, kRows16Slots = 512, kRows16MinSteps = 2;
// Steps up to which a sequence is not cut (a second launch joins pieces).  Few sequences, us a call among others, whole / in pieces:
//   d = 64 (24 heads, one cache)   192 tokens 9.0 / 11.5, 256 10.3 / 11.8, 320 11.7 / 11.8
//   d = 128 (8 heads, one cache)   192 tokens 9.7 / 12.0, 256 11.3 / 11.6, 320 13.0 / 11.7; 16 caches 256 11.8 / 12.3, 320 13.6 / 12.2
//   d = 256 (8 heads, one cache)   128 tokens 12.8 / 15.1, 192 15.7 / 15.0, 256 18.8 / 15.0; 16 caches 128 13.4 / 15.3, 256 19.6 / 15.8
// Where the sequences are a quarter of the workgroups that the chip holds, or more, they fill it uncut (in a graph, 512 and 640 tokens):
//   d = 64, 32 x 24 heads  17.5 / 23.1, 20.7 / 26.9;  128 x 24  37.9 / 44.1, 45.0 / 51.2
//   d = 128, 64 x 8 heads  20.1 / 23.0, 24.0 / 24.8;  128 x 2   19.8 / 21.0, 23.6 / 22.6;  with fewer, 32 x 8  19.2 / 16.8, 22.7 / 17.2
//   d = 256, 64 x 8 heads  33.4 / 37.0, 39.2 / 43.0
constexpr int kRows16Whole = 8, kRows16WholeWide = 4, kRows16WholeMany = 20;         // (wide: above d = 128)
constexpr int kClearGroups = 256;                      // workgroups of a call that clear rows which no sequence computes, at most
constexpr int kTileMinSteps = 8;                       // steps of a piece of the other kernel, at least

struct AttentionPlan {
    bool rows16;            // at most 16 (query, head) rows a cached head: a wave per cached head and piece
    int waves;              // waves of a workgroup
    int groups;             // rows16: workgroups that a token's heads take; otherwise: blocks of rows of a cached head
    int pieces;             // rows16: of all sequences together, about; otherwise of a block of rows that is cut.  1: no partial results
    int piece_steps;        // steps of a piece, at least (the lengths, which the device knows, decide)
    int64_t whole, rest;    // blocks of rows (all sequences, heads) that are not cut, and those that are
    int64_t part_rows;      // (query, head) rows of partial results
};

constexpr int64_t kFar = 1ll << 30;                    // no position is that large: as good as no limit

// max_kv: tokens of the longest cache; a window (with its sink tokens) leaves max_q queries at most so many of them to read
inline AttentionPlan attention_plan(int64_t total_q, int64_t Hq, int64_t H, int64_t d, int64_t max_kv, int64_t B, int64_t max_q, int64_t window,
                                    int64_t sink)
{
    AttentionPlan p{};
    if (window > 0) max_kv = std::min(max_kv, std::min(window, kFar) + max_q + std::min(sink, kFar) + 2 * kTileStep);
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
        p.pieces = (int)std::min(std::max<int64_t>((d > 128 ? kRows16Slots / 2 : kRows16Slots) / p.groups - B, std::min<int64_t>(B, 64)), most);
        if (steps <= (B * p.groups >= kRows16Slots / 4 ? kRows16WholeMany : d > 128 ? kRows16WholeWide : kRows16Whole)) p.pieces = 1;
        p.part_rows = p.pieces <= 1 ? 0 : (p.pieces + B) * max_q * Hq;
    } else {
        // (eight waves: up to d = 64 a step has fewer pieces of keys than lanes, above d = 128 the accumulators leave room for four)
        p.waves = d > 64 && d <= 128 && rows > 128 ? 8 : 4;
        p.groups = (int)((rows + 32 * p.waves - 1) / (32 * p.waves));
        const int64_t steps = std::max<int64_t>(1, (max_kv + kTileStep - 1) / kTileStep);
        // Workgroups that the chip holds at once: as many blocks of rows as fill it a whole number of times walk over all their
        // tokens; what is left over is cut into pieces, so that it takes a part of a round instead of one of its own.  (A
        // piece more costs a pass over its partial results; 336 blocks: 256 whole and 80 in three pieces each take 1.34
        // rounds, all of them in three pieces as long, with four times the partial results.)
        const int64_t items = B * H * p.groups, slots = p.waves == 8 || d > 128 ? 256 : 512;
        const int64_t whole = items / slots * slots, rest = items - whole;
        int best = 1;
        double best_cost = 1e30;
        for (int n = 1; rest > 0 && n <= 64 && (n == 1 || steps / n >= kTileMinSteps); ++n) {
            const double cost = (double)((rest * n + slots - 1) / slots) / n * (1.0 + (n > 1 ? 0.02 * n : 0.0));
            if (cost < best_cost * 0.999) best = n, best_cost = cost;
        }
        p.pieces = best;
        p.piece_steps = kTileMinSteps;
        p.whole = best > 1 ? whole : items;
        p.rest = items - p.whole;
        p.part_rows = p.rest * best * 32 * p.waves;
    }
    return p;
}

inline size_t attention_workspace_bytes(const AttentionPlan &p, int64_t d) { return (size_t)p.part_rows * ((size_t)d * 4 + 8); }

}  // namespace nvfp4
#endif
