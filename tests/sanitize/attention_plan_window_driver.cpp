// The attention plan for windows and sinks as large as they come: as good as none, without an overflow on the way.
#include "../../paper_2605_18739_amd/csrc/nvfp4_attention_plan.h"

#include <cstdint>
#include <cstdio>
#include <cstdlib>

using namespace nvfp4;

static bool same(const AttentionPlan &a, const AttentionPlan &b)
{
    return a.rows16 == b.rows16 && a.waves == b.waves && a.groups == b.groups && a.pieces == b.pieces && a.piece_steps == b.piece_steps &&
           a.whole == b.whole && a.rest == b.rest && a.part_rows == b.part_rows;
}

int main()
{
    int n = 0;
    for (int64_t max_kv : {(int64_t)64, (int64_t)131072, (int64_t)1 << 30})
        for (int64_t max_q : {(int64_t)1, (int64_t)300})
            for (int64_t d : {(int64_t)64, (int64_t)256}) {
                const AttentionPlan none = attention_plan(max_q, 8, 2, d, max_kv, 1, max_q, 0, 0);
                for (int64_t window : {max_kv, (int64_t)1 << 40, INT64_MAX - 1, INT64_MAX})
                    for (int64_t sink : {(int64_t)0, (int64_t)1 << 40, INT64_MAX}) {
                        const AttentionPlan p = attention_plan(max_q, 8, 2, d, max_kv, 1, max_q, window, sink);
                        if (!same(p, none)) {
                            std::printf("window %lld, sink %lld over %lld tokens: %d pieces, %d without\n", (long long)window, (long long)sink, (long long)max_kv, p.pieces, none.pieces);
                            return 1;
                        }
                        // a sink alone bounds nothing that the window does not
                        const AttentionPlan narrow = attention_plan(max_q, 8, 2, d, max_kv, 1, max_q, 16, sink);
                        if (narrow.pieces < 1 || (sink >= max_kv && !same(narrow, none))) return 2;
                        ++n;
                    }
            }
    std::printf("ok %d\n", n);
    return 0;
}
