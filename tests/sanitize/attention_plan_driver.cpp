// The attention plan over seeded shapes: every piece that the kernels can make of the lengths has its launch and its place
// among the partial results, and every block of rows is either whole or cut.
#include "../../paper_2605_18739_amd/csrc/nvfp4_attention_plan.h"

#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

using namespace nvfp4;

static void check(bool ok, const char *what, int64_t a, int64_t b)
{
    if (ok) return;
    std::printf("%s: %lld %lld\n", what, (long long)a, (long long)b);
    std::exit(1);
}

int main()
{
    std::mt19937_64 rng(5);
    auto upto = [&](int64_t n) { return (int64_t)(rng() % (uint64_t)n) + 1; };
    auto log_upto = [&](int bits) { return upto(1ll << upto(bits)); };
    int64_t rows16 = 0, cut = 0;
    for (int round = 0; round < 20000; ++round) {
        const int64_t d = 16 * upto(16), H = upto(24), G = upto(8), B = log_upto(10), max_q = upto(3) == 1 ? 1 : log_upto(12);
        const int64_t page = 16 * upto(64), max_kv = page * log_upto(12), window = upto(3) == 1 ? log_upto(14) : 0, sink = window ? log_upto(10) - 1 : 0;
        const int64_t total_q = std::max<int64_t>(max_q, B * max_q - upto(max_q) + 1);
        const AttentionPlan p = attention_plan(total_q, H * G, H, d, max_kv, B, max_q, window, sink);
        check(p.rows16 == (max_q * G <= 16), "form", max_q, G);
        check(p.waves > 0 && p.groups > 0 && p.pieces > 0, "sizes", p.waves, p.pieces);
        check((attention_workspace_bytes(p, d) == 0) == (p.part_rows == 0) && attention_workspace_bytes(p, d) == (size_t)(p.part_rows * (4 * d + 8)), "workspace", p.part_rows, d);
        if (p.rows16) {
            ++rows16;
            check(p.waves <= kRows16Heads && p.groups * p.waves >= H && (p.groups - 1) * p.waves < H, "heads", p.groups, p.waves);
            // the kernel's arithmetic: pieces of a common length, at least one of a sequence
            int64_t total = 0, pieces = 0;
            std::vector<int64_t> steps((size_t)B);
            for (int64_t &s : steps) {
                const int64_t len = upto(4) == 1 ? max_kv : upto(5) == 1 ? 0 : upto(max_kv);
                s = (len + kRows16Step - 1) / kRows16Step;
                total += s;
            }
            const int64_t length = p.pieces <= 1 ? 0x3FFFFFFF : std::max<int64_t>(std::min<int64_t>((total + p.pieces - 1) / p.pieces, 0x3FFFFFFF), p.piece_steps);
            for (int64_t s : steps) pieces += std::max<int64_t>((s + length - 1) / length, 1);
            const int64_t launched = p.pieces > 1 ? p.pieces + B : B;
            check(pieces <= launched, "pieces", pieces, launched);
            check(p.pieces <= 1 ? p.part_rows == 0 && pieces == B : pieces * max_q * H * G <= p.part_rows, "partial rows", pieces, p.part_rows);
        } else {
            const int64_t rows = max_q * G, items = B * H * p.groups;
            check(p.groups * 32 * p.waves >= rows && (p.groups - 1) * 32 * p.waves < rows, "blocks", p.groups, rows);
            check(p.whole >= 0 && p.rest >= 0 && p.whole + p.rest == items, "whole and cut", p.whole, p.rest);
            check(p.pieces > 1 || p.rest == 0, "nothing cut in one piece", p.pieces, p.rest);
            check(p.part_rows == p.rest * p.pieces * 32 * p.waves, "partial rows", p.part_rows, p.rest);
            const int64_t total = (max_kv + kTileStep - 1) / kTileStep + 1, length = std::max<int64_t>((total + p.pieces - 1) / p.pieces, p.piece_steps);
            check((total + length - 1) / length <= p.pieces, "pieces", total, p.pieces);
            cut += p.rest > 0;
        }
    }
    check(rows16 > 1000 && cut > 100, "both forms, with pieces", rows16, cut);
    std::printf("ok %lld %lld\n", (long long)rows16, (long long)cut);
}
