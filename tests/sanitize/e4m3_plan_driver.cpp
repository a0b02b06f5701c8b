// Which kernel the 8-bit products take.  Without arguments: the rule's own invariants over a sweep of sizes, and every kernel that it can
// choose ("can ..."); with "gated M N" triples: the kernels of these ("takes ...").
#include "../../paper_2605_18739_amd/csrc/nvfp4_e4m3_plan.h"

#include <cstdio>
#include <cstdlib>
#include <set>
#include <string>

using namespace nvfp4;

static std::string kernel(int64_t M, int64_t N, bool gated, bool fast)
{
    char text[96];
    if (M <= kE4m3FewRows) {                               // the form for few rows: exact sums either way
        std::snprintf(text, sizeof text, "%s rows %d %s", gated ? "gated" : "plain", M <= 16 ? 16 : M <= 32 ? 32 : 64, (N + 15) / 16 > 256 ? "many" : "one");
        return text;
    }
    const int i = e4m3_shape(M, N, gated, fast);
    const E4m3Shape &c = kE4m3Shapes[i];
    std::snprintf(text, sizeof text, "%s %s %dx%d stages %d", gated ? "gated" : "plain", fast ? "fast" : "exact", c.bm, c.bn, e4m3_stages(c.bm, c.bn, fast, e4m3_tiles(c, M, N, gated)));
    return text;
}

int main(int argc, char **argv)
{
    std::set<std::string> seen;
    if (argc > 1) {
        for (int i = 1; i + 2 < argc; i += 3)
            for (bool fast : {false, true}) seen.insert(kernel(std::atoll(argv[i + 1]), std::atoll(argv[i + 2]), argv[i][0] == '1', fast));
        for (const std::string &s : seen) std::printf("takes %s\n", s.c_str());
        std::printf("ok\n");
        return 0;
    }
    for (bool gated : {false, true})
        for (bool fast : {false, true})
            for (int64_t M = 1; M < 20000; M += M < 700 ? 7 : 131)
                for (int64_t N = 1; N < 40000; N += N < 700 ? 15 : 241) {
                    seen.insert(kernel(M, N, gated, fast));
                    if (M <= kE4m3FewRows) continue;
                    const E4m3Shape &c = kE4m3Shapes[e4m3_shape(M, N, gated, fast)];
                    // a shape that has a time, gated columns by blocks of 128, LDS of a compute unit
                    if ((fast ? c.fast : c.exact) <= 0 || (gated && c.bn != 256)) return 1;
                    if (e4m3_stages(c.bm, c.bn, fast, e4m3_tiles(c, M, N, gated)) * (c.bm + c.bn) * 128 > 160 * 1024) return 2;
                }
    // sizes at the end of what a call takes
    for (bool gated : {false, true})
        for (bool fast : {false, true})
            if (e4m3_shape((int64_t)1 << 30, 16, gated, fast) < 0 || e4m3_shape(65, (int64_t)1 << 30, gated, fast) < 0) return 3;
    for (const std::string &s : seen) std::printf("can %s\n", s.c_str());
    std::printf("ok\n");
    return 0;
}
