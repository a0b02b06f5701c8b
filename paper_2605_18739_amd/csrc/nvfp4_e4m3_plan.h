// Which kernel a product of 8-bit operands takes: host-only C++, without HIP, so that a test can ask it without a GPU.
#pragma once

#include <cstdint>

namespace nvfp4 {

// Up to 64 rows are bound by the bytes of W and have a kernel of their own, which holds at most 64 rows of A in registers
// (64 x 4096 x 14336: 20 us; 65 rows of it, by tiles of 64 x 64, 33).
constexpr int64_t kE4m3FewRows = 64;

// Tiles: rows of A, rows of W (gated: half of them the gate's, so half as many columns of the result), and the time of a step (128 k) of a
// full round of tiles over the 256 compute units, ns, with exact and with fast sums.  From one size, 4096^3, which takes exact
// 105 / 117 / 106 / 112 / 118 / 160 us with the shapes in this order, fast 56 / 65 / 64 / 69 / 76 / 110.  What a tile takes before its
// first step and behind its last is not counted, so it weighs more than the rule knows where K is short.
struct E4m3Shape {
    int bm, bn, exact, fast;
};
constexpr E4m3Shape kE4m3Shapes[] = {
    {256, 256, 3150, 1750},
    {256, 128, 0, 1000},       // (exact sums 1800, and two rounds of 128 x 128 take 1760: never the least, so there is no such kernel)
    {128, 256, 1640, 980},
    {128, 128, 880, 540},
    {64, 256, 910, 600},
    {64, 64, 300, 215},
};
constexpr int kE4m3ShapeCount = 6;

inline int64_t e4m3_tiles(const E4m3Shape &c, int64_t M, int64_t N, bool gated)
{
    const int64_t bf = gated ? c.bn / 2 : c.bn;
    return ((M + c.bm - 1) / c.bm) * ((N + bf - 1) / bf);
}
// The shape whose rounds take least.  (Gated: a block of 128 columns of the result has to be a tile's, for its scale.)
inline int e4m3_shape(int64_t M, int64_t N, bool gated, bool fast)
{
    int best = -1;
    int64_t least = 0;
    for (int i = 0; i < kE4m3ShapeCount; ++i) {
        const E4m3Shape &c = kE4m3Shapes[i];
        const int step = fast ? c.fast : c.exact;
        if (step == 0 || (gated && c.bn != 256)) continue;
        const int64_t cost = (e4m3_tiles(c, M, N, gated) + 255) / 256 * step;
        if (best < 0 || cost < least) best = i, least = cost;
    }
    return best;
}
// Stages of LDS, (bm + bn) * 128 bytes each.  A tile that has a compute unit to itself has to hide the way to memory by its own copies,
// so four where they fit; with more tiles two of them share a compute unit and its LDS, and hide each other's waits.  Larger tiles: three
// with fast sums where they fit (128 x 256 on 4096^3, a product that the rule gives 256 x 256: 64 us, with two 70; exact sums: even).
constexpr int e4m3_stages(int bm, int bn, bool fast, int64_t tiles)
{
    if (bm + bn <= 128) return 4;
    if (bm + bn <= 320) return tiles <= 256 ? 4 : 2;
    return fast && bm + bn <= 384 ? 3 : 2;
}

}  // namespace nvfp4
