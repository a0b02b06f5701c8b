// Attention over the paged NVFP4 cache for many rows (queries times the heads that share a cached head): chunks of a
// video, prompts.  Bound by the matrix pipes and the vector pipes' exponentials together.
#include "nvfp4_attention.h"

#include <type_traits>

namespace nvfp4 {

// A workgroup takes 32 WAVES rows of one cached head and walks over the cached tokens, 64 at a time:
//  - all its lanes turn the step's codes into f16 (code * block scale, exact) in LDS, once for all rows: keys as they lie,
//    values transposed (a nibble transposition between pairs of tokens in registers), two stages in turn, the next step's
//    codes in flight while this one's products run;
//  - a wave multiplies for its own 32 rows, S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16_f16: a lane holds query
//    row lane & 31 in both, so maxima, sums and rescaling stay in the lane (one exchange with lane ^ 32 when the running
//    maximum rises), and the weights are the second product's operand as they are, once the value columns in LDS are in
//    the order in which S^T leaves its tokens: of every sixteen {0-3, 8-11} for lanes 0-31 and {4-7, 12-15} for lanes 32-63.
// LDS rows are 16-byte chunks, the chunk's place exclusive-or'ed with bits of the row, so that eight neighbouring rows read
// (or written) at one chunk lie in different banks.
// Measured (24 heads of 128, 3520 queries over 18480 tokens, smoothed keys): 945 us and 17 to join, 830 TFLOP/s, where a
// library's product of 8192 x 8192 matrices holds 1170 to 1215: no single pipe is full (counters: matrix instructions 45 % of the SIMDs'
// cycles, vector ones 52, LDS 34 of the CUs'), and the clock depends on the operands (all zeros: a fifth less time).
// 2000 queries over 8192 tokens of 16 heads: d = 64 130 us (matrix 22 %, vector 54: as many exponentials for half of the products),
// 128 163, with smoothed keys 173, 256 450 (25 and 40: one wave a SIMD, whose waits nothing fills).  The same with pages
// whose scales are far apart (16 tokens a page, d = 128, with the join 191): one page of zeros 184, every eighth 365, 2^-8 to 2^8 at
// random 709.  Four waves for up to 128 rows, because waves without rows only load.
template <int D, int WAVES>
struct Tiles {
    static constexpr int kThreads = 64 * WAVES;
    static constexpr int kTasks = 4 * D / kThreads;       // blocks of keys, and pieces of values, of a lane
    uint8_t k[2][kTileStep * D * 2];      // [token][D] f16
    uint8_t v[2][D * kTileStep * 2];      // [element][token] f16
    struct alignas(16) {
        float mean[kTileStep];            // row mean / g_k
        float kg[4], log_v[4], inv_v[4];  // of the four groups of sixteen tokens
        uint8_t exponent[4];              // of their value scales
    } of[2];
    // what only some steps ask for, kept out of the scalar registers, which the addresses of a step's loads fill
    struct {
        int p0, p1, window, sink;         // positions of the block's first and last query
        int unit[WAVES], unit_top[WAVES];
        int pass, again_from[4], again_to[4];       // number of the walk, and of each the steps with groups for the next one
    } rare;
};

// (integral constants 0 .. N - 1, for code that has to be laid out by hand)
template <int N, class F>
__device__ __forceinline__ void each(F &&f)
{
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(std::integral_constant<int, N - 1>());
    }
}

// What a wave does in a turn is laid out by hand, because the compiler reads a fragment right in front of the instruction
// that multiplies it and waits for LDS every time (18480 tokens, 3520 x 24 queries: 1120 us):
//   Q K^T   the next fragments are read while the present ones are multiplied, and the next step's codes are turned into f16
//           in between (their loads were issued a turn before);
//   loads of the step behind that one;
//   the maximum; then the weights of sixteen tokens while the sixteen before are multiplied with their values.
// The fences keep what stands between them in place.
#define NVFP4_FENCE __builtin_amdgcn_sched_barrier(0)

// SMOOTH: the keys' row means enter as an outer product, (mean / g_k) x (sum of the query's elements), by one
// v_mfma_f32_32x32x2_f32 into the accumulator that the codes are then added to: the vector pipe has no time for them.
template <int D, int WAVES, bool SMOOTH, bool F32>
__global__ __launch_bounds__(64 * WAVES, D == 256 ? 1 : 2) void attention_tiles_kernel(const AttentionArgs a, const int32_t *__restrict__ page_table,
                                                                          const int32_t *__restrict__ kv_lens, const int32_t *__restrict__ q_starts,
                                                                          const float *__restrict__ k_global, const float *__restrict__ v_global)
{
    if (blockIdx.x >= a.clear_from) return clear_rest<F32>(a, q_starts);
    using Lds = Tiles<D, WAVES>;
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    Lds &lds = *reinterpret_cast<Lds *>(lds_bytes);
    constexpr int kThreads = Lds::kThreads, kTasks = Lds::kTasks, kRows = 32 * WAVES;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c32 = lane & 31, hi = lane >> 5;

    // whole blocks first, then the pieces of the others: all first pieces, all second ones, ...
    int64_t at = blockIdx.x;
    int piece = -1;
    if (at >= a.plan.whole) {
        const int64_t rest = (a.plan.rest + 7) & ~(int64_t)7, j = at - a.plan.whole;
        piece = (int)(j / rest);
        if (j - piece * rest >= a.plan.rest) return;
        at = a.plan.whole + (j - piece * rest);
    }
    const Block place(a, at);
    const int b = place.b, h = place.h, block = place.block;
    const Sequence seq(a, q_starts, kv_lens, b);
    const int n_q = min(seq.n_q, a.max_q), row0 = block * kRows;
    if (row0 >= n_q * a.G) return;
    const int i0 = row0 / a.G, i1 = min((row0 + kRows - 1) / a.G, n_q - 1);
    const Steps steps(a, seq, i0, i1, kTileStep);
    const int piece_steps = piece < 0 ? steps.total : tile_piece_steps(a, steps.total);
    const bool alone = steps.total <= piece_steps;         // no partial results
    const int n0 = max(piece, 0) * piece_steps, n1 = min(n0 + piece_steps, steps.total);
    if (n0 >= n1 && piece > 0) return;

    // ---- this lane's share of a step: blocks of keys (token, block) and pieces of values (pair of tokens, eight elements).
    // The tasks of a wave lie in one group of sixteen tokens, so its page is the wave's; like everything else it comes
    // through vector loads, which return in order, and it is looked up a step ahead of its use.
    constexpr int NB = D / 16, NE = D / 8;
    static_assert(4 * D >= kThreads, "every lane has a task");
    const uint32_t token_codes = a.token_codes, token_scales = a.token_scales;
    constexpr uint32_t kZero = 0x0Cu;                      // (of a byte permutation: zero)
    uint32_t zero;                                         // (an offset that the compiler takes for a lane's own)
    asm("v_mov_b32 %0, 0" : "=v"(zero));
    // offsets within a group: a lane's task has the same place in each of its groups
    const int token16 = (tid / NB) & 15, blk = tid % NB, pair8 = (tid / NE) & 7, part = tid % NE;
    // (lanes of elements from d on load the row's first ones: the queries are zero there, and those sums are not stored)
    const uint32_t k_blk = 16 * blk < a.d ? blk : 0, v_part = 8 * part < a.d ? part : 0;
    uint32_t k_at = token16 * token_codes + (uint32_t)h * (uint32_t)(a.d >> 1) + 8u * k_blk;
    const uint32_t ks_byte = token16 * token_scales + (uint32_t)h * (uint32_t)(a.d >> 4) + k_blk;
    uint32_t ks_at = ks_byte & ~3u;
    const uint32_t ks_pick = (ks_byte & 3u) * 0x10001u | kZero << 8 | kZero << 24;
    uint32_t v_at0 = 2 * pair8 * token_codes + (uint32_t)h * (uint32_t)(a.d >> 1) + 4u * v_part, v_at1 = v_at0 + token_codes;
    const uint32_t vs_byte0 = 2 * pair8 * token_scales + (uint32_t)h * (uint32_t)(a.d >> 4) + (v_part >> 1), vs_byte1 = vs_byte0 + token_scales;
    uint32_t vs_at0 = vs_byte0 & ~3u, vs_at1 = vs_byte1 & ~3u;
    const uint32_t vs_pick = (vs_byte0 & 3u) | ((vs_byte1 & 3u) + 4u) << 16 | kZero << 8 | kZero << 24;
    uint32_t mean_at = ((uint32_t)(token16 * a.H + h) * 2u) & ~3u;
    const uint32_t mean_shift = ((uint32_t)(token16 * a.H + h) & 1u) * 16u;
    struct Share {
        uint2v k[kTasks];
        uint32_t ks[kTasks], v[kTasks][2], vs[kTasks][2], mean[kTasks], kg[kTasks], vg[kTasks];
        bool valid[kTasks];
    };
    struct Ahead {
        int offset[kTasks];
        uint32_t page[kTasks];
    };
    auto group_of = [&](int t) { return (64 * wave + t * kThreads) / (16 * NB); };
    auto as_loaded = [](uint32_t &v) { asm volatile("" : "+v"(v)); };
    const GlobalBytes table = scalar_base(page_table, (uint64_t)b * a.max_pages * 4), k_scale = scalar_base(k_global, 0), v_scale = scalar_base(v_global, 0);
    auto look_up = [&](int n, int to) {
        Ahead p;
        const int first = steps.first_token(min(n, to - 1), kTileStep);
#pragma unroll
        for (int t = 0; t < kTasks; ++t) {  // (a group past the length is masked; it may be past the table: the step's first group stands in)
            const int token = first + 16 * group_of(t) < seq.len ? first + 16 * group_of(t) : first;
            const int at = (int)a.by_page.small((uint32_t)token);
            p.offset[t] = token - at * a.page_tokens;
            p.page[t] = load_at<uint32_t>(table, 4u * (uint32_t)at + zero);
        }
        return p;
    };
    // fetches the step whose pages were looked up, and looks up those of step n (or of the last one, to - 1)
    auto fetch = [&](Ahead &p, Share &s, int n, int to) {
        uint32_t pages[kTasks];
#pragma unroll
        for (int t = 0; t < kTasks; ++t) {
            as_loaded(p.page[t]);
            pages[t] = (uint32_t)__builtin_amdgcn_readfirstlane((int)p.page[t]);
        }
        const Ahead now = p;
        p = look_up(n, to);
        // (offsets are widened where they are used: widened once in front of the loop, they would no longer be known to have 32 bits)
        as_loaded(k_at), as_loaded(ks_at), as_loaded(v_at0), as_loaded(v_at1), as_loaded(vs_at0), as_loaded(vs_at1), as_loaded(mean_at);
#pragma unroll
        for (int t = 0; t < kTasks; ++t) {
            s.valid[t] = pages[t] < (uint32_t)a.n_pages;
            const uint32_t page = s.valid[t] ? pages[t] : 0u;
            s.kg[t] = load_at<uint32_t>(k_scale, 4u * page + zero);
            s.vg[t] = load_at<uint32_t>(v_scale, 4u * page + zero);
            const Slots at(a, page, now.offset[t]);
            s.k[t] = load_at<uint2v>(at.k_codes, k_at);
            s.ks[t] = load_at<uint32_t>(at.k_scales, ks_at);
            s.v[t][0] = load_at<uint32_t>(at.v_codes, v_at0);
            s.v[t][1] = load_at<uint32_t>(at.v_codes, v_at1);
            s.vs[t][0] = load_at<uint32_t>(at.v_scales, vs_at0);
            s.vs[t][1] = load_at<uint32_t>(at.v_scales, vs_at1);
            if constexpr (SMOOTH) s.mean[t] = load_at<uint32_t>(at.k_mean, mean_at);
        }
        __builtin_amdgcn_sched_barrier(0);                 // (the loads stay in front of what follows)
    };
    // ---- places in LDS: 16-byte chunk c of row r at r * (row size) + (c ^ key(r)) * 16.  Keys: token rows of D / 8 chunks, key
    // r % 16 (r % 8 where there are eight chunks); values: element rows of eight chunks, key (r ^ r / 8) % 8.
    constexpr uint32_t kKRow = 2 * D, kVRow = 2 * kTileStep, kKStage = kTileStep * kKRow, kVStage = D * kVRow, kVBase = 2 * kKStage;
    constexpr int kKeyMask = (D / 8 - 1) & 15;
    const int token0 = tid / NB, pair0 = tid / NE, quarter = (pair0 >> 1) & 3;
    uint32_t k_to = (uint32_t)token0 * kKRow + (uint32_t)(((2 * blk) ^ (token0 & kKeyMask)) << 4);     // (the block's second chunk: ^ 16)
    // tokens 2 pair and 2 pair + 1 of their sixteen lie in quarter (pair / 2) % 4; quarter 2 x + y goes to chunk y (of the sixteen's two), half x
    uint32_t v_to = kVBase + 8u * part * kVRow + (uint32_t)(((2 * group_of(0) + (quarter & 1)) ^ part) & 7) * 16u + 8u * (quarter >> 1) + 4u * (pair0 & 1);
    constexpr int kPieces = 7;                             // of a task
    uint32_t even[kTasks], odd[kTasks];
    half2v sv[kTasks];
    // a stage is chosen by one bit of an address, so it is flipped by ^ kKStage, ^ kVStage; k_to, v_to point at the stage that
    // is written, k_from, v_from at the one that is read
    auto store_piece = [&](Share &s, int stage, auto piece_constant) {
        constexpr int t = decltype(piece_constant)::value / kPieces, i = decltype(piece_constant)::value % kPieces;
        constexpr uint32_t k_off = t * (kThreads / NB) * kKRow;
        if constexpr (i < 2) {
            const half2v sk = scale_pair(__builtin_amdgcn_perm(0u, s.ks[t], ks_pick));
            *(half8v *)(lds_bytes + (k_to ^ (i == 0 ? 0u : 16u)) + k_off) = eight_codes(i == 0 ? s.k[t].x : s.k[t].y, sk);
        } else if constexpr (i == 2) {
            // nibbles of the two tokens side by side: byte j of `even` is element 2 j of both, of `odd` element 2 j + 1
            even[t] = (s.v[t][0] & 0x0F0F0F0Fu) | ((s.v[t][1] << 4) & 0xF0F0F0F0u);
            odd[t] = ((s.v[t][0] >> 4) & 0x0F0F0F0Fu) | (s.v[t][1] & 0xF0F0F0F0u);
            sv[t] = scale_pair(__builtin_amdgcn_perm(s.vs[t][1], s.vs[t][0], vs_pick));
            if (blk == 0) {
                const float kg = __uint_as_float(s.kg[t]), vg = __uint_as_float(s.vg[t]);
                if constexpr (SMOOTH) lds.of[stage].mean[token0 + t * (kThreads / NB)] = __uint_as_float((s.mean[t] >> mean_shift) << 16) * __builtin_amdgcn_rcpf(kg);
                if (token16 == 0) {
                    lds.of[stage].kg[group_of(t)] = kg;
                    lds.of[stage].log_v[group_of(t)] = __builtin_amdgcn_logf(vg);
                    lds.of[stage].inv_v[group_of(t)] = __builtin_amdgcn_rcpf(vg);
                    lds.of[stage].exponent[group_of(t)] = (uint8_t)(s.valid[t] ? scale_exponent(s.vg[t]) : kNoPage);
                }
            }
        } else {
            constexpr int b = i - 3;                       // elements 2 b and 2 b + 1 of the eight
            const uint32_t to = v_to ^ (uint32_t)((2 * (group_of(t) ^ group_of(0))) << 4);
            *(half2v *)(lds_bytes + (to ^ (2 * b) << 4) + 2 * b * kVRow) = code_pair<b>(even[t]) * sv[t];
            *(half2v *)(lds_bytes + (to ^ (2 * b + 1) << 4) + (2 * b + 1) * kVRow) = code_pair<b>(odd[t]) * sv[t];
        }
    };

    // the first step's loads go out before the queries are read
    Share share;
    Ahead ahead = {};
    if (n0 < n1) {
        ahead = look_up(n0, n1);
        fetch(ahead, share, n0 + 1, n1);
    }

    // ---- queries of this wave's rows: lane holds row c32, elements 16 step + 8 hi .. + 7 of every k step
    const int my_row = row0 + 32 * wave + c32, i = my_row / a.G, head = h * a.G + (my_row - i * a.G);
    const bool row = i < n_q;
    const Sight sight(a, seq.position(a, i));
    const int64_t query = (int64_t)seq.start + i;
    half8v q[D / 16];
    float factor, sum_q;                                   // score = (S + (mean / g_k) sum_q) factor g_k, base 2
    {
        uint4v w[D / 16];
        float amax = 0.0f, sum = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            const int e = 16 * c + 8 * hi;
            w[c] = uint4v{0u, 0u, 0u, 0u};
            if (row && e < a.d) w[c] = *(const uint4v *)(a.q + query * a.ldq + (int64_t)head * a.d + e);
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) amax = absmax8(w[c], amax);
        amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
        const int e = row_exponent(amax);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            q[c] = query_pairs(w[c], e);
            if constexpr (SMOOTH) sum = sum8(w[c], e, sum);
        }
        sum += __shfl_xor(sum, 32, 64);
        factor = fmaxf(__builtin_amdgcn_ldexpf(a.scale, -e), 0x1p-126f);
        sum_q = hi == 0 ? sum : 0.0f;        // (the outer product has two terms, one of them zero)
    }

    float m = kLowest, r = kLowest, l = 0.0f;
    uint32_t lowest4 = 0u;                                 // of the wave's unit (0: none yet, or not the first walk)
    float16v o[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;

    // steps from sure_from on (a window's rear) up to sure_to (the first query) are seen whole by all rows
    const int sure_to = seq.position(a, i0) - kTileStep + 1, sure_from = a.window > 0 ? seq.position(a, i1) - a.window : -1;
    if (tid == 0) lds.rare.p0 = seq.position(a, i0), lds.rare.p1 = seq.position(a, i1), lds.rare.window = a.window, lds.rare.sink = a.sink;
    if (lane == 0) lds.rare.unit[tid >> 6] = lds.rare.unit_top[tid >> 6] = kNoUnit;
    if (tid < 4) lds.rare.again_from[tid] = 0x7FFFFFFF, lds.rare.again_to[tid] = 0;
    const bool busy = row0 + 32 * wave < n_q * a.G;        // (a wave behind the last row only loads)
    // this lane's chunks: keys 2 c + hi of row c32 (+ 32), values 2 g + hi of row c32 (+ 32 c, whose key has bit 2 the other way where c is odd)
    uint32_t k_from = (uint32_t)c32 * kKRow + (uint32_t)((hi ^ (c32 & kKeyMask)) << 4);
    uint32_t v_from = kVBase + (uint32_t)c32 * kVRow + (uint32_t)((hi ^ c32 ^ (c32 >> 3)) & 7) * 16u;

    constexpr int KF = D / 16, VF = D / 32, NK = 2 * KF, kDepth = 8;       // fragments of a step's keys, of sixteen tokens' values; keys read ahead
    auto k_fragment = [&](auto f) {                            // fragment f: tile f % 2, chunk pair f / 2
        constexpr int F = decltype(f)::value, t = F & 1, c = F >> 1;
        return *(const half8v *)(lds_bytes + (k_from ^ (uint32_t)((c & 7) << 5)) + (t * 32 * kKRow + (c >> 3) * 256));
    };
    auto v_fragment = [&](auto f) {                            // fragment f: group f / VF, rows 32 (f % VF) on
        constexpr int F = decltype(f)::value, g = F / VF, c = F % VF;
        return *(const half8v *)(lds_bytes + (v_from ^ (uint32_t)((g ^ ((c & 1) << 1)) << 5)) + c * 32 * kVRow);
    };
    auto turn = [&](int n, int from, int to, auto runs) {
        const int stage = (n - from) & 1;
        const auto &of = lds.of[stage];
        constexpr int kStore = kTasks * kPieces;
        const int first = steps.first_token(n, kTileStep);
        // (what is made from these is made again in every turn: kept, it would push the queries out of the registers)
        as_loaded(k_to), as_loaded(v_to), as_loaded(k_from), as_loaded(v_from);
        if constexpr (!decltype(runs)::value) {
            each<kStore>([&](auto i) { store_piece(share, stage ^ 1, i); });
            fetch(ahead, share, n + 3, to);
            return;
        }

        // ---- S^T = K Q^T
        half8v kf[kDepth];
        float16v x[2];
        each<kDepth>([&](auto f) { kf[decltype(f)::value] = k_fragment(f); });
        float mean[2] = {0.0f, 0.0f};
        if constexpr (SMOOTH) {
            mean[0] = of.mean[c32];
            mean[1] = of.mean[32 + c32];
        }
        const uint32_t exponents = *(const uint32_t *)of.exponent;
        float4v kg = *(const float4v *)of.kg, log_v = *(const float4v *)of.log_v, inv_v = *(const float4v *)of.inv_v;
        NVFP4_FENCE;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[t][e] = 0.0f;
        each<NK>([&](auto f) {
            constexpr int F = decltype(f)::value, t = F & 1, c = F >> 1;
            x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[F % kDepth], q[c], x[t], 0, 0, 0);
            if constexpr (F + kDepth < NK) kf[F % kDepth] = k_fragment(std::integral_constant<int, F + kDepth>());
            if constexpr (SMOOTH && c == KF / 2) x[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(mean[t], sum_q, x[t], 0, 0, 0);
            constexpr int p0 = F * kStore / NK, p1 = (F + 1) * kStore / NK;
            each<p1 - p0>([&](auto i) { store_piece(share, stage ^ 1, std::integral_constant<int, p0 + decltype(i)::value>()); });
            NVFP4_FENCE;
        });
        const uint32_t there = (uint32_t)__builtin_amdgcn_readfirstlane((int)exponents);
        const bool known = unit_holds4(lowest4, there);        // (all four pages are ones of the cache, among other things)
        const bool masked = (first > sure_to) | (first <= sure_from);
        half8v vf[2][VF];
        each<VF>([&](auto f) { vf[0][decltype(f)::value] = v_fragment(f); });
        fetch(ahead, share, n + 3, to);

        // ---- the row's maximum.  x[t][e]: token 32 t + 8 (e / 4) + 4 hi + e % 4, group 2 t + e / 8
        bool moved = false;
        if (masked | !known) {
            int at = first;
            asm volatile("" : "+s"(at));                        // (what is made from it stays in here)
            const int p0 = __builtin_amdgcn_readfirstlane(lds.rare.p0), p1 = __builtin_amdgcn_readfirstlane(lds.rare.p1);
            const int window = __builtin_amdgcn_readfirstlane(lds.rare.window), sink = __builtin_amdgcn_readfirstlane(lds.rare.sink);
            uint32_t seen = 0u;                                 // groups of which some row sees some token
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if ((there >> 8 * g & 255u) != kNoPage && group_seen(at + 16 * g, p0, p1, window, sink)) seen |= 1u << g;
            if (masked | (seen != 15u)) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int j = 32 * t + 8 * (e >> 2) + 4 * hi + (e & 3), g = 2 * t + (e >> 3);
                        x[t][e] = (((seen >> g & 1u) != 0u) & sight.of(at + j)) ? x[t][e] : -__builtin_inff();
                    }
                // (of a page that is not in use anything may stand there; and no product of factors is so small that it is zero, which makes
                // no number of a masked score)
                const float least = __builtin_amdgcn_rcpf(factor) * 0x1p-126f;
#pragma unroll
                for (int g = 0; g < 4; ++g) kg[g] = (seen >> g & 1u) != 0u ? fmaxf(kg[g], least) : 1.0f;
            }
            // the unit of the pages: it moves in front of the step, and groups whose pages are far from the others' wait for another walk
            const int before = __builtin_amdgcn_readfirstlane(lds.rare.unit[tid >> 6]), pass = __builtin_amdgcn_readfirstlane(lds.rare.pass);
            Units units = {before, __builtin_amdgcn_readfirstlane(lds.rare.unit_top[tid >> 6])};
            const uint32_t mine = units.enter<4>(there, seen, pass);
            if (seen != 0u) lds.rare.again_from[pass] = min(lds.rare.again_from[pass], n), lds.rare.again_to[pass] = n + 1;      // (every wave writes the same)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float log_g = log_v[g], inv_g = inv_v[g];
                units.page((int)(there >> 8 * g & 255u), log_g, inv_g);
                log_v[g] = (mine >> g & 1u) != 0u ? log_g : -__builtin_inff();
                inv_v[g] = (mine >> g & 1u) != 0u ? inv_g : 0.0f;
            }
            moved = units.now != before;
            lds.rare.unit[tid >> 6] = units.now, lds.rare.unit_top[tid >> 6] = units.top;
            lowest4 = pass == 0 && units.now != kNoUnit ? unit_lowest4(units.now) : 0u;
        }
        float f[4], top = kLowest;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f[g] = factor * kg[g];                               // (positive: the largest score is the largest product)
            const float16v &v = x[g >> 1];
            const int e = 8 * (g & 1);
            const float t0 = fmaxf(fmaxf(v[e], v[e + 1]), v[e + 2]), t1 = fmaxf(fmaxf(v[e + 3], v[e + 4]), v[e + 5]);
            top = fmaxf(top, fmaxf(fmaxf(t0, t1), fmaxf(v[e + 6], v[e + 7])) * f[g]);
        }
        if (__ballot(top > m + kAbove) != 0ull || moved) {
            m = fmaxf(floorf(fmaxf(top, __shfl_xor(top, 32, 64)) - kBelow), m);
            const float to = m + (float)(lds.rare.unit[tid >> 6] - kUnitBias), f = __builtin_amdgcn_exp2f(r - to);
            l = moved_sum(l, r, to);
            r = to;
#pragma unroll
            for (int t = 0; t < VF; ++t) o[t] *= f;
        }

        // ---- weights, O^T = V^T P^T
        half8v w[2], w_low[2];
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        auto weights = [&](auto group, auto pair_constant) {   // two of a group's eight
            constexpr int g = decltype(group)::value, e = 2 * decltype(pair_constant)::value;
            const float add = log_v[g] - r;
            const float v0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[g >> 1][8 * (g & 1) + e], f[g], add));
            const float v1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[g >> 1][8 * (g & 1) + e + 1], f[g], add));
            sum[g] += v0;
            sum[g] += v1;
            const half2v both = {(_Float16)v0, (_Float16)v1};
            w[g & 1][e] = both.x;
            w[g & 1][e + 1] = both.y;
            if constexpr (F32) {
                w_low[g & 1][e] = (_Float16)(v0 - (float)both.x);
                w_low[g & 1][e + 1] = (_Float16)(v1 - (float)both.y);
            }
        };
        each<4>([&](auto i) { weights(std::integral_constant<int, 0>(), i); });
        NVFP4_FENCE;
        each<4>([&](auto group) {
            constexpr int g = decltype(group)::value;
            each<VF>([&](auto column) {
                constexpr int c = decltype(column)::value;
                if constexpr (g < 3) vf[(g + 1) & 1][c] = v_fragment(std::integral_constant<int, (g + 1) * VF + c>());
                o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[g & 1][c], w[g & 1], o[c], 0, 0, 0);
                if constexpr (F32) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[g & 1][c], w_low[g & 1], o[c], 0, 0, 0);
                if constexpr (g < 3) {
                    constexpr int p0 = c * 4 / VF, p1 = (c + 1) * 4 / VF;
                    each<p1 - p0>([&](auto i) { weights(std::integral_constant<int, g + 1>(), std::integral_constant<int, p0 + decltype(i)::value>()); });
                }
                NVFP4_FENCE;
            });
        });
#pragma unroll
        for (int g = 0; g < 4; ++g) l = __builtin_fmaf(sum[g], inv_v[g], l);
        asm volatile("" : "+v"(l));                             // (summed up here: sunk behind the barrier, the weights would wait for it in registers)
    };

    // A turn reads one stage and writes the other; the barrier behind it says that both are done.  (What is fetched past the
    // last step is the last step again.)  Groups that a walk leaves out are taken by another one over the steps that have some
    // (four groups, four walks at most).
    for (int pass = 0, from = n0, to = n1; from < to; ++pass) {
        if (tid == 0) lds.rare.pass = pass;
        if (pass > 0) lowest4 = 0u;
        each<kTasks * kPieces>([&](auto i) { store_piece(share, 0, i); });
        fetch(ahead, share, from + 2, to);
        k_to ^= kKStage, v_to ^= kVStage;
        __syncthreads();
        auto walk = [&](auto runs) {
            for (int n = from; n < to; ++n) {
                turn(n, from, to, runs);
                k_to ^= kKStage, v_to ^= kVStage, k_from ^= kKStage, v_from ^= kVStage;
                __syncthreads();
            }
        };
        if (busy) walk(std::true_type());
        else walk(std::false_type());
        if (((to - from) & 1) == 0) k_to ^= kKStage, v_to ^= kVStage;        // (the next walk begins with stage 0 again)
        else k_from ^= kKStage, v_from ^= kVStage;
        from = __builtin_amdgcn_readfirstlane(lds.rare.again_from[pass]), to = __builtin_amdgcn_readfirstlane(lds.rare.again_to[pass]);
        if (from < to) {
            ahead = look_up(from, to);
            fetch(ahead, share, from + 1, to);
        }
    }

    l += __shfl_xor(l, 32, 64);
    if (!row) return;
    // o[c][e]: element 32 c + 8 (e / 4) + 4 hi + e % 4
    const int64_t out_row = query * a.Hq + head;
    if (alone) {
        const float inv = inverse_sum(l);
        if (a.lse && hi == 0) a.lse[out_row] = log_sum(r, l);
        const int64_t at = query * a.ldo + (int64_t)head * a.d;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int first = 32 * c + 2 * e + 4 * hi;
                if (first >= a.d) continue;
                if constexpr (F32) *(float4v *)((float *)a.out + at + first) = float4v{o[c][e] * inv, o[c][e + 1] * inv, o[c][e + 2] * inv, o[c][e + 3] * inv};
                else *(uint2v *)((uint16_t *)a.out + at + first) = uint2v{pack_bf16x2(o[c][e] * inv, o[c][e + 1] * inv), pack_bf16x2(o[c][e + 2] * inv, o[c][e + 3] * inv)};
            }
        return;
    }
    const int64_t part_row = ((at - a.plan.whole) * a.plan.pieces + piece) * kRows + (32 * wave + c32);
    if (hi == 0) a.part_ml[part_row] = float2{r, l};
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int first = 32 * c + 2 * e + 4 * hi;
            if (first < a.d) *(float4v *)(a.part_o + part_row * a.d + first) = float4v{o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]};
        }
}

template <int D, int WAVES, bool SMOOTH, bool F32>
static hipError_t launch_variant(AttentionArgs a, const KvAttention &k, hipStream_t s)
{
    auto kernel = attention_tiles_kernel<D, WAVES, SMOOTH, F32>;
    constexpr int bytes = (int)sizeof(Tiles<D, WAVES>);
    static bool raised[64] = {};                                       // the dynamic LDS limit, once per device
    int dev = -1;
    if (hipError_t e = hipGetDevice(&dev)) return e;
    if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
    if (!raised[dev]) {
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes)) return e;
        raised[dev] = true;
    }
    const unsigned grid = attention_grid(a, k, (unsigned)(a.plan.whole + ((a.plan.rest + 7) & ~(int64_t)7) * a.plan.pieces));
    kernel<<<grid, 64 * WAVES, bytes, s>>>(a, k.page_table, k.kv_lens, k.q_starts, k.cache.k_global, k.cache.v_global);
    return hipGetLastError();
}
template <int D, int WAVES>
static hipError_t launch_tiles(const AttentionArgs &a, const KvAttention &k, hipStream_t s)
{
    if (a.k_mean) return k.out_f32 ? launch_variant<D, WAVES, true, true>(a, k, s) : launch_variant<D, WAVES, true, false>(a, k, s);
    return k.out_f32 ? launch_variant<D, WAVES, false, true>(a, k, s) : launch_variant<D, WAVES, false, false>(a, k, s);
}

hipError_t launch_attention_tiles(AttentionArgs a, const KvAttention &k, hipStream_t s)
{
    if (a.d > 128) return launch_tiles<256, 4>(a, k, s);
    if (a.d <= 64) return launch_tiles<64, 4>(a, k, s);
    return a.plan.waves == 8 ? launch_tiles<128, 8>(a, k, s) : launch_tiles<128, 4>(a, k, s);
}

}  // namespace nvfp4
