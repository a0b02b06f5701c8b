// Attention over the paged NVFP4 cache for at most sixteen (query, head) rows a cached head: single tokens and small
// groups of heads.  Bound by the cache's bytes: 0.5625 B an element of keys and of values.
#include "nvfp4_attention.h"

#include <type_traits>

namespace nvfp4 {

// A wave takes one cached head and one piece of a sequence's tokens, 32 tokens a step; the waves of a workgroup take
// neighbouring heads of the same tokens, whose rows share cache lines.  Nothing goes through LDS:
//   S^T = K Q^T   v_mfma_f32_16x16x32_f16, keys as the A operand: lane (r = lane & 15, g = lane >> 4) needs elements of token r;
//                 which elements of the row belong to group g is free as long as the queries agree, so a lane takes the
//                 D / 4 neighbours from g D / 4 on: one load of D / 8 bytes.  The result leaves lane (r, g) with tokens
//                 4 g .. 4 g + 3 of both groups of sixteen for query row r.
//   O^T = V^T P^T the same lane then holds its eight weights as the B operand already, in the token order
//                 {4 g .. 4 g + 3, 16 + 4 g .. 16 + 4 g + 3}; the values are loaded in that order, a lane taking
//                 D / 16 neighbouring elements of each of its eight tokens, and a nibble transposition between pairs of
//                 tokens turns them into the A operand.  Rows of O^T are elements, columns query rows: maxima, sums and
//                 rescaling never cross lanes.
// SMOOTH: the keys' row means enter as an outer product of their own, (mean / g_k) x (sum of the query's elements), by one
// v_mfma_f32_16x16x4_f32 into the accumulator that the codes are then added to.
// FULL: d = D.  Otherwise lanes of elements from d on load the row's first ones (finite, and the queries are zero there).
// The loop's loads are whole aligned words without branches, so that the compiler can count them: a step's loads are in
// flight while the one before is multiplied, and the pages of the step behind it are looked up.  Scale bytes and means come
// as the word that holds them (slots start at multiples of sixteen rows, so which byte it is does not change from step to
// step, and the planes' sizes are multiples of sixteen bytes: no word reaches past the end).
// The same word is asked for once where lanes share it: a step takes 16 loads, and lanes hand scales and means on (d = 128;
// with a load for every lane's own, 28 loads: 41 us where this takes 39, d = 80 24 -> 22).
// Measured (eight caches of up to 28672 tokens, 114688 together, 32 query heads of 8 cached, d = 128, smoothed keys, 134 MB): 38 us and
// 6 to join, 3.5 TB/s; 7 us of it before the first product (launch, lengths, pages, first loads, queries), the rest 4.3 TB/s.  A
// third buffer of loads, three workgroups to a compute unit and codes that go through LDS to load rows in order changed nothing
// (40, 39, 38 us); with every page the same one, and so from L2, 33 us.  Counters: vector instructions 43 % of the SIMDs' cycles, matrix
// ones 8, waves waiting 25 % of theirs, 1.2 waves a SIMD (a wave has the registers of two steps).  Eight caches of up to 16384
// tokens in pages of 16 whose scales are far apart (with the join 41): one page of zeros 41, every eighth 77, 2^-8 to 2^8 at random 81.
template <int D, bool FULL>
struct Step {
    static constexpr int KW = D / 32;                      // key words of a lane
    static constexpr int KS = D / 64;                      // words with scale bytes: FULL: of a token, otherwise of a lane's blocks
    static constexpr int SW = D == 256 ? 2 : 1;            // FULL: of these, words that a lane loads
    uint32_t k[2][KW], ks[FULL ? 1 : 2][FULL ? SW : KS], v[8], v_hi[D == 256 ? 8 : 1], vs[FULL ? SW : 8], mean[FULL ? 1 : 2];
    uint32_t kg, vg;                                       // the pages' scales (fp32): lanes 0-31 of the first group's page, the others of the second's
    int first;                                             // the step's first token
    bool valid[2];                                         // the group of sixteen lies on a page of the cache
};

template <int D, bool FULL, bool SMOOTH, bool F32>
__global__ __launch_bounds__(64 * kRows16Heads, D == 256 ? 1 : 2) void attention_rows16_kernel(const AttentionArgs a, const int32_t *__restrict__ page_table,
                                                               const int32_t *__restrict__ kv_lens, const int32_t *__restrict__ q_starts,
                                                               const float *__restrict__ k_global, const float *__restrict__ v_global)
{
    if (blockIdx.x >= a.clear_from) return clear_rest<F32>(a, q_starts);
    constexpr int KD = D / 4, NT = D / 16;                 // elements of a lane's key part; column tiles of the values
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int d = FULL ? D : a.d;
    // pieces go round the eight chiplets (workgroup id modulo 8); the head groups of a piece, whose scales share cache lines,
    // follow each other on one chiplet
    const int at = (int)(blockIdx.x >> 3) / a.plan.groups * 8 + (int)(blockIdx.x & 7u), hg = (int)(blockIdx.x >> 3) % a.plan.groups;
    const Pieces pieces(a, q_starts, kv_lens, at, false);
    const int b = pieces.b;
    if (b >= a.B) return;
    const int h = hg * a.plan.waves + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (h >= a.H) return;
    const Sequence seq = pieces.seq;
    const int n_q = min(seq.n_q, a.max_q);
    const Steps steps(a, seq, 0, n_q - 1, kRows16Step);
    const bool alone = pieces.count == 1;                  // no partial results
    const int n0 = alone ? 0 : (at - pieces.first) * pieces.steps, n1 = alone ? steps.total : min(n0 + pieces.steps, steps.total);

    // ---- pages of a step, and what a lane loads of it, as offsets from the group's first slot.
    // Pages and their scales are the same for the whole wave, but they come through vector loads like the rest: those return
    // in order, so that waiting for one of them does not wait for what was asked for after it.
    struct Ahead {
        int first, offset[2];
        uint32_t page;                                     // lanes 0-31: of the first group, the others: of the second
    };
    const bool second = lane >= 32;
    const GlobalBytes table = scalar_base(page_table, (uint64_t)b * a.max_pages * 4), k_scale = scalar_base(k_global, 0), v_scale = scalar_base(v_global, 0);
    auto look_up = [&](int n, int to) {
        Ahead p;
        p.first = steps.first_token(min(n, to - 1), kRows16Step);
        uint32_t at[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {  // (a group past the length is masked; it may be past the table: the step's first group stands in)
            const int token = p.first + 16 * x < seq.len ? p.first + 16 * x : p.first;
            at[x] = a.by_page.small((uint32_t)token);
            p.offset[x] = token - (int)at[x] * a.page_tokens;
        }
        p.page = load_at<uint32_t>(table, 4u * (second ? at[1] : at[0]));
        return p;
    };
    const uint32_t token_codes = a.token_codes, token_scales = a.token_scales;
    const uint32_t head_codes = (uint32_t)h * (uint32_t)(d >> 1), head_scales = (uint32_t)h * (uint32_t)(d >> 4);
    constexpr uint32_t kZero = 0x0Cu;                      // (of a byte permutation: zero)
    constexpr int KB = D / 64;                             // blocks of a lane's key part
    // (lanes of elements from d on load the row's first ones: the queries are zero there, and those sums are not stored)
    uint32_t k_at[KB], ks_at[KB], ks_pick[KB];      // offsets, and the scales' bytes in their words (twice, for both halves of a register)
#pragma unroll
    for (int c = 0; c < KB; ++c) {
        const uint32_t blk = FULL || 16 * (g * KB + c) < d ? g * KB + c : 0;
        k_at[c] = r * token_codes + head_codes + 8u * blk;
        const uint32_t at = r * token_scales + head_scales + blk;
        ks_at[c] = at & ~3u;
        ks_pick[c] = (at & 3u) * 0x10001u | kZero << 8 | kZero << 24;
    }
    const int v_element = FULL || r * NT < d ? r * NT : 0;                   // the lane's elements of a value row
    const uint32_t v_shift = D == 64 ? (uint32_t)(v_element & 4) * 4u : 0u;
    uint32_t v_at[4], vs_at[4], vs_pick[2];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        v_at[t] = (4 * g + t) * token_codes + head_codes + ((uint32_t)(v_element >> 1) & ~3u);
        const uint32_t at = (4 * g + t) * token_scales + head_scales + (uint32_t)(v_element >> 4);
        vs_at[t] = at & ~3u;
        if (t & 1) vs_pick[t >> 1] |= ((at & 3u) + 4u) << 16 | kZero << 24;
        else vs_pick[t >> 1] = (at & 3u) | kZero << 8;
    }
    uint32_t mean_at = ((uint32_t)(r * a.H + h) * 2u) & ~3u;
    const uint32_t mean_shift = ((uint32_t)(r * a.H + h) & 1u) * 16u;
    // FULL: the scales of the step's 32 tokens are loaded once, a lane taking word lane_word of token lane_token (and the next
    // one), the means a lane each, and handed from lane to lane: a lane needs the word with its blocks of token r (+ 16), and
    // that with block r D / 256 of its eight tokens (times four: the exchange counts bytes)
    constexpr int kTokenLanes = D == 64 ? 1 : 2;
    const int lane_token = D == 64 ? lane & 31 : lane >> 1;
    uint32_t scales_at = (lane_token & 15) * token_scales + head_scales + (D == 64 ? 0u : 4u * (lane & 1) * Step<D, FULL>::SW);
    const uint32_t ks_from = 4u * (r * kTokenLanes + (D == 64 ? 0 : g >> 1)), vs_from = 4u * (4 * g * kTokenLanes + (D == 64 ? 0 : r >> 3));
    auto from_lane = [](uint32_t lane4, uint32_t v) { return (uint32_t)__builtin_amdgcn_ds_bpermute((int)lane4, (int)v); };
    auto as_loaded = [](uint32_t &v) { asm volatile("" : "+v"(v)); };
    // fetches the step whose pages were looked up, and looks up those of step n (or of the last one, to - 1)
    auto fetch = [&](Ahead &p, Step<D, FULL> &s, int n, int to) {
        as_loaded(p.page);
        uint32_t pages[2] = {(uint32_t)__builtin_amdgcn_readfirstlane((int)p.page), (uint32_t)__builtin_amdgcn_readlane((int)p.page, 32)};
        const Ahead now = p;
        p = look_up(n, to);
        // (offsets are widened where they are used: widened once in front of the loop, they would no longer be known to have 32 bits)
        if constexpr (FULL) as_loaded(scales_at);
        as_loaded(mean_at);
#pragma unroll
        for (int c = 0; c < KB; ++c) {
            if (!FULL || c == 0) as_loaded(k_at[c]);
            if constexpr (!FULL) as_loaded(ks_at[c]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            as_loaded(v_at[t]);
            if constexpr (!FULL) as_loaded(vs_at[t]);
        }
        s.first = now.first;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            s.valid[x] = pages[x] < (uint32_t)a.n_pages;
            pages[x] = s.valid[x] ? pages[x] : 0u;
        }
        const Slots both[2] = {Slots(a, pages[0], now.offset[0]), Slots(a, pages[1], now.offset[1])};
        const uint32_t page4 = 4u * (second ? pages[1] : pages[0]);
        s.kg = load_at<uint32_t>(k_scale, page4);
        s.vg = load_at<uint32_t>(v_scale, page4);
        if constexpr (FULL) {
            const GlobalBytes ks = lane_token < 16 ? both[0].k_scales : both[1].k_scales, vs = lane_token < 16 ? both[0].v_scales : both[1].v_scales;
#pragma unroll
            for (int c = 0; c < Step<D, FULL>::SW; ++c) {
                s.ks[0][c] = load_at<uint32_t>(ks, scales_at + 4u * c);
                s.vs[c] = load_at<uint32_t>(vs, scales_at + 4u * c);
            }
            if constexpr (SMOOTH) s.mean[0] = load_at<uint32_t>((lane & 16) ? both[1].k_mean : both[0].k_mean, mean_at);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const Slots &at = both[x];
            if constexpr (!FULL) {
#pragma unroll
                for (int c = 0; c < KB; ++c) s.ks[x][c] = load_at<uint32_t>(at.k_scales, ks_at[c]);
                if constexpr (SMOOTH) s.mean[x] = load_at<uint32_t>(at.k_mean, mean_at);
            }
            if constexpr (FULL && D >= 128) {
#pragma unroll
                for (int c = 0; c < KB; c += 2) {
                    const uint4v w = load_at<uint4v>(at.k_codes, k_at[0] + 8u * c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s.k[x][2 * c + i] = w[i];
                }
            } else {
#pragma unroll
                for (int c = 0; c < KB; ++c) {
                    const uint2v w = load_at<uint2v>(at.k_codes, k_at[c]);
                    s.k[x][2 * c] = w.x; s.k[x][2 * c + 1] = w.y;
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int m = 4 * x + t;
                if constexpr (D < 256) s.v[m] = load_at<uint32_t>(at.v_codes, v_at[t]);
                else {
                    const uint2v w = load_at<uint2v>(at.v_codes, v_at[t]);
                    s.v[m] = w.x;
                    s.v_hi[m] = w.y;
                }
                if constexpr (!FULL) s.vs[m] = load_at<uint32_t>(at.v_scales, vs_at[t]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);                 // (the loads stay in front of what follows)
    };

    // the first step's loads go out before the queries are read
    Step<D, FULL> sa, sb;
    Ahead ahead = {};
    if (n0 < n1) {
        ahead = look_up(n0, n1);
        fetch(ahead, sa, n0 + 1, n1);
    }

    // ---- queries
    const int i = r / a.G, head = h * a.G + (r - i * a.G);
    const bool row = i < n_q;
    const Sight sight(a, seq.position(a, i));
    const int64_t query = (int64_t)seq.start + i;
    half8v q[KD / 8];
    float factor, sum_q;                                   // score = (S + (mean / g_k) sum_q) factor g_k, base 2
    {
        uint4v w[KD / 8];
        float amax = 0.0f, sum = 0.0f;
#pragma unroll
        for (int c = 0; c < KD / 8; ++c) {
            const int e = g * KD + 8 * c;
            w[c] = uint4v{0u, 0u, 0u, 0u};
            if (row && e < d) w[c] = *(const uint4v *)(a.q + query * a.ldq + (int64_t)head * d + e);
        }
#pragma unroll
        for (int c = 0; c < KD / 8; ++c) amax = absmax8(w[c], amax);
        amax = fmaxf(amax, __shfl_xor(amax, 16, 64));
        amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
        const int e = row_exponent(amax);
#pragma unroll
        for (int c = 0; c < KD / 8; ++c) {
            q[c] = query_pairs(w[c], e);
            if constexpr (SMOOTH) sum = sum8(w[c], e, sum);
        }
        factor = __builtin_amdgcn_ldexpf(a.scale, -e);
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        sum_q = g == 0 ? sum : 0.0f;       // (the outer product has four terms, three of them zero)
    }

    float m = kLowest, ref = kLowest, l = 0.0f;            // ref: the r of a weight
    Units units = {kNoUnit, kNoUnit};
    constexpr uint32_t kNoLowest = 0x10000u;
    uint32_t lowest = kNoLowest;                           // lowest exponent that the unit holds for (none: not the first walk)
    int pass = 0, again_from = 0x7FFFFFFF, again_to = 0;   // walks over the steps; those with a page for the next walk
    float4v o[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) o[j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    // (what a step loaded is used as it is where it is taken, and no earlier: folded into the turn before, the first shift
    //  or mask of a loaded value would wait for all of them there)
    auto take = [&](Step<D, FULL> &s, int n) {
        float x[8];
        as_loaded(s.kg), as_loaded(s.vg);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int c = 0; c < Step<D, FULL>::KW; ++c) as_loaded(s.k[t][c]);
            if constexpr (!FULL) {
#pragma unroll
                for (int c = 0; c < KB; ++c) as_loaded(s.ks[t][c]);
                if constexpr (SMOOTH) as_loaded(s.mean[t]);
            }
        }
        uint32_t kw[2], vw[8];                                 // FULL: words with this lane's scales
        float mean[2] = {0.0f, 0.0f};
        if constexpr (FULL) {
#pragma unroll
            for (int c = 0; c < Step<D, FULL>::SW; ++c) as_loaded(s.ks[0][c]), as_loaded(s.vs[c]);
            if constexpr (SMOOTH) as_loaded(s.mean[0]);
            auto word = [&](const uint32_t (&v)[Step<D, FULL>::SW], uint32_t from, bool odd) {
                const uint32_t w = from_lane(from, v[0]);
                if constexpr (D < 256) return w;
                else {
                    const uint32_t w1 = from_lane(from, v[1]);         // (every lane takes part in both)
                    return odd ? w1 : w;
                }
            };
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                kw[t] = word(s.ks[0], ks_from + 64u * kTokenLanes * t, g & 1);
                if constexpr (SMOOTH) mean[t] = __uint_as_float(from_lane(4u * (16 * t + r), s.mean[0] >> mean_shift << 16));
            }
#pragma unroll
            for (int t = 0; t < 8; ++t) vw[t] = word(s.vs, vs_from + 4u * kTokenLanes * (16 * (t >> 2) + (t & 3)), (r >> 2) & 1);
        } else if constexpr (SMOOTH) {
#pragma unroll
            for (int t = 0; t < 2; ++t) mean[t] = __uint_as_float(s.mean[t] >> mean_shift << 16);
        }
        // of the two pages: scale, its inverse (keys), logarithm and inverse (values)
        auto of_pages = [](float v, float (&two)[2]) {
            two[0] = __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v)));
            two[1] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 32));
        };
        const float kg = __uint_as_float(s.kg), vg = __uint_as_float(s.vg);        // (of a page that is not in use, anything)
        float f[2], inv_k[2], log_v[2], inv_v[2];
        of_pages(kg, f);
        if constexpr (SMOOTH) of_pages(__builtin_amdgcn_rcpf(kg), inv_k);
        of_pages(__builtin_amdgcn_logf(vg), log_v);
        of_pages(__builtin_amdgcn_rcpf(vg), inv_v);
        const bool known = __ballot((s.vg >> 23) - lowest > (uint32_t)(kUnitHigh - kUnitLow)) == 0ull;         // (the unit holds for both pages)
        auto key_word = [&](int t, int c) {
            if constexpr (FULL) return kw[t];
            else return s.ks[t][c];
        };
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float4v acc = {0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (SMOOTH)
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(mean[t] * inv_k[t], sum_q, acc, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < KD / 8; ++c) {             // block of the lane's word c: c / 2
                const half2v sk = scale_pair(__builtin_amdgcn_perm(0u, key_word(t, c >> 1), ks_pick[c >> 1]));
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_codes(s.k[t][c], sk), q[c], acc, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * t + e] = acc[e] * (factor * f[t]);
        }
        // tokens that some row does not see (the same for the whole wave)
        const bool masked = !(s.valid[0] & s.valid[1]) || s.first + kRows16Step - 1 > seq.p0 ||
                            (a.window > 0 && s.first <= seq.position(a, n_q - 1) - a.window);
        bool moved = false;
        if (masked | !known) {
            uint32_t left = 0u;                                // pages of which some row sees some token
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (s.valid[t] & group_seen(s.first + 16 * t, seq.p0, seq.position(a, n_q - 1), a.window, a.sink)) left |= 1u << t;
            if (masked) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = s.first + 16 * (e >> 2) + 4 * g + (e & 3);
                    x[e] = (s.valid[e >> 2] & sight.of(j)) ? x[e] : -__builtin_inff();
                }
            }
            // the unit of the pages: it moves in front of the step, and a page that is far from the other one waits for another walk
            if (!known | (left != 3u)) {
                const uint32_t ev = scale_exponent((uint32_t)__builtin_amdgcn_readfirstlane((int)s.vg)) | scale_exponent((uint32_t)__builtin_amdgcn_readlane((int)s.vg, 32)) << 8;
                const int before = units.now;
                if (__ballot(m > kLowest) != 0ull) units.top = max(units.top, before);        // (it has been used)
                const uint32_t mine = units.enter<2>(ev, left, pass);
                if (left != 0u) again_from = min(again_from, n), again_to = n + 1;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    units.page((int)(ev >> 8 * t & 255u), log_v[t], inv_v[t]);
                    log_v[t] = (mine >> t & 1u) != 0u ? log_v[t] : -__builtin_inff();
                    inv_v[t] = (mine >> t & 1u) != 0u ? inv_v[t] : 0.0f;
                }
                moved = units.now != before;
                lowest = pass == 0 ? (uint32_t)(units.now + kUnitLow) : kNoLowest;
            }
        }
        const float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (__ballot(top > m + kAbove) != 0ull || moved) {
            float t = fmaxf(top, __shfl_xor(top, 16, 64));
            t = fmaxf(t, __shfl_xor(t, 32, 64));
            m = fmaxf(floorf(t - kBelow), m);
            const float to = m + (float)(units.now - kUnitBias), f = __builtin_amdgcn_exp2f(ref - to);
            l = moved_sum(l, ref, to);
            ref = to;
#pragma unroll
            for (int j = 0; j < NT; ++j) o[j] *= f;
        }
        half8v w, w_low;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float sum = 0.0f;
            const float add = log_v[t] - ref;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = __builtin_amdgcn_exp2f(x[4 * t + e] + add);
                sum += v;
                w[4 * t + e] = (_Float16)v;
                if constexpr (F32) w_low[4 * t + e] = (_Float16)(v - (float)w[4 * t + e]);
            }
            l = __builtin_fmaf(sum, inv_v[t], l);
        }
        asm volatile("" : "+v"(l));                            // (here: put off, the weights would wait for it in registers)
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            as_loaded(s.v[t]);
            if constexpr (!FULL) {
                as_loaded(s.vs[t]);
                vw[t] = s.vs[t];
            }
            if constexpr (D == 256) as_loaded(s.v_hi[t]);
        }
        half2v sv[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) sv[t] = scale_pair(__builtin_amdgcn_perm(vw[2 * t + 1], vw[2 * t], vs_pick[t & 1]));
        // nibbles of two tokens side by side: byte k of `even` holds element 2k of both, of `odd` element 2k + 1
        auto half_row = [&](const uint32_t (&v)[8], auto first_column) {
            constexpr int first = decltype(first_column)::value;
            uint32_t even[4], odd[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t u = D == 64 ? v[2 * t] >> v_shift : v[2 * t], n = D == 64 ? v[2 * t + 1] >> v_shift : v[2 * t + 1];
                even[t] = (u & 0x0F0F0F0Fu) | ((n << 4) & 0xF0F0F0F0u);
                odd[t] = ((u >> 4) & 0x0F0F0F0Fu) | (n & 0xF0F0F0F0u);
            }
            auto column = [&](int j, const uint32_t (&e)[4], auto byte) {
                constexpr int BYTE = decltype(byte)::value;
                const half8v c = join8(code_pair<BYTE>(e[0]) * sv[0], code_pair<BYTE>(e[1]) * sv[1], code_pair<BYTE>(e[2]) * sv[2], code_pair<BYTE>(e[3]) * sv[3]);
                o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c, w, o[j], 0, 0, 0);
                if constexpr (F32) o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c, w_low, o[j], 0, 0, 0);
            };
            column(first, even, std::integral_constant<int, 0>());
            column(first + 1, odd, std::integral_constant<int, 0>());
            column(first + 2, even, std::integral_constant<int, 1>());
            column(first + 3, odd, std::integral_constant<int, 1>());
            if constexpr (D > 64) {
                column(first + 4, even, std::integral_constant<int, 2>());
                column(first + 5, odd, std::integral_constant<int, 2>());
                column(first + 6, even, std::integral_constant<int, 3>());
                column(first + 7, odd, std::integral_constant<int, 3>());
            }
        };
        half_row(s.v, std::integral_constant<int, 0>());
        if constexpr (D == 256) half_row(s.v_hi, std::integral_constant<int, 8>());
    };

    // two steps a turn, so that neither is copied; what is fetched past the last step is the last step again.  Pages that a walk
    // leaves out are taken by another one over the steps that have some.
    for (int from = n0, to = n1; from < to; ++pass) {
        __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0): the turns count their own loads alone
        if (pass == 0) {                                   // (the unit of the first page, which most first steps find to hold)
            units.now = max((int)scale_exponent((uint32_t)__builtin_amdgcn_readfirstlane((int)sa.vg)), kUnitLeast);
            lowest = (uint32_t)(units.now + kUnitLow);
        }
        for (int n = from; n < to; n += 2) {
            fetch(ahead, sb, n + 2, to);
            take(sa, n);
            if (n + 1 >= to) break;
            fetch(ahead, sa, n + 3, to);
            take(sb, n + 1);
        }
        from = again_from, to = again_to;
        again_from = 0x7FFFFFFF, again_to = 0, lowest = kNoLowest;
        if (from < to) {
            ahead = look_up(from, to);
            fetch(ahead, sa, from + 1, to);
        }
    }

    // ---- the row's sum, and the result: element (4 g + e) NT + j of row r stands in o[j][e]
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (!row) return;
    const int64_t out_row = query * a.Hq + head;
    if (alone) {
        const float inv = inverse_sum(l);
        if (a.lse && g == 0) a.lse[out_row] = log_sum(ref, l);
        const int64_t at = query * a.ldo + (int64_t)head * d;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int first = (4 * g + e) * NT;
            if (!FULL && first >= d) continue;
#pragma unroll
            for (int j = 0; j < NT; j += 4) {
                if constexpr (F32)
                    *(float4v *)((float *)a.out + at + first + j) = float4v{o[j][e] * inv, o[j + 1][e] * inv, o[j + 2][e] * inv, o[j + 3][e] * inv};
                else
                    *(uint2v *)((uint16_t *)a.out + at + first + j) = uint2v{pack_bf16x2(o[j][e] * inv, o[j + 1][e] * inv), pack_bf16x2(o[j + 2][e] * inv, o[j + 3][e] * inv)};
            }
        }
        return;
    }
    const int64_t part = ((int64_t)at * a.max_q + i) * a.Hq + head;
    if (g == 0) a.part_ml[part] = float2{ref, l};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int first = (4 * g + e) * NT;
        if (!FULL && first >= d) continue;
#pragma unroll
        for (int j = 0; j < NT; j += 4)
            *(float4v *)(a.part_o + part * d + first + j) = float4v{o[j][e], o[j + 1][e], o[j + 2][e], o[j + 3][e]};
    }
}

template <int D>
static void launch_rows16(AttentionArgs a, const KvAttention &k, hipStream_t s)
{
    const int64_t pieces = a.plan.pieces > 1 ? a.plan.pieces + a.B : a.B;
    const dim3 grid(attention_grid(a, k, (unsigned)(((pieces + 7) >> 3 << 3) * a.plan.groups))), block((unsigned)(64 * a.plan.waves));
    auto go = [&](auto kernel) { kernel<<<grid, block, 0, s>>>(a, k.page_table, k.kv_lens, k.q_starts, k.cache.k_global, k.cache.v_global); };
    auto smooth = [&](auto full) {
        constexpr bool FULL = decltype(full)::value;
        if (a.k_mean) k.out_f32 ? go(attention_rows16_kernel<D, FULL, true, true>) : go(attention_rows16_kernel<D, FULL, true, false>);
        else k.out_f32 ? go(attention_rows16_kernel<D, FULL, false, true>) : go(attention_rows16_kernel<D, FULL, false, false>);
    };
    if (a.d == D) smooth(std::true_type());
    else smooth(std::false_type());
}

hipError_t launch_attention_rows16(AttentionArgs a, const KvAttention &k, hipStream_t s)
{
    if (a.d <= 64) launch_rows16<64>(a, k, s);
    else if (a.d <= 128) launch_rows16<128>(a, k, s);
    else launch_rows16<256>(a, k, s);
    return hipGetLastError();
}

}  // namespace nvfp4
