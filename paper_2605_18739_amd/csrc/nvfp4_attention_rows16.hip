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
// FULL: d = D.  Otherwise elements from d on load from the row's start and take a scale of zero.
// The loop's loads are whole aligned words without branches, so that the compiler can count them: a step's loads are in
// flight while the one before is multiplied, and the pages of the step behind it are looked up.  Scale bytes and means come
// as the word that holds them (slots start at multiples of sixteen rows, so which byte it is does not change from step to
// step, and the planes' sizes are multiples of sixteen bytes: no word reaches past the end).
template <int D, bool FULL>
struct Step {
    static constexpr int KW = D / 32;                      // key words of a lane
    static constexpr int KS = FULL ? 1 : D / 64;           // words with scale bytes of its blocks
    uint32_t k[2][KW], ks[2][KS], v[8], v_hi[D == 256 ? 8 : 1], vs[8], mean[2];
    uint32_t kg[2], vg[2];                                 // the pages' scales (fp32)
    int first;                                             // the step's first token
    bool valid[2];                                         // the group of sixteen lies on a page of the cache
};

template <int D, bool FULL, bool SMOOTH, bool F32>
__global__ __launch_bounds__(64 * kRows16Heads) void attention_rows16_kernel(const AttentionArgs a, const int32_t *__restrict__ page_table,
                                                               const int32_t *__restrict__ kv_lens, const int32_t *__restrict__ q_starts,
                                                               const float *__restrict__ k_global, const float *__restrict__ v_global)
{
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
    const Sequence seq(a, q_starts, kv_lens, b);
    const int n_q = min(seq.n_q, a.max_q);
    const Steps steps(a, seq, 0, n_q - 1, kRows16Step);
    const bool alone = pieces.count == 1;                  // no partial results
    const int n0 = alone ? 0 : (at - pieces.first) * pieces.steps, n1 = alone ? steps.total : min(n0 + pieces.steps, steps.total);

    // ---- pages of a step, and what a lane loads of it, as offsets from the group's first slot.
    // Pages and their scales are the same for the whole wave, but they come through vector loads like the rest: those return
    // in order, so that waiting for one of them does not wait for what was asked for after it.
    uint32_t zero;                                         // (an offset that the compiler takes for a lane's own)
    asm("v_mov_b32 %0, 0" : "=v"(zero));
    struct Ahead {
        int first, offset[2];
        uint32_t page[2];
    };
    auto look_up = [&](int n) {
        Ahead p;
        p.first = steps.first_token(min(n, n1 - 1), kRows16Step);
#pragma unroll
        for (int x = 0; x < 2; ++x) {  // (a group past the length is masked; it may be past the table: the step's first group stands in)
            const int token = p.first + 16 * x < seq.len ? p.first + 16 * x : p.first;
            const int at = (int)a.by_page.small((uint32_t)token);
            p.offset[x] = token - at * a.page_tokens;
            p.page[x] = ((const uint32_t *)page_table)[(int64_t)b * a.max_pages + at + zero];
        }
        return p;
    };
    const uint32_t token_codes = (uint32_t)a.H * (uint32_t)(d >> 1), token_scales = (uint32_t)a.H * (uint32_t)(d >> 4);
    const uint32_t head_codes = (uint32_t)h * (uint32_t)(d >> 1), head_scales = (uint32_t)h * (uint32_t)(d >> 4);
    constexpr uint32_t kOutside = 0x7FFFFF00u;             // (loads behind the sixteen tokens give zeros)
    constexpr uint32_t kZero = 0x0Cu;                      // (of a byte permutation: zero)
    constexpr int KB = D / 64;                             // blocks of a lane's key part
    uint32_t k_at[KB], ks_at[Step<D, FULL>::KS], ks_pick[KB];      // offsets, and the scales' bytes in their words (twice, for both halves of a register)
#pragma unroll
    for (int c = 0; c < KB; ++c) {
        const int blk = g * KB + c;
        const bool in = FULL || 16 * blk < d;
        k_at[c] = in ? r * token_codes + head_codes + 8u * blk : kOutside;
        const uint32_t at = r * token_scales + head_scales + blk;
        if (!FULL || c == 0) ks_at[FULL ? 0 : c] = in ? at & ~3u : kOutside;
        ks_pick[c] = (at & 3u) * 0x10001u | kZero << 8 | kZero << 24;
    }
    const int v_element = r * NT;                          // the lane's elements of a value row
    const bool v_in = FULL || v_element < d;
    const uint32_t v_at = v_in ? 4 * g * token_codes + head_codes + ((uint32_t)(v_element >> 1) & ~3u) : kOutside;
    const uint32_t v_shift = D == 64 ? (uint32_t)(v_element & 4) * 4u : 0u;
    uint32_t vs_at[4], vs_pick[2];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t at = (4 * g + t) * token_scales + head_scales + (uint32_t)(v_element >> 4);
        vs_at[t] = v_in ? at & ~3u : kOutside;
        if (t & 1) vs_pick[t >> 1] |= ((at & 3u) + 4u) << 16 | kZero << 24;
        else vs_pick[t >> 1] = (at & 3u) | kZero << 8;
    }
    const uint32_t mean_at = ((uint32_t)(r * a.H + h) * 2u) & ~3u, mean_shift = ((uint32_t)(r * a.H + h) & 1u) * 16u;
    auto as_loaded = [](uint32_t &v) { asm volatile("" : "+v"(v)); };
    // sixteen tokens of a plane, as a buffer: addresses are a scalar base and a lane's 32-bit offset
    auto group = [](const void *base, int64_t at, uint32_t bytes) {
        return __builtin_amdgcn_make_buffer_rsrc((void *)((const uint8_t *)base + at), 0, (int)bytes, 0x00020000);
    };
    // fetches the step whose pages were looked up, and looks up those of step n
    auto fetch = [&](Ahead &p, Step<D, FULL> &s, int n) {
        uint32_t pages[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            as_loaded(p.page[x]);
            pages[x] = (uint32_t)__builtin_amdgcn_readfirstlane((int)p.page[x]);
        }
        const Ahead now = p;
        p = look_up(n);
        s.first = now.first;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            s.valid[x] = pages[x] < (uint32_t)a.n_pages;
            const uint32_t page = s.valid[x] ? pages[x] : 0u;
            s.kg[x] = ((const uint32_t *)k_global)[page + zero];
            s.vg[x] = ((const uint32_t *)v_global)[page + zero];
            const int64_t row = ((int64_t)page * a.page_tokens + now.offset[x]) * a.H;
            const __amdgpu_buffer_rsrc_t kc = group(a.k_codes, row * (d >> 1), 16u * token_codes), vc = group(a.v_codes, row * (d >> 1), 16u * token_codes);
            const __amdgpu_buffer_rsrc_t ksc = group(a.k_scales, row * (d >> 4), 16u * token_scales), vsc = group(a.v_scales, row * (d >> 4), 16u * token_scales);
            if constexpr (FULL && D >= 128) {
#pragma unroll
                for (int c = 0; c < KB; c += 2) {
                    const uint4v w = __builtin_amdgcn_raw_buffer_load_b128(kc, k_at[c], 0, 0);
                    s.k[x][2 * c] = w.x; s.k[x][2 * c + 1] = w.y; s.k[x][2 * c + 2] = w.z; s.k[x][2 * c + 3] = w.w;
                }
            } else {
#pragma unroll
                for (int c = 0; c < KB; ++c) {
                    const uint2v w = __builtin_amdgcn_raw_buffer_load_b64(kc, k_at[c], 0, 0);
                    s.k[x][2 * c] = w.x; s.k[x][2 * c + 1] = w.y;
                }
            }
#pragma unroll
            for (int c = 0; c < Step<D, FULL>::KS; ++c) s.ks[x][c] = __builtin_amdgcn_raw_buffer_load_b32(ksc, ks_at[c], 0, 0);
            if constexpr (SMOOTH) s.mean[x] = __builtin_amdgcn_raw_buffer_load_b32(group(a.k_mean, 2 * row, 32u * (uint32_t)a.H), mean_at, 0, 0);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int m = 4 * x + t;
                if constexpr (D < 256) s.v[m] = __builtin_amdgcn_raw_buffer_load_b32(vc, v_at, t * (int)token_codes, 0);
                else {
                    const uint2v w = __builtin_amdgcn_raw_buffer_load_b64(vc, v_at, t * (int)token_codes, 0);
                    s.v[m] = w.x;
                    s.v_hi[m] = w.y;
                }
                s.vs[m] = __builtin_amdgcn_raw_buffer_load_b32(vsc, vs_at[t], 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);                 // (the loads stay in front of what follows)
    };

    // the first step's loads go out before the queries are read
    Step<D, FULL> sa, sb;
    Ahead ahead = {};
    if (n0 < n1) {
        ahead = look_up(n0);
        fetch(ahead, sa, n0 + 1);
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
        for (int c = 0; c < KD / 8; ++c) {
            amax = absmax8(w[c], amax);
            if constexpr (SMOOTH) sum = sum8(w[c], sum);
        }
        amax = fmaxf(amax, __shfl_xor(amax, 16, 64));
        amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
        const int e = row_exponent(amax);
#pragma unroll
        for (int c = 0; c < KD / 8; ++c) q[c] = query_pairs(w[c], e);
        factor = __builtin_amdgcn_ldexpf(a.scale, -e);
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        sum_q = g == 0 ? __builtin_amdgcn_ldexpf(sum, e) : 0.0f;       // (the outer product has four terms, three of them zero)
    }

    float m = kLowest, l = 0.0f;
    float4v o[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) o[j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    // (what a step loaded is used as it is where it is taken, and no earlier: folded into the turn before, the first shift
    //  or mask of a loaded value would wait for all of them there)
    auto take = [&](Step<D, FULL> &s) {
        float x[8];
        float inv_v[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int c = 0; c < Step<D, FULL>::KW; ++c) as_loaded(s.k[t][c]);
#pragma unroll
            for (int c = 0; c < Step<D, FULL>::KS; ++c) as_loaded(s.ks[t][c]);
            if constexpr (SMOOTH) as_loaded(s.mean[t]);
            as_loaded(s.kg[t]);
            as_loaded(s.vg[t]);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float kg = __uint_as_float(s.kg[t]), vg = __uint_as_float(s.vg[t]);
            float4v acc = {0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (SMOOTH)
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((s.mean[t] >> mean_shift) << 16) * __builtin_amdgcn_rcpf(kg), sum_q, acc, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < KD / 8; ++c) {             // block of the lane's word c: c / 2
                const half2v sk = scale_pair(__builtin_amdgcn_perm(0u, s.ks[t][FULL ? 0 : c >> 1], ks_pick[c >> 1]));
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_codes(s.k[t][c], sk), q[c], acc, 0, 0, 0);
            }
            const float log_v = __builtin_amdgcn_logf(vg), f = factor * kg;
            inv_v[t] = __builtin_amdgcn_rcpf(vg);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * t + e] = __builtin_fmaf(acc[e], f, log_v);
        }
        // tokens that some row does not see (the same for the whole wave)
        const bool masked = !(s.valid[0] & s.valid[1]) || s.first + kRows16Step - 1 > seq.p0 ||
                            (a.window > 0 && s.first <= seq.position(a, n_q - 1) - a.window);
        if (masked) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = s.first + 16 * (e >> 2) + 4 * g + (e & 3);
                x[e] = (s.valid[e >> 2] & sight.of(j)) ? x[e] : -__builtin_inff();
            }
        }
        const float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (__ballot(top > m + kSlack) != 0ull) {
            float t = fmaxf(top, __shfl_xor(top, 16, 64));
            t = fmaxf(t, __shfl_xor(t, 32, 64));
            t = fmaxf(t, m);
            const float f = __builtin_amdgcn_exp2f(m - t);
            m = t;
            l *= f;
#pragma unroll
            for (int j = 0; j < NT; ++j) o[j] *= f;
        }
        half8v w, w_low;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = __builtin_amdgcn_exp2f(x[4 * t + e] - m);
                sum += v;
                w[4 * t + e] = (_Float16)v;
                if constexpr (F32) w_low[4 * t + e] = (_Float16)(v - (float)w[4 * t + e]);
            }
            l = __builtin_fmaf(sum, inv_v[t], l);
        }
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            as_loaded(s.v[t]);
            as_loaded(s.vs[t]);
            if constexpr (D == 256) as_loaded(s.v_hi[t]);
        }
        half2v sv[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) sv[t] = scale_pair(__builtin_amdgcn_perm(s.vs[2 * t + 1], s.vs[2 * t], vs_pick[t & 1]));
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

    // two steps a turn, so that neither is copied; what is fetched past the last step is the last step again
    __builtin_amdgcn_s_waitcnt(0x0F70);                    // vmcnt(0): the turns count their own loads alone
    for (int n = n0; n < n1; n += 2) {
        fetch(ahead, sb, n + 2);
        take(sa);
        if (n + 1 >= n1) break;
        fetch(ahead, sa, n + 3);
        take(sb);
    }

    // ---- the row's sum, and the result: element (4 g + e) NT + j of row r stands in o[j][e]
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (!row) return;
    const int64_t out_row = query * a.Hq + head;
    if (alone) {
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        if (a.lse && g == 0) a.lse[out_row] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -__builtin_inff();
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
    if (g == 0) a.part_ml[part] = float2{m, l};
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
static void launch_rows16(const AttentionArgs &a, const KvAttention &k, hipStream_t s)
{
    const int64_t pieces = a.plan.pieces > 1 ? a.plan.pieces + a.B : a.B;
    const dim3 grid((unsigned)(((pieces + 7) >> 3 << 3) * a.plan.groups)), block((unsigned)(64 * a.plan.waves));
    auto go = [&](auto kernel) { kernel<<<grid, block, 0, s>>>(a, k.page_table, k.kv_lens, k.q_starts, k.cache.k_global, k.cache.v_global); };
    auto smooth = [&](auto full) {
        constexpr bool FULL = decltype(full)::value;
        if (a.k_mean) k.out_f32 ? go(attention_rows16_kernel<D, FULL, true, true>) : go(attention_rows16_kernel<D, FULL, true, false>);
        else k.out_f32 ? go(attention_rows16_kernel<D, FULL, false, true>) : go(attention_rows16_kernel<D, FULL, false, false>);
    };
    if (a.d == D) smooth(std::true_type());
    else smooth(std::false_type());
}

hipError_t launch_attention_rows16(const AttentionArgs &a, const KvAttention &k, hipStream_t s)
{
    if (a.d <= 64) launch_rows16<64>(a, k, s);
    else if (a.d <= 128) launch_rows16<128>(a, k, s);
    else launch_rows16<256>(a, k, s);
    return hipGetLastError();
}

}  // namespace nvfp4
