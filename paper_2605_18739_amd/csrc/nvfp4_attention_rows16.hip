// Attention over the paged NVFP4 cache for at most sixteen (query, head) rows a cached head: single tokens and small
// groups of heads.  Bound by the cache's bytes: 0.5625 B an element of keys and of values.
#include "nvfp4_attention.h"

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
template <int D>
struct Step {
    static constexpr int KW = D / 32, VB = D / 32;         // key words of a lane; value bytes of a lane and token
    uint32_t k[2][KW], ks[2], v[8], v_hi[D == 256 ? 8 : 1], vs[8], mean[8];
    float kg[2], vg[2];                                    // the pages' scales
    int first;                                             // the step's first token
    uint32_t valid;                                        // bit x: group x lies on a page of the cache
};

template <int D, bool F32>
__global__ __launch_bounds__(512) void attention_rows16_kernel(const AttentionArgs a, const int32_t *__restrict__ page_table,
                                                               const int32_t *__restrict__ kv_lens, const int32_t *__restrict__ q_starts,
                                                               const float *__restrict__ k_global, const float *__restrict__ v_global)
{
    constexpr int KD = D / 4, NT = D / 16;                 // elements of a lane's key part; column tiles of the values
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    // neighbouring workgroups: the head groups of a piece, then the sequences
    int id = blockIdx.x;
    const int hg = id % a.plan.groups;
    id /= a.plan.groups;
    const int b = id % a.B, piece = id / a.B;
    const int h = hg * a.plan.waves + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (h >= a.H) return;
    const Sequence seq(a, q_starts, kv_lens, b);
    const int n_q = min(seq.n_q, a.max_q);
    if (n_q <= 0) return;
    const Steps steps(a, seq, 0, n_q - 1, kRows16Step);
    const int n0 = piece * a.plan.piece_steps, n1 = min(n0 + a.plan.piece_steps, steps.total);
    const bool alone = steps.total <= a.plan.piece_steps;  // this sequence has one piece: no partial results
    if (n0 >= n1 && piece > 0) return;

    // ---- queries
    const int i = r / a.G, head = h * a.G + (r - i * a.G);
    const bool row = i < n_q;
    const int p = seq.position(a, i);
    const int64_t query = (int64_t)seq.start + i;
    half8v q[KD / 8];
    float factor, sum_q;                                   // score = S factor (g_k) + mean sum_q, base 2
    {
        uint4v w[KD / 8];
        float amax = 0.0f, sum = 0.0f;
#pragma unroll
        for (int c = 0; c < KD / 8; ++c) {
            const int e = g * KD + 8 * c;
            w[c] = uint4v{0u, 0u, 0u, 0u};
            if (row && e < a.d) w[c] = *(const uint4v *)(a.q + query * a.ldq + (int64_t)head * a.d + e);
            amax = absmax8(w[c], amax);
            sum = sum8(w[c], sum);
        }
        amax = fmaxf(amax, __shfl_xor(amax, 16, 64));
        amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        const int e = row_exponent(amax);
#pragma unroll
        for (int c = 0; c < KD / 8; ++c) q[c] = query_pairs(w[c], e);
        factor = __builtin_amdgcn_ldexpf(a.scale, -e);
        sum_q = sum * a.scale;
    }

    // ---- what a lane loads of a step, as offsets from the row (group's first token, head h)
    const bool smooth = a.k_mean != nullptr;
    const uint32_t token_codes = (uint32_t)a.H * (uint32_t)(a.d >> 1), token_scales = (uint32_t)a.H * (uint32_t)(a.d >> 4);
    const uint32_t k_at = r * token_codes + g * (KD / 2), ks_at = r * token_scales + g * (KD / 16);
    const int v_element = r * NT;                          // the lane's elements of a value row
    const bool v_in = v_element < a.d;
    const uint32_t v_at = 4 * g * token_codes + (uint32_t)(v_element >> 1), vs_at = 4 * g * token_scales + (uint32_t)(v_element >> 4);
    auto fetch = [&](int n, Step<D> &s) {
        s.first = steps.first_token(n, kRows16Step);
        s.valid = 0u;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            // (a group past the length is masked; where it is past the table, the step's first group stands in)
            const int token = s.first + 16 * x < seq.len ? s.first + 16 * x : s.first;
            int offset;
            int page = page_of(a, page_table, b, token, offset);
            if (page >= 0) s.valid |= 1u << x;
            page = max(page, 0);
            s.kg[x] = k_global[page];
            s.vg[x] = v_global[page];
            const int64_t first_row = ((int64_t)page * a.page_tokens + offset) * a.H + h;
            const uint8_t *kc = a.k_codes + first_row * (a.d >> 1), *vc = a.v_codes + first_row * (a.d >> 1);
            const uint8_t *ksc = a.k_scales + first_row * (a.d >> 4), *vsc = a.v_scales + first_row * (a.d >> 4);
#pragma unroll
            for (int c = 0; c < Step<D>::KW; ++c) s.k[x][c] = 0u;
            s.ks[x] = 0u;
            // whole blocks of sixteen at a time: rows of d < D elements end behind one
            if (a.d == D) {
                if constexpr (D == 64) {
                    const uint2v w = *(const uint2v *)(kc + k_at);
                    s.k[x][0] = w.x; s.k[x][1] = w.y;
                    s.ks[x] = ksc[ks_at];
                } else {
#pragma unroll
                    for (int c = 0; c < KD / 32; ++c) {
                        const uint4v w = *(const uint4v *)(kc + k_at + 16 * c);
                        s.k[x][4 * c] = w.x; s.k[x][4 * c + 1] = w.y; s.k[x][4 * c + 2] = w.z; s.k[x][4 * c + 3] = w.w;
                    }
                    if constexpr (D == 128) s.ks[x] = *(const uint16_t *)(ksc + ks_at);
                    else s.ks[x] = *(const uint32_t *)(ksc + ks_at);
                }
            } else {
#pragma unroll
                for (int c = 0; c < KD / 16; ++c)
                    if (g * KD + 16 * c < a.d) {
                        s.k[x][2 * c] = *(const uint32_t *)(kc + k_at + 8 * c);
                        s.k[x][2 * c + 1] = *(const uint32_t *)(kc + k_at + 8 * c + 4);
                        s.ks[x] |= (uint32_t)ksc[ks_at + c] << (8 * c);
                    }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int m = 4 * x + t;
                s.v[m] = 0u;
                s.vs[m] = 0u;
                if constexpr (D == 256) s.v_hi[m] = 0u;
                if (v_in) {
                    const uint8_t *at = vc + v_at + t * token_codes;
                    if constexpr (D == 64) s.v[m] = *(const uint16_t *)at;
                    else s.v[m] = *(const uint32_t *)at;
                    if constexpr (D == 256) s.v_hi[m] = *(const uint32_t *)(at + 4);
                    s.vs[m] = vsc[vs_at + t * token_scales];
                }
                s.mean[m] = smooth ? (uint32_t)a.k_mean[first_row + (int64_t)((4 * g + t) * a.H)] : 0u;
            }
        }
    };

    float m = kLowest, l = 0.0f;
    float4v o[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) o[j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    auto take = [&](const Step<D> &s) {
        float x[8];
        float log_v[2], inv_v[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float4v acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < KD / 8; ++c) {
                // block of the lane's word c: c / 2
                const uint32_t sb = (s.ks[t] >> (8 * (c >> 1))) & 0xFFu;
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_codes(s.k[t][c], scale_pair(sb * 0x10001u)), q[c], acc, 0, 0, 0);
            }
            log_v[t] = __builtin_amdgcn_logf(s.vg[t]);
            inv_v[t] = __builtin_amdgcn_rcpf(s.vg[t]);
            const float f = factor * s.kg[t];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float mean = __uint_as_float(s.mean[4 * t + e] << 16);
                x[4 * t + e] = __builtin_fmaf(acc[e], f, __builtin_fmaf(mean, sum_q, log_v[t]));
            }
        }
        // tokens that some row does not see (the same for the whole wave)
        const bool masked = s.valid != 3u || s.first + kRows16Step - 1 > seq.p0 ||
                            (a.window > 0 && s.first <= seq.position(a, n_q - 1) - a.window);
        if (masked) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = s.first + 16 * (e >> 2) + 4 * g + (e & 3);
                x[e] = (((s.valid >> (e >> 2)) & 1u) != 0u && seen(a, j, p)) ? x[e] : -__builtin_inff();
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
        half2v sv[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) sv[t] = scale_pair(s.vs[2 * t] | (s.vs[2 * t + 1] << 16));
        // nibbles of two tokens side by side: byte k of `even` holds element 2k of both, of `odd` element 2k + 1
        auto half_row = [&](const uint32_t (&v)[8], int first) {
            uint32_t even[4], odd[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t u = v[2 * t], n = v[2 * t + 1];
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
        half_row(s.v, 0);
        if constexpr (D == 256) half_row(s.v_hi, 8);
    };

    if (n0 < n1) {
        Step<D> s, next;
        fetch(n0, s);
        for (int n = n0; n < n1; ++n) {
            if (n + 1 < n1) fetch(n + 1, next);
            take(s);
            s = next;
        }
    }

    // ---- the row's sum, and the result: element (4 g + e) NT + j of row r stands in o[j][e]
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (!row) return;
    const int64_t out_row = query * a.Hq + head;
    if (alone) {
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        if (a.lse && g == 0) a.lse[out_row] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -__builtin_inff();
        const int64_t at = query * a.ldo + (int64_t)head * a.d;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int first = (4 * g + e) * NT;
            if (first >= a.d) continue;
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
    const int64_t part = (int64_t)piece * a.total_q * a.Hq + out_row;
    if (g == 0) a.part_ml[part] = float2{m, l};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int first = (4 * g + e) * NT;
        if (first >= a.d) continue;
#pragma unroll
        for (int j = 0; j < NT; j += 4)
            *(float4v *)(a.part_o + part * a.d + first + j) = float4v{o[j][e], o[j + 1][e], o[j + 2][e], o[j + 3][e]};
    }
}

hipError_t launch_attention_rows16(const AttentionArgs &a, const KvAttention &k, hipStream_t s)
{
    const dim3 grid((unsigned)((int64_t)a.plan.groups * a.B * a.plan.pieces)), block((unsigned)(64 * a.plan.waves));
    auto go = [&](auto kernel) { kernel<<<grid, block, 0, s>>>(a, k.page_table, k.kv_lens, k.q_starts, k.cache.k_global, k.cache.v_global); };
    if (a.d <= 64) k.out_f32 ? go(attention_rows16_kernel<64, true>) : go(attention_rows16_kernel<64, false>);
    else if (a.d <= 128) k.out_f32 ? go(attention_rows16_kernel<128, true>) : go(attention_rows16_kernel<128, false>);
    else k.out_f32 ? go(attention_rows16_kernel<256, true>) : go(attention_rows16_kernel<256, false>);
    return hipGetLastError();
}

}  // namespace nvfp4
