// Attention over the paged NVFP4 cache for many rows (queries times the heads that share a cached head): chunks of a
// video, prompts.  Bound by the matrix pipes and the vector pipes' exponentials together.
#include "nvfp4_attention.h"

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
template <int D, int WAVES>
struct Tiles {
    static constexpr int kThreads = 64 * WAVES;
    static constexpr int kTasks = 4 * D / kThreads > 0 ? 4 * D / kThreads : 1;    // blocks of keys, and pieces of values, of a lane
    uint8_t k[2][kTileStep * D * 2];      // [token][D] f16
    uint8_t v[2][D * kTileStep * 2];      // [element][token] f16
    float mean[2][kTileStep];
    float kg[2][4], log_v[2][4], inv_v[2][4];       // of the four groups of sixteen tokens
    uint32_t valid[2][4];
};

template <int D>
__device__ __forceinline__ uint32_t k_place(int token, int chunk) { return (uint32_t)(token * (2 * D) + ((chunk ^ (token & (D / 8 - 1) & 15)) << 4)); }
__device__ __forceinline__ uint32_t v_place(int element, int chunk) { return (uint32_t)(element * (2 * kTileStep) + (((chunk ^ element ^ (element >> 3)) & 7) << 4)); }

template <int D, int WAVES, bool F32>
__global__ __launch_bounds__(64 * WAVES, D == 256 ? 1 : 2) void attention_tiles_kernel(const AttentionArgs a, const int32_t *__restrict__ page_table,
                                                                          const int32_t *__restrict__ kv_lens, const int32_t *__restrict__ q_starts,
                                                                          const float *__restrict__ k_global, const float *__restrict__ v_global)
{
    using Lds = Tiles<D, WAVES>;
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    Lds &lds = *reinterpret_cast<Lds *>(lds_bytes);
    constexpr int kThreads = Lds::kThreads, kTasks = Lds::kTasks, kRows = 32 * WAVES;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c32 = lane & 31, hi = lane >> 5;

    // workgroups that read the same tokens of the same head follow each other on one of the eight chiplets (each has an L2)
    int id = blockIdx.x, block, b, h, piece;
    {
        const int same = a.plan.groups, sets = a.B * a.H * a.plan.pieces, full = sets & ~7;
        int set;
        if (id < full * same) {
            set = id / (8 * same) * 8 + (id & 7);
            block = (id >> 3) % same;
        } else {
            id -= full * same;
            set = full + id / same;
            block = id % same;
        }
        h = set % a.H;
        set /= a.H;
        b = set % a.B;
        piece = set / a.B;
    }
    const Sequence seq(a, q_starts, kv_lens, b);
    const int n_q = min(seq.n_q, a.max_q), row0 = block * kRows;
    if (row0 >= n_q * a.G) return;
    const int i0 = row0 / a.G, i1 = min((row0 + kRows - 1) / a.G, n_q - 1);
    const Steps steps(a, seq, i0, i1, kTileStep);
    const int n0 = piece * a.plan.piece_steps, n1 = min(n0 + a.plan.piece_steps, steps.total);
    const bool alone = steps.total <= a.plan.piece_steps;
    if (n0 >= n1 && piece > 0) return;
    const bool smooth = a.k_mean != nullptr;

    // ---- queries of this wave's rows: lane holds row c32, elements 16 step + 8 hi .. + 7 of every k step
    const int my_row = row0 + 32 * wave + c32, i = my_row / a.G, head = h * a.G + (my_row - i * a.G);
    const bool row = i < n_q;
    const int p = seq.position(a, i);
    const int64_t query = (int64_t)seq.start + i;
    half8v q[D / 16];
    float factor, sum_q;
    {
        uint4v w[D / 16];
        float amax = 0.0f, sum = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            const int e = 16 * c + 8 * hi;
            w[c] = uint4v{0u, 0u, 0u, 0u};
            if (row && e < a.d) w[c] = *(const uint4v *)(a.q + query * a.ldq + (int64_t)head * a.d + e);
            amax = absmax8(w[c], amax);
            sum = sum8(w[c], sum);
        }
        amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
        sum += __shfl_xor(sum, 32, 64);
        const int e = row_exponent(amax);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) q[c] = query_pairs(w[c], e);
        factor = __builtin_amdgcn_ldexpf(a.scale, -e);
        sum_q = sum * a.scale;
    }

    // ---- this lane's share of a step: blocks of keys (token, block) and pieces of values (pair of tokens, eight elements)
    struct Share {
        uint2v k[kTasks];
        uint32_t ks[kTasks], v[kTasks][2], vs[kTasks];
        uint32_t mean;
        float kg, vg;
        uint32_t valid;
    };
    constexpr int NB = D / 16, NE = D / 8;
    // first slot of a token's group, times H: the row of its codes (a group past the length: the step's first one)
    auto group_slot = [&](int first, int group, bool &valid) {
        const int token = first + 16 * group < seq.len ? first + 16 * group : first;
        int offset;
        const int page = raw_page(a, page_table, b, token, offset);
        valid = (uint32_t)page < (uint32_t)a.n_pages;
        return (int64_t)(valid ? page : 0) * a.page_tokens + offset;
    };
    auto fetch = [&](int n, Share &s) {
        const int first = steps.first_token(n, kTileStep);
#pragma unroll
        for (int t = 0; t < kTasks; ++t) {
            const int task = tid + t * kThreads;
            s.k[t] = uint2v{0u, 0u};
            s.ks[t] = s.v[t][0] = s.v[t][1] = s.vs[t] = 0u;
            if (task < 4 * D) {
                bool valid;
                const int token = task / NB, blk = task % NB;
                if (16 * blk < a.d) {
                    const int64_t at = (group_slot(first, token >> 4, valid) + (token & 15)) * a.H + h;
                    const uint32_t *c = (const uint32_t *)(a.k_codes + at * (a.d >> 1)) + 2 * blk;
                    s.k[t] = *(const uint2v *)c;
                    s.ks[t] = a.k_scales[at * (a.d >> 4) + blk];
                }
                const int pair = task / NE, part = task % NE;
                if (8 * part < a.d) {
                    const int64_t at = (group_slot(first, pair >> 3, valid) + ((2 * pair) & 15)) * a.H + h;
                    const uint8_t *c = a.v_codes + at * (a.d >> 1) + 4 * part;
                    s.v[t][0] = *(const uint32_t *)c;
                    s.v[t][1] = *(const uint32_t *)(c + (int64_t)a.H * (a.d >> 1));
                    const uint8_t *sc = a.v_scales + at * (a.d >> 4) + (part >> 1);
                    s.vs[t] = (uint32_t)sc[0] | ((uint32_t)sc[(int64_t)a.H * (a.d >> 4)] << 16);
                }
            }
        }
        if (tid < kTileStep) {
            bool valid;
            const int64_t slot = group_slot(first, tid >> 4, valid);
            s.valid = valid;
            s.mean = smooth ? (uint32_t)a.k_mean[(slot + (tid & 15)) * a.H + h] : 0u;
            const int64_t page = slot / a.page_tokens;
            s.kg = k_global[page];
            s.vg = v_global[page];
        }
    };
    auto store = [&](const Share &s, int stage) {
#pragma unroll
        for (int t = 0; t < kTasks; ++t) {
            const int task = tid + t * kThreads;
            if (task < 4 * D) {
                const int token = task / NB, blk = task % NB;
                const half2v sk = scale_pair(s.ks[t] * 0x10001u);
                *(half8v *)(lds.k[stage] + k_place<D>(token, 2 * blk)) = eight_codes(s.k[t].x, sk);
                *(half8v *)(lds.k[stage] + k_place<D>(token, 2 * blk + 1)) = eight_codes(s.k[t].y, sk);
                const int pair = task / NE, part = task % NE;
                // nibbles of the two tokens side by side: byte j of `even` is element 2 j of both, of `odd` element 2 j + 1
                const uint32_t even = (s.v[t][0] & 0x0F0F0F0Fu) | ((s.v[t][1] << 4) & 0xF0F0F0F0u);
                const uint32_t odd = ((s.v[t][0] >> 4) & 0x0F0F0F0Fu) | (s.v[t][1] & 0xF0F0F0F0u);
                const half2v sv = scale_pair(s.vs[t]);
                // token 2 pair: of its sixteen in quarter (pair / 2) % 4; quarter 2 x + y goes to chunk y (of the sixteen's two), half x
                const int quarter = (pair >> 1) & 3, chunk = 2 * (pair >> 3) + (quarter & 1);
                const uint32_t in_chunk = (uint32_t)(8 * (quarter >> 1) + 4 * (pair & 1));
                uint8_t *to = lds.v[stage] + in_chunk;
                const int e = 8 * part;
                *(half2v *)(to + v_place(e, chunk)) = code_pair<0>(even) * sv;
                *(half2v *)(to + v_place(e + 1, chunk)) = code_pair<0>(odd) * sv;
                *(half2v *)(to + v_place(e + 2, chunk)) = code_pair<1>(even) * sv;
                *(half2v *)(to + v_place(e + 3, chunk)) = code_pair<1>(odd) * sv;
                *(half2v *)(to + v_place(e + 4, chunk)) = code_pair<2>(even) * sv;
                *(half2v *)(to + v_place(e + 5, chunk)) = code_pair<2>(odd) * sv;
                *(half2v *)(to + v_place(e + 6, chunk)) = code_pair<3>(even) * sv;
                *(half2v *)(to + v_place(e + 7, chunk)) = code_pair<3>(odd) * sv;
            }
        }
        if (tid < kTileStep) {
            lds.mean[stage][tid] = __uint_as_float(s.mean << 16);
            if ((tid & 15) == 0) {
                lds.kg[stage][tid >> 4] = s.kg;
                lds.log_v[stage][tid >> 4] = __builtin_amdgcn_logf(s.vg);
                lds.inv_v[stage][tid >> 4] = __builtin_amdgcn_rcpf(s.vg);
                lds.valid[stage][tid >> 4] = s.valid;
            }
        }
    };

    float m = kLowest, l = 0.0f;
    float16v o[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;

    auto take = [&](int n, int stage) {
        const int first = steps.first_token(n, kTileStep);
        float x[2][16];
        const uint32_t all_valid = lds.valid[stage][0] & lds.valid[stage][1] & lds.valid[stage][2] & lds.valid[stage][3];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float16v acc;
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                const half8v kf = *(const half8v *)(lds.k[stage] + k_place<D>(32 * t + c32, 2 * c + hi));
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, q[c], acc, 0, 0, 0);
            }
            // acc[e]: token 32 t + 8 (e / 4) + 4 hi + e % 4
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const int group = 2 * t + (e4 >> 1);
                const float f = factor * lds.kg[stage][group];
                float4v add = {lds.log_v[stage][group], lds.log_v[stage][group], lds.log_v[stage][group], lds.log_v[stage][group]};
                if (smooth) {
                    const float4v mean = *(const float4v *)&lds.mean[stage][32 * t + 8 * e4 + 4 * hi];
#pragma unroll
                    for (int e = 0; e < 4; ++e) add[e] = __builtin_fmaf(mean[e], sum_q, add[e]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) x[t][4 * e4 + e] = __builtin_fmaf(acc[4 * e4 + e], f, add[e]);
            }
        }
        const bool masked = all_valid == 0u || first + kTileStep - 1 > seq.position(a, i0) ||
                            (a.window > 0 && first <= seq.position(a, i1) - a.window);
        if (masked) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int at = 32 * t + 8 * (e >> 2) + 4 * hi + (e & 3);
                    x[t][e] = (lds.valid[stage][2 * t + (e >> 3)] != 0u && seen(a, first + at, p)) ? x[t][e] : -__builtin_inff();
                }
        }
        float top = kLowest;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 2) top = fmaxf(fmaxf(top, x[t][e]), x[t][e + 1]);
        if (__ballot(top > m + kSlack) != 0ull) {
            const float raised = fmaxf(fmaxf(top, __shfl_xor(top, 32, 64)), m);
            const float f = __builtin_amdgcn_exp2f(m - raised);
            m = raised;
            l *= f;
#pragma unroll
            for (int t = 0; t < D / 32; ++t) o[t] *= f;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {                        // sixteen tokens
                half8v w, w_low;
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = __builtin_amdgcn_exp2f(x[t][8 * s + e] - m);
                    sum += v;
                    w[e] = (_Float16)v;
                    if constexpr (F32) w_low[e] = (_Float16)(v - (float)w[e]);
                }
                l = __builtin_fmaf(sum, lds.inv_v[stage][2 * t + s], l);
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    const half8v vf = *(const half8v *)(lds.v[stage] + v_place(32 * c + c32, 2 * (2 * t + s) + hi));
                    o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, w, o[c], 0, 0, 0);
                    if constexpr (F32) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, w_low, o[c], 0, 0, 0);
                }
            }
    };

    if (n0 < n1) {
        Share s;
        fetch(n0, s);
        store(s, 0);
        __syncthreads();
        for (int n = n0; n < n1; ++n) {
            const int stage = (n - n0) & 1;
            if (n + 1 < n1) fetch(n + 1, s);
            take(n, stage);
            // (the other stage was read in the turn before, which every wave has left behind the barrier)
            if (n + 1 < n1) store(s, stage ^ 1);
            __syncthreads();
        }
    }

    l += __shfl_xor(l, 32, 64);
    if (!row) return;
    // o[c][e]: element 32 c + 8 (e / 4) + 4 hi + e % 4
    const int64_t out_row = query * a.Hq + head;
    if (alone) {
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        if (a.lse && hi == 0) a.lse[out_row] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -__builtin_inff();
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
    const int64_t part = (int64_t)piece * a.total_q * a.Hq + out_row;
    if (hi == 0) a.part_ml[part] = float2{m, l};
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int first = 32 * c + 2 * e + 4 * hi;
            if (first < a.d) *(float4v *)(a.part_o + part * a.d + first) = float4v{o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]};
        }
}

template <int D, int WAVES, bool F32>
static hipError_t launch_tiles(const AttentionArgs &a, const KvAttention &k, hipStream_t s)
{
    auto kernel = attention_tiles_kernel<D, WAVES, F32>;
    constexpr int bytes = (int)sizeof(Tiles<D, WAVES>);
    static bool raised[64] = {};                                       // the dynamic LDS limit, once per device
    int dev = -1;
    if (hipError_t e = hipGetDevice(&dev)) return e;
    if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
    if (!raised[dev]) {
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes)) return e;
        raised[dev] = true;
    }
    const unsigned grid = (unsigned)((int64_t)a.plan.groups * a.B * a.H * a.plan.pieces);
    kernel<<<grid, 64 * WAVES, bytes, s>>>(a, k.page_table, k.kv_lens, k.q_starts, k.cache.k_global, k.cache.v_global);
    return hipGetLastError();
}

hipError_t launch_attention_tiles(const AttentionArgs &a, const KvAttention &k, hipStream_t s)
{
    const bool f = k.out_f32;
    if (a.d > 128) return f ? launch_tiles<256, 4, true>(a, k, s) : launch_tiles<256, 4, false>(a, k, s);
    if (a.plan.waves == 8) {
        if (a.d <= 64) return f ? launch_tiles<64, 8, true>(a, k, s) : launch_tiles<64, 8, false>(a, k, s);
        return f ? launch_tiles<128, 8, true>(a, k, s) : launch_tiles<128, 8, false>(a, k, s);
    }
    if (a.d <= 64) return f ? launch_tiles<64, 4, true>(a, k, s) : launch_tiles<64, 4, false>(a, k, s);
    return f ? launch_tiles<128, 4, true>(a, k, s) : launch_tiles<128, 4, false>(a, k, s);
}

}  // namespace nvfp4
