// Joins the partial results of attention over pieces of the cached tokens, and the launcher of both attention kernels.
#include "nvfp4_attention.h"

namespace nvfp4 {

// Threads threads take a row (query, head): the pieces' maxima and sums first (every wave for itself, a lane a piece), then
// their partial sums, d / 4 lanes to a piece, as many pieces side by side as there are lanes for.  Pieces are added in an
// order that does not depend on when they finished.  A wave a row where there are few pieces and many rows (chunks: 84480
// rows in three pieces took 53 us, a workgroup to each 182), a workgroup where there are many pieces (single tokens: 256
// rows in 50 pieces 9 us and 6).
constexpr int kJoinThreads = 256, kJoinFew = 8;
template <int THREADS>
__global__ __launch_bounds__(kJoinThreads) void attention_join_kernel(const AttentionArgs a, const int32_t *__restrict__ kv_lens, const int32_t *__restrict__ q_starts,
                                                                      const float *__restrict__ part_o, const float2 *__restrict__ part_ml, int out_f32)
{
    __shared__ float4v sums[THREADS > 64 ? THREADS : 1];
    const int lane = threadIdx.x & 63, tid = (int)threadIdx.x & (THREADS - 1);
    const int64_t id = (int64_t)blockIdx.x * (kJoinThreads / THREADS) + __builtin_amdgcn_readfirstlane((int)threadIdx.x / THREADS);
    int i, b, head, pieces;
    int64_t first, stride;                                    // partial rows of this row: first + s * stride
    if (a.plan.rows16) {
        head = (int)(id % a.Hq);
        i = (int)(id / a.Hq % a.max_q);
        b = (int)(id / a.Hq / a.max_q);
        if (b >= a.B) return;
    } else {
        const int rows = 32 * a.plan.waves;
        const int64_t j = id / rows;
        if (j >= a.plan.rest) return;
        const Block place(a, a.plan.whole + j);
        const int row = place.block * rows + (int)(id - j * rows);
        i = row / a.G;
        head = place.h * a.G + (row - i * a.G);
        b = place.b;
        first = j * a.plan.pieces * rows + (id - j * rows);
        stride = rows;
    }
    Sequence seq;
    if (a.plan.rows16) {
        const Pieces p(a, q_starts, kv_lens, b, true);
        seq = p.seq;
        pieces = p.count;
        first = ((int64_t)p.first * a.max_q + i) * a.Hq + head;
        stride = (int64_t)a.max_q * a.Hq;
    } else seq = Sequence(a, q_starts, kv_lens, b);
    const int n_q = min(seq.n_q, a.max_q);
    if (i >= n_q) return;
    const int64_t query = (int64_t)seq.start + i, out_row = query * a.Hq + head;
    if (!a.plan.rows16) {
        const int rows = 32 * a.plan.waves, row0 = (i * a.G + head % a.G) / rows * rows;
        const Steps steps(a, seq, row0 / a.G, min((row0 + rows - 1) / a.G, n_q - 1), kTileStep);
        const int piece_steps = tile_piece_steps(a, steps.total);
        pieces = (steps.total + piece_steps - 1) / piece_steps;
    }
    if (pieces <= 1) return;                                  // (written by its workgroup)

    float m = kLowest;
    for (int s = lane; s < pieces; s += 64) m = fmaxf(m, part_ml[first + s * stride].x);
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
    float l = 0.0f;
    for (int s = lane; s < pieces; s += 64) {
        const float2 v = part_ml[first + s * stride];
        l += moved_sum(v.y, v.x, m);
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) l += __shfl_xor(l, x, 64);
    const int lanes = THREADS > 64 ? a.d >> 2 : 64, side = THREADS / lanes, sub = tid / lanes, e = 4 * (tid - sub * lanes);
    float4v o = {0.0f, 0.0f, 0.0f, 0.0f};
    if (sub < side && e < a.d) {
#pragma unroll 4
        for (int s = sub; s < pieces; s += side) {
            const int64_t row = first + s * stride;
            const float w = __builtin_amdgcn_exp2f(part_ml[row].x - m);
            o += *(const float4v *)(part_o + row * a.d + e) * w;
        }
    }
    if constexpr (THREADS > 64) {
        sums[tid] = o;
        __syncthreads();
        if (sub == 0)
            for (int s = 1; s < side; ++s) o += sums[s * lanes + tid];
    }
    if (sub == 0 && e < a.d) {
        o *= inverse_sum(l);
        const int64_t at = query * a.ldo + (int64_t)head * a.d + e;
        if (out_f32) *(float4v *)((float *)a.out + at) = o;
        else *(uint2v *)((uint16_t *)a.out + at) = uint2v{pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w)};
    }
    if (a.lse && tid == 0) a.lse[out_row] = log_sum(m, l);
}

hipError_t launch_attention_join(const AttentionArgs &a, const KvAttention &k, hipStream_t s)
{
    const int64_t rows = a.plan.rows16 ? (int64_t)a.B * a.max_q * a.Hq : a.plan.rest * 32 * a.plan.waves;
    const bool few = !a.plan.rows16 && a.plan.pieces <= kJoinFew;
    const unsigned grid = (unsigned)(few ? (rows + 3) / 4 : rows);
    if (few) attention_join_kernel<64><<<grid, kJoinThreads, 0, s>>>(a, k.kv_lens, k.q_starts, a.part_o, a.part_ml, k.out_f32);
    else attention_join_kernel<kJoinThreads><<<grid, kJoinThreads, 0, s>>>(a, k.kv_lens, k.q_starts, a.part_o, a.part_ml, k.out_f32);
    return hipGetLastError();
}

hipError_t launch_kv_attention(const KvAttention &k, void *workspace, hipStream_t s)
{
    const KvPages &c = k.cache;
    AttentionArgs a{};
    a.q = k.q;
    a.ldq = k.ldq;
    a.ldo = k.ldo;
    a.total_q = (int)k.total_q;
    a.Hq = (int)k.Hq;
    a.H = c.H;
    a.G = (int)(k.Hq / c.H);
    a.d = c.d;
    a.n_pages = (int)c.n_pages;
    a.page_tokens = (int)c.page_tokens;
    a.max_pages = (int)k.max_pages;
    a.B = (int)k.B;
    a.max_q = (int)k.max_q;
    a.k_codes = c.k_codes;
    a.k_scales = c.k_scales;
    a.v_codes = c.v_codes;
    a.v_scales = c.v_scales;
    a.k_mean = c.k_mean;
    a.scale = k.softmax_scale * 1.4426950408889634f;
    a.causal = k.causal;
    a.window = (int)std::min(k.window, kFar);
    a.sink = (int)std::min(k.sink, kFar);
    a.out = k.out;
    a.lse = k.lse;
    a.plan = attention_plan(k.total_q, k.Hq, c.H, c.d, k.max_pages * c.page_tokens, k.B, k.max_q, k.window, k.sink);
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<float2 *>(a.part_o + a.plan.part_rows * c.d);
    a.token_codes = (uint32_t)(c.H * (c.d >> 1));
    a.token_scales = (uint32_t)(c.H * (c.d >> 4));
    a.page_scales = (uint32_t)c.page_tokens * a.token_scales;
    a.page_means = (uint32_t)c.page_tokens * 2u * (uint32_t)c.H;
    a.by_page = Divisor(c.page_tokens, k.max_pages * c.page_tokens);
    const hipError_t e = a.plan.rows16 ? launch_attention_rows16(a, k, s) : launch_attention_tiles(a, k, s);
    if (e != hipSuccess || a.plan.pieces <= 1) return e;
    return launch_attention_join(a, k, s);
}

}  // namespace nvfp4
