// What the two attention kernels share: which tokens a sequence's queries see, the values of a tile's page, the running
// maximum, and how partial results are laid out.
#pragma once

#include "nvfp4_attention_plan.h"
#include "nvfp4_device.h"
#include "nvfp4_kernels.h"

namespace nvfp4 {

struct AttentionArgs {
    const uint16_t *q;
    int64_t ldq, ldo;
    int32_t total_q, Hq, H, G, d, n_pages, page_tokens, max_pages, B, max_q;      // G: query heads of a cached head
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    const uint16_t *k_mean;
    float scale;                          // softmax scale times log2(e): scores are exponents of two
    int32_t causal, window, sink;
    void *out;
    float *lse;
    AttentionPlan plan;
    float *part_o;                        // [partial row][d], partial sums relative to ...
    float2 *part_ml;                      // [partial row] ... 2^r of their row, and r (base 2) and the sum of its weights
    Divisor by_page;
    uint32_t token_codes, token_scales;   // bytes of a slot: codes, scales
    uint32_t page_scales, page_means;     // bytes of a page: scales, means
    uint32_t clear_from;                  // number of the first workgroup that clears rows, 0xFFFFFFFF: none
    int32_t clear_out, clear_lse, out_row;        // what it clears; 16-byte pieces of a row of `out`
};

// Sixteen cached tokens of a page: where their slots begin in each plane, as scalar bases for a lane's 32-bit offset.  (Two
// 32 x 32 bit products give them all, codes being eight times as long as scales.)
using GlobalBytes = const __attribute__((address_space(1))) uint8_t *;
__device__ __forceinline__ GlobalBytes scalar_base(const void *base, uint64_t at) { return (GlobalBytes)base + at; }
template <class T>
__device__ __forceinline__ T load_at(GlobalBytes base, uint32_t offset) { return *(const __attribute__((address_space(1))) T *)(base + offset); }
struct Slots {
    GlobalBytes k_codes, v_codes, k_scales, v_scales, k_mean;
    __device__ __forceinline__ Slots(const AttentionArgs &a, uint32_t page, int offset)
    {
        const uint64_t at = (uint64_t)page * a.page_scales + (uint32_t)offset * a.token_scales;
        k_codes = scalar_base(a.k_codes, at << 3);
        v_codes = scalar_base(a.v_codes, at << 3);
        k_scales = scalar_base(a.k_scales, at);
        v_scales = scalar_base(a.v_scales, at);
        k_mean = scalar_base(a.k_mean, (uint64_t)page * a.page_means + (uint32_t)offset * (2u * (uint32_t)a.H));
    }
};

// Queries and cached tokens of a sequence (clamped to what the call describes), and the steps of kStep tokens that some
// query among i0 .. i1 sees: sink_steps steps from token 0, then those from lo_step on.
struct Sequence {
    int start, n_q, len, p0;              // p0: position of query 0; query i stands at p0 + i (causal) or p0
    Sequence() = default;
    __device__ __forceinline__ Sequence(const AttentionArgs &a, const int32_t *__restrict__ q_starts, const int32_t *__restrict__ kv_lens, int b)
    {
        start = min(max(q_starts[b], 0), a.total_q);
        n_q = min(max(q_starts[b + 1], start), a.total_q) - start;
        len = min(max(kv_lens[b], 0), a.max_pages * a.page_tokens);
        p0 = a.causal ? len - n_q : len - 1;
    }
    __device__ __forceinline__ int position(const AttentionArgs &a, int i) const { return a.causal ? p0 + i : p0; }
};
struct Steps {
    int sink_steps, lo_step, total;
    __device__ __forceinline__ Steps(const AttentionArgs &a, const Sequence &q, int i0, int i1, int step_tokens)
    {
        const int hi = q.position(a, i1) + 1;                                    // (at most q.len)
        const int lo = a.window > 0 ? max(q.position(a, i0) - a.window + 1, 0) : 0;
        lo_step = lo / step_tokens;
        const int hi_step = hi > 0 ? (hi + step_tokens - 1) / step_tokens : 0;
        sink_steps = a.window > 0 && hi > 0 ? min((min(a.sink, hi) + step_tokens - 1) / step_tokens, lo_step) : 0;
        total = sink_steps + max(hi_step - lo_step, 0);
    }
    __device__ __forceinline__ int first_token(int n, int step_tokens) const { return (n < sink_steps ? n : n - sink_steps + lo_step) * step_tokens; }
};

// rows16: the pieces of all sequences, one behind the other, in the order of the sequences.  A piece is as many steps as
// make about plan.pieces of them out of what the lengths on the device ask for, so that the work is spread evenly whatever
// the lengths are (pieces laid out for the longest sequence left a third of the chip's shader engines with twice the others'
// work: workgroups go round them by number, the empty ones too).  Every wave finds its place by a scan over the sequences,
// 64 at a time, in registers.
struct Pieces {
    int steps;                            // of a piece
    int first, count;                     // pieces in front of sequence b, and its own
    int b;                                // sequence of piece number `at`, B: behind the last one
    Sequence seq;
    // steps of sequence s (-1: no queries, or behind the last one)
    __device__ __forceinline__ static int sequence_steps(const AttentionArgs &a, const Sequence &s, bool there)
    {
        const int n_q = min(s.n_q, a.max_q);
        return there && n_q > 0 ? Steps(a, s, 0, max(n_q, 1) - 1, kRows16Step).total : -1;
    }
    // inclusive sum over the lanes up to each: within rows of sixteen, then row 0 into 1 and 2 into 3, then the lower half into the upper
    __device__ __forceinline__ static uint32_t up_to(uint32_t v)
    {
        v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, true);
        v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, true);
        v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, true);
        v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, true);
        v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);
        v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);
        return v;
    }
    // by_sequence: `at` is a sequence, its pieces are what is asked for
    __device__ __forceinline__ Pieces(const AttentionArgs &a, const int32_t *__restrict__ q_starts, const int32_t *__restrict__ kv_lens, int at, bool by_sequence)
    {
        const int lane = threadIdx.x & 63;
        const int last = a.B - 1;
        Sequence lanes(a, q_starts, kv_lens, min(lane, last));               // this lane's sequence, of 64 (the first 64 until the second loop asks for more)
        int mine = sequence_steps(a, lanes, lane <= last);
        int64_t total = (uint32_t)__builtin_amdgcn_readlane((int)up_to((uint32_t)max(mine, 0)), 63);         // (64 of at most 2^25 steps)
        for (int b0 = 64; b0 < a.B; b0 += 64) {
            const Sequence other(a, q_starts, kv_lens, min(b0 + lane, last));
            total += (uint32_t)__builtin_amdgcn_readlane((int)up_to((uint32_t)max(sequence_steps(a, other, b0 + lane <= last), 0)), 63);
        }
        steps = a.plan.pieces <= 1 ? 0x3FFFFFFF : max((int)min((total + a.plan.pieces - 1) / a.plan.pieces, (int64_t)0x3FFFFFFF), a.plan.piece_steps);
        int before = 0;
        for (int b0 = 0; b0 < a.B; b0 += 64) {
            if (b0 > 0) {
                lanes = Sequence(a, q_starts, kv_lens, min(b0 + lane, last));
                mine = sequence_steps(a, lanes, b0 + lane <= last);
            }
            const int n = mine < 0 ? 0 : max((int)(((uint32_t)mine + (uint32_t)steps - 1u) / (uint32_t)steps), 1);       // (a sequence without tokens has one, which writes its zeros)
            const int upto = (int)up_to((uint32_t)n);
            const bool here = by_sequence ? b0 + lane == at : (at >= before + upto - n) & (at < before + upto);
            if (const uint64_t found = __ballot(here)) {
                const int l = (int)__builtin_ctzll(found);
                b = b0 + l;
                count = __builtin_amdgcn_readlane(n, l);
                first = before + __builtin_amdgcn_readlane(upto, l) - count;
                seq.start = __builtin_amdgcn_readlane(lanes.start, l);
                seq.n_q = __builtin_amdgcn_readlane(lanes.n_q, l);
                seq.len = __builtin_amdgcn_readlane(lanes.len, l);
                seq.p0 = __builtin_amdgcn_readlane(lanes.p0, l);
                return;
            }
            before += __builtin_amdgcn_readlane(upto, 63);
        }
        b = a.B;
        first = count = 0;
        seq = lanes;
    }
};

// Blocks of rows (tiles): number `at` of all blocks <-> sequence, cached head and block.  Blocks that read the same tokens of
// the same head are eight numbers apart, and so on one of the eight chiplets, each of which has an L2.
struct Block {
    int b, h, block;
    __device__ __forceinline__ Block(const AttentionArgs &a, int64_t at)
    {
        const int64_t same = a.plan.groups, full = (int64_t)a.B * a.H & ~(int64_t)7;
        int64_t set;
        if (at < full * same) {
            set = at / (8 * same) * 8 + (at & 7);
            block = (int)((at >> 3) % same);
        } else {
            set = full + (at - full * same) / same;
            block = (int)((at - full * same) % same);
        }
        h = (int)(set % a.H);
        b = (int)(set / a.H);
    }
};
// steps of a piece of a block that is cut
__device__ __forceinline__ int tile_piece_steps(const AttentionArgs &a, int total) { return max((total + a.plan.pieces - 1) / a.plan.pieces, a.plan.piece_steps); }

// What a query at position p sees: token j <= p, behind `after` or in front of the sink's end.
struct Sight {
    int p, after, sink;
    __device__ __forceinline__ Sight(const AttentionArgs &a, int position) : p(position), after(a.window > 0 ? position - a.window : -0x40000000), sink(a.sink) {}
    __device__ __forceinline__ bool of(int j) const { return (j <= p) & ((j > after) | (j < sink)); }
};

// A token's weight in the second product is 2^(s - m) g / 2^U = 2^(s + log2 g - r), r = m + U, and the values enter it as code *
// block scale, exact in f16.
//   m   lies kBelow binades (rounded down to a whole number, which r then is too) under the row's running maximum of s, and is
//       raised to there only when a score exceeds it by kAbove: most steps then need no reduction between lanes and no rescaling.
//   g   value scale of the token's page; the sum of the weights takes it out again.
//   2^U the unit in which a wave counts.  It stays where it is while the exponents of a step's pages are kUnitLow .. kUnitHigh from it
//       (pages whose scales differ by a few times), else it moves and the accumulators are rescaled.  Pages of one step that no
//       unit holds for together are taken in walks of their own over the steps that have such ones.  (With weights relative
//       to the largest 2^s g, a page of large scale and small values cost the others their digits; a page of zeros has scale one.)
// Weights stay below 2^(kAbove + 1 + kUnitHigh) = 2^15.  What f16 cannot hold is 2^-25, and so 2^-30 of the largest 2^s (kBelow
// and kUnitLow) whatever the pages' scales are; with the maximum itself for m a long tail behind a token with nearly all of the
// sum was lost from the product while the sum kept it.
// The unit does not go below 2^-84, nor further than kUnitReach below the largest that it has been: no rescaling overflows (2^15 *
// 2688 * 2^30 tokens are 2^57), and neither does a sum of weights / g (2^(kAbove + 30 + 84)).  Pages that it does not reach lose
// digits, and from kUnitLost below it on their weights count in the sum alone.
constexpr float kBelow = 7.0f, kAbove = 13.0f, kLowest = -3.0e38f;      // (kLowest: below every score, and 2^(-inf - kLowest) is still 0)
constexpr int kUnitLow = -2, kUnitHigh = 1, kUnitReach = 64, kUnitLost = 40, kUnitBias = 127, kUnitLeast = 43;       // (exponent fields as in fp32)
constexpr int kNoUnit = -512;
struct Units {
    int now, top;                         // U as an fp32 exponent field (at first kNoUnit), and the largest it has been
    __device__ __forceinline__ bool holds(int e) const { return (uint32_t)(e - now - kUnitLow) <= (uint32_t)(kUnitHigh - kUnitLow); }
    // for a page with exponent field e: log2 g and 1 / g as they enter a weight and the sum
    __device__ __forceinline__ void page(int e, float &log_g, float &inv_g) const
    {
        if (e < now - kUnitLost) {
            log_g = (float)(now - kUnitBias - kUnitLost);
            inv_g = __builtin_amdgcn_exp2f(-log_g);
        }
    }
    // Groups of sixteen tokens, a bit each in `groups`, their pages' exponent fields the bytes of e.  Those that one unit can hold for
    // make a class, from the largest on (so that the classes do not depend on the unit).  Of class number `pass` the bits, and
    // in `groups` what the classes behind it have; the unit is made to hold.
    template <int GROUPS>
    __device__ __forceinline__ uint32_t enter(uint32_t e, uint32_t &groups, int pass)
    {
        uint32_t mine = 0u;
        int largest = 0;
        bool held = true;
        for (int k = 0; k <= pass; ++k) {
            groups &= ~mine;
            mine = 0u;
            largest = 0;
            held = true;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
                if ((groups >> g & 1u) != 0u) largest = max(largest, (int)(e >> 8 * g & 255u));
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const int eg = (int)(e >> 8 * g & 255u);
                if ((groups >> g & 1u) == 0u || eg < largest - (kUnitHigh - kUnitLow)) continue;
                mine |= 1u << g;
                held &= holds(eg);
            }
        }
        groups &= ~mine;
        if (!held) {
            now = max(max(largest - kUnitHigh, kUnitLeast), top - kUnitReach);
            top = max(top, now);
        }
        return mine;
    }
};
// Does a unit hold for the exponent fields in the four bytes of e?  Its lowest one in every byte, subtracted, leaves less than four in each; a
// difference that is negative borrows and leaves higher bits.
static_assert(kUnitHigh - kUnitLow == 3);
__device__ __forceinline__ uint32_t unit_lowest4(int now) { return (uint32_t)(now + kUnitLow) * 0x01010101u; }
__device__ __forceinline__ bool unit_holds4(uint32_t lowest4, uint32_t e) { return ((e - lowest4) & 0xFCFCFCFCu) == 0u; }
// exponent field of a page's scale: 4 .. 254 whatever stands there (255: not a page of the cache), so that zero is the lowest one of no unit
__device__ __forceinline__ uint32_t scale_exponent(uint32_t bits) { return min(max(bits >> 23 & 255u, 4u), 254u); }
constexpr uint32_t kNoPage = 255u;
// do some of the rows at positions p0 .. p1 see some of the sixteen tokens from `first` on?
__device__ __forceinline__ bool group_seen(int first, int p0, int p1, int window, int sink)
{
    return (first <= p1) & ((window <= 0) | (first + 15 > p0 - window) | (first < sink));
}

// A sum of weights relative to 2^from, relative to 2^to (both whole numbers: units may be further apart than a factor's range).
__device__ __forceinline__ float moved_sum(float l, float from, float to) { return __builtin_amdgcn_ldexpf(l, (int)fmaxf(from - to, -1024.0f)); }

// Of a row's sum of weights l relative to 2^r: what its products are multiplied by, and its log-sum-exp.  Nothing seen: zero and
// -inf; a sum that is no number (scores that are none) stays one.
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ float log_sum(float r, float l) { return l == 0.0f ? -__builtin_inff() : (r + __builtin_amdgcn_logf(l)) * 0.6931471805599453f; }

// E4M3 bytes in the low halves of two 16-bit lanes -> f16 values times 2^-8, exact (subnormal f16 where the byte is
// below 2^-6), for every byte: sign bit dropped, no NaN, so slots that were never written cannot reach a sum.
__device__ __forceinline__ half2v scale_pair(uint32_t b) { return __builtin_bit_cast(half2v, (b & 0x007F007Fu) << 7); }
// two codes -> f16 times 2^8; times a scale from scale_pair: code * block scale
template <int BYTE>
__device__ __forceinline__ half2v code_pair(uint32_t w) { return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 256.0f, BYTE); }

__device__ __forceinline__ half8v join8(half2v a, half2v b, half2v c, half2v d)
{
    return half8v{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// eight codes along a row (one word) times one scale
__device__ __forceinline__ half8v eight_codes(uint32_t w, half2v s)
{
    return join8(code_pair<0>(w) * s, code_pair<1>(w) * s, code_pair<2>(w) * s, code_pair<3>(w) * s);
}

// bf16 queries -> f16 times 2^row_exponent, which puts the row's largest magnitude into [2^14, 2^15): exact but for elements 2^-29 of
// it and less.  (-113 for the largest numbers; at most 110, which leaves every one above 2^-24.)
__device__ __forceinline__ int row_exponent(float amax) { return amax > 0.0f ? min(15 - __builtin_amdgcn_frexp_expf(amax), 110) : 0; }
__device__ __forceinline__ half8v query_pairs(uint4v w, int e)
{
    half8v r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[2 * i] = (_Float16)__builtin_amdgcn_ldexpf(bf16lo_to_f32(w[i]), e);
        r[2 * i + 1] = (_Float16)__builtin_amdgcn_ldexpf(bf16hi_to_f32(w[i]), e);
    }
    return r;
}
__device__ __forceinline__ float absmax8(uint4v w, float m)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(fmaxf(m, fabsf(bf16lo_to_f32(w[i]))), fabsf(bf16hi_to_f32(w[i])));
    return m;
}
// (of the queries times 2^e, whose sum cannot overflow)
__device__ __forceinline__ float sum8(uint4v w, int e, float s)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) s += __builtin_amdgcn_ldexpf(bf16lo_to_f32(w[i]), e) + __builtin_amdgcn_ldexpf(bf16hi_to_f32(w[i]), e);
    return s;
}

// Rows that no sequence computes, in outputs that hold nothing yet: in front of the first query and behind the last one, and
// from max_q on.  Workgroups behind those of a kernel's own work (a.clear_from on) set them to zero and -inf.
__device__ __forceinline__ void clear_rows(const AttentionArgs &a, int64_t from, int64_t to, int64_t by, int out_bytes)
{
    for (int64_t row = from; row < to; row += by) {
        uint4v *const out = (uint4v *)((uint8_t *)a.out + row * a.ldo * out_bytes);
        for (int i = threadIdx.x; a.clear_out && i < a.out_row; i += blockDim.x) out[i] = uint4v{0u, 0u, 0u, 0u};
        for (int i = threadIdx.x; a.clear_lse && i < a.Hq; i += blockDim.x) a.lse[row * a.Hq + i] = -__builtin_inff();
    }
}
template <bool F32>
__device__ __forceinline__ void clear_rest(const AttentionArgs &a, const int32_t *__restrict__ q_starts)
{
    constexpr int bytes = F32 ? 4 : 2;
    const int part = (int)(blockIdx.x - a.clear_from), parts = (int)(gridDim.x - a.clear_from);
    const int first = min(max(q_starts[0], 0), a.total_q), last = min(max(q_starts[a.B], first), a.total_q);
    clear_rows(a, part, first, parts, bytes);
    clear_rows(a, last + part, a.total_q, parts, bytes);
    for (int b = part; b < a.B; b += parts) {
        const int start = min(max(q_starts[b], 0), a.total_q), end = min(max(q_starts[b + 1], start), a.total_q);
        clear_rows(a, (int64_t)start + a.max_q, end, 1, bytes);
    }
}
// a grid of `own` workgroups and those that clear
inline unsigned attention_grid(AttentionArgs &a, const KvAttention &k, unsigned own)
{
    a.clear_out = k.clear_out;
    a.clear_lse = k.clear_lse;
    a.out_row = (int32_t)(k.Hq * k.cache.d * (k.out_f32 ? 4 : 2) / 16);
    a.clear_from = k.clear_out || k.clear_lse ? own : 0xFFFFFFFFu;
    return own + (a.clear_from == own ? (unsigned)std::min<int64_t>(std::max<int64_t>(k.total_q / 64, 8), kClearGroups) : 0u);
}

hipError_t launch_attention_rows16(AttentionArgs a, const KvAttention &k, hipStream_t s);
hipError_t launch_attention_tiles(AttentionArgs a, const KvAttention &k, hipStream_t s);
hipError_t launch_attention_join(const AttentionArgs &a, const KvAttention &k, hipStream_t s);

}  // namespace nvfp4
