// Product of 8-bit operands for gfx950:  Y[m, n] = sum over blocks of 128 k of 2^(sA + sW) sum_k A[m, k] W[n, k].
//
// Two ways through the matrix pipes, one kernel otherwise:
//   exact sums  The codes become bf16 in registers, scale included (v_cvt_scalef32_pk_bf16_fp8: an E4M3 number times a power of
//               two is a bf16 number), and v_mfma_f32_32x32x16_bf16 adds the exact products in fp32.
//   fast sums   v_mfma_scale_f32_32x32x64_f8f6f4 takes codes and scale bytes as they are, at twice the rate.  But this
//               instruction aligns eight neighbouring products to the largest of them and drops what lies 2^-14 below it
//               (found by crafted operands: of 2^16 and a second product in the same eight, 2^3 is kept and 2^2 is lost; in
//               another eight 2^-7 is kept).  Normal operands: 1.4e-5 off relative to the result, and 5e-5 where the channels'
//               magnitudes span 2^6; the sums of eights are fp32.  So it is the caller's choice.
//
// The instruction's row operand is W, its column operand A: a lane ends up with one row m and runs of four neighbouring n.
#pragma once

#include "nvfp4_e4m3.h"
#include "nvfp4_e4m3_plan.h"
#include "nvfp4_gemm_tile.h"

namespace nvfp4 {

// What leaves a tile: fp32, bf16, or for gate and up projections side by side the activated product in 8 bits (and bf16).
enum { kE4m3F32 = 0, kE4m3Bf16 = 1, kE4m3Silu = 2, kE4m3Gelu = 3 };

// One tile of BM x BN outputs (gated: BM x BN / 2, the W rows are BN / 2 of the gate and as many of the up projection), four
// waves of BM / 2 x BN / 2.  A step is 128 k: 128 bytes of every row, in STAGES stages of LDS filled by copies that write LDS
// directly.  LDS: chunk c (16 bytes) of row r stands at 128 r + 16 (c ^ ((r >> 1) & 7)), so that sixteen rows of one chunk,
// what sixteen lanes read at once, fall on distinct banks; the copies fetch the chunks in that order.
//
// Schedule of a step s with fast sums, fragments of its two halves (64 k each) in registers F0 and F1:
//   first half    multiplies F0, reads F1 from stage s % STAGES
//   then          waits for the own copies of step s + 1 and the reads, joins a barrier: stage s % STAGES is free, step s + 1 is in
//   second half   multiplies F1, starts the copies of step s + STAGES into that stage, reads F0 of step s + 1
// One barrier a step; a copy has STAGES - 1 steps to arrive, a read half a step.
// With exact sums a step is four phases of two sub-steps (16 k each): a phase reads the next one's codes, a sub-step expands the
// next one's operands between its matrix instructions, the barrier and the copies stand in front of and in the last phase.
// (Rows of 64 bytes in four slots, with a barrier every 64 k and three half steps for a copy, took 2 to 6 % longer on large products.)
// What bounds it is the clock that the matrix pipes hold: 3520 x 4096 x 14336 takes 182 to 185 us with fast sums (2.25 PFLOP/s, matrix
// instructions in 54 % of the SIMDs' cycles) and 316 with exact ones (1.31); gated 3520 x 2*11008 x 4096, gate and up kept, 470 to 490 with
// exact sums (1.3), 285 with fast ones (2.2: prologue and epilogue of its five rounds of tiles are not hidden, 96 us at K = 128);
// 4096 x 2048 x 17600, 256 tiles of 128 x 256, 280 (1.05: the two stages do not cover a line's first way from memory in full).
template <int BM, int BN, int KIND, bool FAST, int STAGES>
__global__ __launch_bounds__(256) void e4m3_gemm_kernel(const E4m3GemmArgs g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool GATED = KIND >= kE4m3Silu;
    constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32;   // wave tile, in 32 x 32 tiles
    constexpr int BF = GATED ? BN / 2 : BN, WF = BF / 2, TF = WF / 32;    // columns of the result
    constexpr int UA = BM / 32, UW = BN / 32;                             // copies (8 rows) of a wave and step
    constexpr int STAGE = (BM + BN) * 128;
    constexpr int NF = TM + TN, NMF = TM * TN;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    typedef __attribute__((address_space(3))) void *lds_ptr_t;

    // ---- tile: each of the eight chiplets (workgroup id modulo 8) takes neighbouring tiles, in groups of kGroup tile rows
    constexpr int kGroup = 8;
    const int per_xcd = (int)(gridDim.x >> 3), at = (int)(blockIdx.x & 7u) * per_xcd + (int)(blockIdx.x >> 3);
    if (at >= g.tiles_m * g.tiles_n) return;
    const int in_group = kGroup * g.tiles_n, group = at / in_group, first_m = group * kGroup, rows_m = min(kGroup, g.tiles_m - first_m);
    const int rest = at - group * in_group, tile_n = rest / rows_m, tile_m = first_m + rest - tile_n * rows_m;
    const int64_t m0 = (int64_t)tile_m * BM, n0 = (int64_t)tile_n * BF;

    const int tid = threadIdx.x, lane = tid & 63, lrow = lane & 31, lhalf = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
    const int K = (int)g.K, S = (K + 127) >> 7;

    // ---- copies.  The tile's rows are the range that is checked: rows past the operand's end, and chunks past the end of a
    // row (given an offset past the range), read as zeros.
    const int rows_a = (int)min((int64_t)BM, g.M - m0), rows_w = (int)min((int64_t)BF, g.N - n0);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void *)(g.codes_a + m0 * K), 0, rows_a * K, 0x00020000);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void *)(g.codes_w + n0 * K), 0, rows_w * K, 0x00020000);
    const __amdgpu_buffer_rsrc_t ru = __builtin_amdgcn_make_buffer_rsrc((void *)(g.codes_w + (GATED ? g.N + n0 : n0) * K), 0, rows_w * K, 0x00020000);
    constexpr int kPast = 0x40000000;                      // (a tile has at most 256 rows of 2^22 bytes; with the row added it stays below 2^31)
    int chunk_at[2];                                       // byte of the row that a lane fetches, in copies of even and odd number
#pragma unroll
    for (int p = 0; p < 2; ++p) chunk_at[p] = ((lane & 7) ^ ((4 * p + (lane >> 4)) & 7)) << 4;
    const int row_at = (lane >> 3) * K;
    // copy x of step s: rows 8 u .. 8 u + 7, u = the wave's first copy + x (even for x even: a wave's counts are even)
    static_assert(UA % 2 == 0 && (GATED ? UW / 2 : UW) % 2 == 0, "copies of a wave");
    int place[STAGES];                                     // of the stages of steps s0, s0 + 1, ...: they change places where four steps are no whole turns
#pragma unroll
    for (int i = 0; i < STAGES; ++i) place[i] = i * STAGE;
    auto next_turn = [&] {
        if constexpr (4 % STAGES != 0) {
            int moved[STAGES];
#pragma unroll
            for (int i = 0; i < STAGES; ++i) moved[i] = place[(i + 4) % STAGES];
#pragma unroll
            for (int i = 0; i < STAGES; ++i) place[i] = moved[i];
        }
    };
    int from[2];                                           // lane offsets of the step being copied
    auto start_step = [&](int s) {
        const int left = K - s * 128;
#pragma unroll
        for (int p = 0; p < 2; ++p) from[p] = chunk_at[p] < left ? row_at + chunk_at[p] + s * 128 : kPast;
    };
    auto copy = [&](int s, auto x_c) {
        constexpr int x = decltype(x_c)::value;
        uint8_t *stage = lds + place[s % STAGES];
        if constexpr (x < UA) {
            const int u = wave * UA + x;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr_t)(stage + u * 1024), 16, from[x & 1] + u * 8 * K, 0, 0, 0);
        } else {
            // gated: half of the wave's copies are gate rows (LDS rows BM ..), the other half up rows (BM + BN / 2 ..)
            constexpr int y = x - UA;
            constexpr bool up = GATED && y >= UW / 2;
            const int u = GATED ? wave * (UW / 2) + (up ? y - UW / 2 : y) : wave * UW + y;
            uint8_t *dst = stage + BM * 128 + (up ? BF * 128 : 0) + u * 1024;
            const int off = from[y & 1] + u * 8 * K;
            if constexpr (up) __builtin_amdgcn_raw_ptr_buffer_load_lds(ru, (lds_ptr_t)dst, 16, off, 0, 0, 0);
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_ptr_t)dst, 16, off, 0, 0, 0);
        }
    };

    // ---- fragments: f < TM rows of A, then rows of W (gated: first the gate's, then the up projection's)
    auto frag_row0 = [&](int f) {
        if (f < TM) return wm * WM + f * 32;
        const int i = f - TM;
        if constexpr (GATED) return BM + (i >= TF ? BF : 0) + wn * WF + (i >= TF ? i - TF : i) * 32;
        return BM + wn * WN + i * 32;
    };
    int frag_at[4];                                        // 16-byte chunks 2 c + half of the lane's row
#pragma unroll
    for (int c = 0; c < 4; ++c) frag_at[c] = lrow * 128 + (((2 * c + lhalf) ^ ((lrow >> 1) & 7)) << 4);
    auto read_chunk = [&](int s, int c, int f) { return *(const uint4v *)(lds + place[s % STAGES] + frag_row0(f) * 128 + frag_at[c]); };

    // ---- scales: a word holds those of four steps of a fragment's row
    const int nb = S;
    uint32_t next_scale[NF];
    int scale_at[NF];                                      // of the lane's row, from the tile's first
    const uint8_t *scales_a = g.scales_a + m0 * nb;
    const int64_t w_first = g.w_tiles ? n0 >> 7 : n0;
    const uint8_t *scales_w = g.scales_w + w_first * nb;
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        if (f < TM) scale_at[f] = min(frag_row0(f) + lrow, rows_a - 1) * nb;
        else {
            int r = frag_row0(f) - BM + lrow;
            const bool up = GATED && r >= BF;
            r = min(up ? r - BF : r, rows_w - 1);
            const int64_t n = n0 + r + (up ? g.N : 0);
            scale_at[f] = (int)((g.w_tiles ? n >> 7 : n) - w_first) * nb;
        }
    }
    auto load_scales = [&](int group) {                    // of steps 4 group .. + 3; bytes behind the row's last become 0
        const uint32_t mine = 4 * group + 4 > nb ? (1u << 8 * (nb - 4 * group)) - 1u : 0xFFFFFFFFu;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const uint8_t *p = (f < TM ? scales_a : scales_w) + scale_at[f];
            if (g.scale_words) next_scale[f] = *(const uint32_t *)(p + 4 * group);
            else {                                         // at any address; one that would end behind the array is moved back to its last word
                typedef uint32_t any_word __attribute__((aligned(1)));
                const int64_t bytes = f < TM ? g.scales_a_bytes : g.scales_w_bytes, left = bytes - (p - (f < TM ? g.scales_a : g.scales_w));
                if (bytes >= 4) {
                    const int at = (int)min((int64_t)(4 * group), left - 4);
                    next_scale[f] = *(const any_word *)(p + at) >> 8 * (4 * group - at) & mine;
                } else {                                   // (a single group)
                    uint32_t w = 0u;
                    for (int b = 0; b < nb; ++b) w |= (uint32_t)p[b] << 8 * b;
                    next_scale[f] = w;
                }
            }
        }
    };

    float16v acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    // all but the last N copies have arrived, all reads are back
    auto wait_and_join = [&](auto n_c) {
        constexpr int n = decltype(n_c)::value;
        static_assert(n < 64, "vmcnt");
        NVFP4_COMPILER_FENCE();
        __builtin_amdgcn_s_waitcnt(0x0070 | (n & 15) | (n >> 4) << 14);
        __builtin_amdgcn_s_barrier();
        NVFP4_COMPILER_FENCE();
    };
    using InFlight = std::integral_constant<int, (STAGES - 2) * (UA + UW)>;      // at a step's barrier: the copies behind the next step's

    load_scales(0);
    uint32_t word[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) word[f] = next_scale[f];
    static_for<0, STAGES>([&](auto s) {
        start_step(s);
        static_for<0, UA + UW>([&](auto x) { copy(s, x); });
    });
    wait_and_join(std::integral_constant<int, (STAGES - 1) * (UA + UW)>());

    // Four steps (a word of scales) are one basic block: a branch between matrix instructions would let the compiler move them
    // behind it, out of the shadow of what they are placed around.  So copies past the end of K go out with offsets past the
    // range, and the steps that fill up the last four multiply the zeros that these leave.
    if constexpr (FAST) {
        union Frag {
            uint4v q[2];
            int8v v;
        };
        Frag frag[2][NF];
        uint32_t scale[NF];
        static_for<0, NF>([&](auto f) {
            frag[0][f].q[0] = read_chunk(0, 0, f);
            frag[0][f].q[1] = read_chunk(0, 1, f);
            scale[f] = word[f];
        });
        for (int s0 = 0; s0 < S; s0 += 4) {
            load_scales(min((s0 >> 2) + 1, (S - 1) >> 2));
            static_for<0, 8>([&](auto half_c) {
                constexpr int q = decltype(half_c)::value / 2, h = decltype(half_c)::value % 2;
                if constexpr (h == 1) {
                    wait_and_join(InFlight());
                    start_step(s0 + q + STAGES);
                }
                static_for<0, NMF>([&](auto t_c) {
                    constexpr int t = decltype(t_c)::value, i = t / TM, j = t % TM;
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag[h][TM + i].v, frag[h][j].v, acc[i][j], 0, 0, 0, (int)scale[TM + i], 0, (int)scale[j]);
                    __builtin_amdgcn_sched_barrier(0);
                    // the 2 NF reads of a half go behind the first matrix instructions, two to one: they are back when it ends
                    constexpr int kEach = (2 * NF + NMF - 1) / NMF > 2 ? (2 * NF + NMF - 1) / NMF : 2;
                    static_for<0, 2 * NF>([&](auto pc) {
                        if constexpr (pc / kEach == t) frag[1 - h][pc / 2].q[pc % 2] = read_chunk(q + h, 2 * (1 - h) + pc % 2, pc / 2);
                    });
                    if constexpr (h == 1)
                        static_for<0, UA + UW>([&](auto x) {
                            if constexpr (x * NMF / (UA + UW) == t) copy(q, x);
                        });
                    __builtin_amdgcn_sched_barrier(0);
                });
                if constexpr (h == 1) {
#pragma unroll
                    for (int f = 0; f < NF; ++f) scale[f] = q == 3 ? next_scale[f] : scale[f] >> 8;
                }
            });
            next_turn();
        }
    } else {
        typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
        uint4v codes[2][NF], frag[2][NF];
        float scale[NF];
        // two of the eight elements that a lane of fragment f has in sub-step j of a phase whose codes are `codes[set]`
        auto expand = [&](int set, int j, int f, int d) {
            const uint32_t w = codes[set][f][2 * j + (d >> 1)];
            uint32_t x = d & 1 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale[f], true))
                               : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale[f], false));
            NVFP4_PIN1(x);                                 // (where it is written: left alone it sinks to its use)
            frag[j][f][d] = x;
        };
        // an E8M0 byte is the exponent of an fp32 number; the conversion takes nothing else of its scale (0 is 2^-127, 255 NaN)
        auto take_scales = [&](int q) {
#pragma unroll
            for (int f = 0; f < NF; ++f) scale[f] = __uint_as_float((word[f] >> 8 * q & 255u) << 23);
        };
        static_for<0, NF>([&](auto f) { codes[0][f] = read_chunk(0, 0, f); });
        take_scales(0);
        static_for<0, 4 * NF>([&](auto pc) { expand(0, 0, pc / 4, pc % 4); });
        for (int s0 = 0; s0 < S; s0 += 4) {
            load_scales(min((s0 >> 2) + 1, (S - 1) >> 2));
            static_for<0, 32>([&](auto sub_c) {
                constexpr int q = decltype(sub_c)::value / 8, c = decltype(sub_c)::value / 2 % 4, j = decltype(sub_c)::value % 2, set = c & 1;
                if constexpr (c == 3 && j == 0) {
                    wait_and_join(InFlight());
                    start_step(s0 + q + STAGES);
                }
                if constexpr (c == 3 && j == 1) {
                    if constexpr (q == 3) {
#pragma unroll
                        for (int f = 0; f < NF; ++f) word[f] = next_scale[f];
                    }
                    take_scales((q + 1) & 3);
                }
                static_for<0, NMF>([&](auto t_c) {
                    constexpr int t = decltype(t_c)::value, i = t / TM, jj = t % TM;
                    acc[i][jj] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8v, frag[j][TM + i]), __builtin_bit_cast(bf16x8v, frag[j][jj]), acc[i][jj], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    static_for<0, 4 * NF>([&](auto pc) {
                        if constexpr (pc * NMF / (4 * NF) == t) expand(j == 0 ? set : set ^ 1, 1 - j, pc / 4, pc % 4);
                    });
                    static_for<0, NF>([&](auto f) {
                        if constexpr (j == 0 && frag_slot<NMF, NF>(f) == t) codes[set ^ 1][f] = read_chunk(c == 3 ? q + 1 : q, (c + 1) & 3, f);
                    });
                    if constexpr (c == 3)
                        static_for<0, UA + UW>([&](auto x) {
                            if constexpr (x * 2 * NMF / (UA + UW) == j * NMF + t) copy(q, x);
                        });
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            next_turn();
        }
    }
    wait_and_join(std::integral_constant<int, 0>());       // (reads and copies past the end: the epilogue takes LDS over)

    // ---- epilogue.  A wave turns 32 rows at a time in LDS of its own and stores whole rows of its tile.
    const int64_t wave_m = m0 + wm * WM, wave_n = n0 + wn * WF;
    constexpr int kPitch = WF * 4 + 16, kSlab = 32 * kPitch;
    uint8_t *slab = lds + wave * kSlab;
    // columns [0, WF) of rows 32 j .. 32 j + 31: values of tiles i0 .. i0 + TF - 1 -> p[row * ld + column], columns below `limit`
    auto store_bf16 = [&](auto j_c, auto i0_c, uint16_t *p, int64_t ld, int64_t column, int64_t limit) {
        constexpr int j = decltype(j_c)::value, i0 = decltype(i0_c)::value, pitch = WF * 2 + 16;
#pragma unroll
        for (int i = 0; i < TF; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(uint2v *)(slab + lrow * pitch + (i * 32 + 8 * q + 4 * lhalf) * 2) =
                    uint2v{pack_bf16x2(acc[i0 + i][j][4 * q], acc[i0 + i][j][4 * q + 1]), pack_bf16x2(acc[i0 + i][j][4 * q + 2], acc[i0 + i][j][4 * q + 3])};
        NVFP4_COMPILER_FENCE();
        const bool whole = (ld & 7) == 0 && (column & 7) == 0 && ((uintptr_t)p & 15) == 0;
        constexpr int GPR = WF / 8;
#pragma unroll
        for (int x = 0; x < 32 * GPR / 64; ++x) {
            const int idx = x * 64 + lane, r = idx / GPR, c = idx % GPR * 8;
            const uint4v o = *(const uint4v *)(slab + r * pitch + c * 2);
            const int64_t m = wave_m + j * 32 + r, n = wave_n + c;
            if (m < g.M && n < limit) {
                uint16_t *dst = p + m * ld + column + n;
                if (whole && n + 8 <= limit) *(uint4v *)dst = o;
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (n + e < limit) dst[e] = (uint16_t)(o[e >> 1] >> 16 * (e & 1));
                }
            }
        }
        NVFP4_COMPILER_FENCE();
    };
    if constexpr (KIND == kE4m3F32) {
        float *p = (float *)g.y;
        const bool whole = (g.ldy & 3) == 0 && ((uintptr_t)p & 15) == 0;
        static_for<0, TM>([&](auto j_c) {
            constexpr int j = decltype(j_c)::value, GPR = WF / 4;
#pragma unroll
            for (int i = 0; i < TF; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(float4v *)(slab + lrow * kPitch + (i * 32 + 8 * q + 4 * lhalf) * 4) = float4v{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            NVFP4_COMPILER_FENCE();
#pragma unroll
            for (int x = 0; x < 32 * GPR / 64; ++x) {
                const int idx = x * 64 + lane, r = idx / GPR, c = idx % GPR * 4;
                const float4v o = *(const float4v *)(slab + r * kPitch + c * 4);
                const int64_t m = wave_m + j * 32 + r, n = wave_n + c;
                if (m < g.M && n < g.N) {
                    float *dst = p + m * g.ldy + n;
                    if (whole && n + 4 <= g.N) *(float4v *)dst = o;
                    else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (n + e < g.N) dst[e] = o[e];
                    }
                }
            }
            NVFP4_COMPILER_FENCE();
        });
    } else if constexpr (KIND == kE4m3Bf16) {
        static_for<0, TM>([&](auto j) { store_bf16(j, std::integral_constant<int, 0>(), (uint16_t *)g.y, g.ldy, 0, g.N); });
    } else {
        // gate and up of a column stand in the same place of tiles i and i + TF.  Their block of 128 columns is the workgroup's:
        // its largest magnitude is that of two lanes and two waves.
        uint32_t *top = (uint32_t *)(lds + 4 * kSlab);     // [BM][2]
        uint8_t *rows = lds + 4 * kSlab + BM * 8;          // [BM], 128 codes and 16 bytes of room each
        constexpr int kRow = 144;
        static_for<0, TM>([&](auto j_c) {
            constexpr int j = decltype(j_c)::value;
            // Of 256 accumulators those of the bands behind this one stay where the matrix instructions left them: taken over all at once,
            // 32 of them went to scratch memory and came back one by one, each a wait behind the stores (3 to 5 us a tile).
            if constexpr (NMF * 16 >= 256) {
#pragma unroll
                for (int jj = j + 1; jj < TM; ++jj)
#pragma unroll
                    for (int i = 0; i < TN; ++i) asm volatile("" : "+a"(acc[i][jj]));
            }
            if (g.gate_up) {
                store_bf16(j_c, std::integral_constant<int, 0>(), g.gate_up, g.ld_gate_up, 0, g.N);
                store_bf16(j_c, std::integral_constant<int, TF>(), g.gate_up, g.ld_gate_up, g.N, g.N);
            }
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < TF; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    acc[i][j][e] = activation<KIND == kE4m3Silu ? kActSilu : kActGelu>(acc[i][j][e]) * acc[i + TF][j][e];
                    most = abs_max(most, acc[i][j][e]);
                }
            uint32_t m = abs_bits(most);
            m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
            if (lhalf == 0) top[(wm * WM + j * 32 + lrow) * 2 + wn] = m;
            if (g.h_bf16) store_bf16(j_c, std::integral_constant<int, 0>(), g.h_bf16, g.ld_h, 0, g.N);
        });
        if (!g.codes) return;
        __syncthreads();
        static_for<0, TM>([&](auto j_c) {
            constexpr int j = decltype(j_c)::value;
            const int r = wm * WM + j * 32 + lrow;
            const uint32_t byte = e8m0_of_amax(max(top[2 * r], top[2 * r + 1]));
            const float scale = e8m0_scale(byte);
            if (wn == 0 && lhalf == 0 && m0 + r < g.M) g.scales[(m0 + r) * ((g.N + 127) >> 7) + tile_n] = (uint8_t)byte;
#pragma unroll
            for (int i = 0; i < TF; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(uint32_t *)(rows + r * kRow + wn * WF + i * 32 + 8 * q + 4 * lhalf) =
                        e4m3_pack4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3], scale);
        });
        __syncthreads();
#pragma unroll
        for (int x = 0; x < BM * 8 / 256; ++x) {
            const int idx = x * 256 + tid, r = idx >> 3, c = (idx & 7) * 16;
            if (m0 + r < g.M && n0 + c < g.N) *(uint4v *)(g.codes + (m0 + r) * g.N + n0 + c) = *(const uint4v *)(rows + r * kRow + c);
        }
    }
#else
    (void)g;
#endif
}

template <int BM, int BN, int KIND, bool FAST, int STAGES>
static hipError_t launch_e4m3_stages(const E4m3GemmArgs &g, hipStream_t s)
{
    constexpr bool GATED = KIND >= kE4m3Silu;
    constexpr int BF = GATED ? BN / 2 : BN, main = STAGES * (BM + BN) * 128, turn = 4 * 32 * (BF / 2 * 4 + 16) + (GATED ? BM * (8 + 144) : 0);
    constexpr int smem = main > turn ? main : turn;
    static_assert(smem <= 160 * 1024, "LDS");
    // the dynamic LDS limit is raised once per kernel variant and device
    static uint64_t attr_set = 0;
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    if (((attr_set >> (dev & 63)) & 1u) == 0) {
        if (hipError_t e = hipFuncSetAttribute((const void *)e4m3_gemm_kernel<BM, BN, KIND, FAST, STAGES>, hipFuncAttributeMaxDynamicSharedMemorySize, smem)) return e;
        attr_set |= 1ull << (dev & 63);
    }
    const unsigned per_xcd = (unsigned)((g.tiles_m * (int64_t)g.tiles_n + 7) / 8);
    e4m3_gemm_kernel<BM, BN, KIND, FAST, STAGES><<<8 * per_xcd, 256, smem, s>>>(g);
    return hipGetLastError();
}

template <int BM, int BN, int KIND, bool FAST>
static hipError_t launch_e4m3_shape(E4m3GemmArgs g, hipStream_t s)
{
    constexpr int BF = KIND >= kE4m3Silu ? BN / 2 : BN;
    g.tiles_m = (int)((g.M + BM - 1) / BM);
    g.tiles_n = (int)((g.N + BF - 1) / BF);
    constexpr int few = e4m3_stages(BM, BN, FAST, 1), many = e4m3_stages(BM, BN, FAST, 1 << 30);
    if constexpr (few != many)
        if (e4m3_stages(BM, BN, FAST, g.tiles_m * (int64_t)g.tiles_n) == few) return launch_e4m3_stages<BM, BN, KIND, FAST, few>(g, s);
    return launch_e4m3_stages<BM, BN, KIND, FAST, many>(g, s);
}

template <int BM, int BN, bool FAST>
static hipError_t launch_e4m3_kind(int kind, const E4m3GemmArgs &g, hipStream_t s)
{
    if (kind == kE4m3F32) return launch_e4m3_shape<BM, BN, kE4m3F32, FAST>(g, s);
    if (kind == kE4m3Bf16) return launch_e4m3_shape<BM, BN, kE4m3Bf16, FAST>(g, s);
    if constexpr (BN == 256) {
        if (kind == kE4m3Silu) return launch_e4m3_shape<BM, BN, kE4m3Silu, FAST>(g, s);
        return launch_e4m3_shape<BM, BN, kE4m3Gelu, FAST>(g, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_e4m3_256x256(int kind, const E4m3GemmArgs &g, hipStream_t s);
hipError_t launch_e4m3_256x128(int kind, const E4m3GemmArgs &g, hipStream_t s);
hipError_t launch_e4m3_128x256(int kind, const E4m3GemmArgs &g, hipStream_t s);
hipError_t launch_e4m3_64x256(int kind, const E4m3GemmArgs &g, hipStream_t s);
hipError_t launch_e4m3_128x128(int kind, const E4m3GemmArgs &g, hipStream_t s);
hipError_t launch_e4m3_64x64(int kind, const E4m3GemmArgs &g, hipStream_t s);

}  // namespace nvfp4
