// 64x64 tiles of the product of 8-bit operands (see nvfp4_e4m3_gemm.h), for results with few tiles.
#include "nvfp4_e4m3_gemm.h"

namespace nvfp4 {

// With exact sums: the four waves cut the 128 k of a step between them, each multiplies its 32 for the whole tile, and the sums are
// added in LDS in a fixed order.  So a wave expands 128 rows of 32 k for the step, half of the codes that 32 x 32 outputs of all
// 128 k would need.  Stages, copies and the order of chunks in LDS are those of e4m3_gemm_kernel.
//   A lane (row lane & 31 of a fragment, half lane >> 5) holds chunk 2 wave + half: sixteen k, for two sub-steps.
//   Schedule of a step: one barrier (its codes are in registers, the next step's in LDS); the first sub-step reads the next step's
//   codes and expands its own second half, the second expands the next step's first half; copies go out behind the barrier.
// 777 x 1111 x 2000 takes 9.1 us (10.0 with 32 x 32 outputs to a wave), 64 x 4096 x 14336 on 64 compute units 33 (45), 4096^3 163
// (181).  A step's 16 KB take a compute unit some 215 ns to load (the step with fast sums), reads behind the barrier the rest.  Eight waves in two groups with a part of K and stages each
// took 10.1, 30 and 200; eight waves with whole blocks and a slot of their own each, without barriers, 10.3, 28 and 155.
// With fast sums there is nothing to expand, and e4m3_gemm_kernel takes the tile (8.0, 25, 115).
template <int KIND>
__global__ __launch_bounds__(256) void e4m3_split_kernel(const E4m3GemmArgs g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int STAGES = 4, STAGE = 128 * 128;
    typedef __attribute__((address_space(3))) void *lds_ptr_t;
    typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];

    // ---- tile: each of the eight chiplets (workgroup id modulo 8) takes neighbouring tiles, in groups of kGroup tile rows
    constexpr int kGroup = 8;
    const int per_xcd = (int)(gridDim.x >> 3), place = (int)(blockIdx.x & 7u) * per_xcd + (int)(blockIdx.x >> 3);
    if (place >= g.tiles_m * g.tiles_n) return;
    const int in_group = kGroup * g.tiles_n, group = place / in_group, first_m = group * kGroup, rows_m = min(kGroup, g.tiles_m - first_m);
    const int rest = place - group * in_group, tile_n = rest / rows_m, tile_m = first_m + rest - tile_n * rows_m;
    const int64_t m0 = (int64_t)tile_m * 64, n0 = (int64_t)tile_n * 64;

    const int lane = threadIdx.x & 63, lrow = lane & 31, lhalf = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int K = (int)g.K, S = (K + 127) >> 7;

    // ---- copies: rows past the operands' ends, and chunks past the end of a row, read as zeros
    const int rows_a = (int)min((int64_t)64, g.M - m0), rows_w = (int)min((int64_t)64, g.N - n0);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void *)(g.codes_a + m0 * K), 0, rows_a * K, 0x00020000);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void *)(g.codes_w + n0 * K), 0, rows_w * K, 0x00020000);
    constexpr int kPast = 0x40000000;                      // (64 rows have at most 2^28 bytes)
    int chunk_at[2];                                       // byte of the row that a lane fetches, in copies of even and odd number
#pragma unroll
    for (int p = 0; p < 2; ++p) chunk_at[p] = ((lane & 7) ^ ((4 * p + (lane >> 4)) & 7)) << 4;
    const int row_at = (lane >> 3) * K + wave * 16 * K;
    auto copy = [&](int st, int stage) {                   // rows 16 wave .. + 15 of both operands
        const int left = K - st * 128;
        uint8_t *to = lds + stage * STAGE + wave * 2048;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int from = chunk_at[p] < left ? row_at + 8 * p * K + chunk_at[p] + st * 128 : kPast;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_ptr_t)(to + p * 1024), 16, from, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr_t)(to + 8192 + p * 1024), 16, from, 0, 0, 0);
        }
    };

    // ---- scales: a word holds those of four blocks of a fragment's row (any address; moved back where it would end behind the array)
    const uint8_t *scales[4];                              // fragments: 32 rows of W, 32 more, 32 of A, 32 more
    int64_t scales_left[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
        const int r = 32 * (f & 1) + lrow;
        const int64_t n = n0 + min(r, rows_w - 1), at = (f < 2 ? (g.w_tiles ? n >> 7 : n) : m0 + min(r, rows_a - 1)) * S;
        scales[f] = (f < 2 ? g.scales_w : g.scales_a) + at;
        scales_left[f] = (f < 2 ? g.scales_w_bytes : g.scales_a_bytes) - at;
    }
    uint32_t next_word[4];
    auto load_words = [&](int b) {                         // of blocks b .. b + 3; bytes behind the row's last become 0
        const uint32_t mine = b + 4 > S ? (1u << 8 * (S - b)) - 1u : 0xFFFFFFFFu;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            typedef uint32_t any_word __attribute__((aligned(1)));
            if (g.scale_words) next_word[f] = *(const uint32_t *)(scales[f] + b);
            else if ((f < 2 ? g.scales_w_bytes : g.scales_a_bytes) >= 4) {
                const int at = (int)min((int64_t)b, scales_left[f] - 4);
                next_word[f] = *(const any_word *)(scales[f] + at) >> 8 * (b - at) & mine;
            } else {                                       // (a single word)
                uint32_t w = 0u;
                for (int k = 0; k < S; ++k) w |= (uint32_t)scales[f][k] << 8 * k;
                next_word[f] = w;
            }
        }
    };

    float16v acc[2][2];                                    // [rows of W][rows of A]
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    const int frag_at = lrow * 128 + (((2 * wave + lhalf) ^ ((lrow >> 1) & 7)) << 4);
    auto wait_and_join = [&](auto n_c) {                   // all but the last N copies have arrived, all reads are back
        constexpr int n = decltype(n_c)::value;
        NVFP4_COMPILER_FENCE();
        __builtin_amdgcn_s_waitcnt(0x0070 | (n & 15) | (n >> 4) << 14);
        __builtin_amdgcn_s_barrier();
        NVFP4_COMPILER_FENCE();
    };
    uint4v codes[2][4], frag[2][4];
    float scale[4];
    auto read = [&](int stage, int f) { return *(const uint4v *)(lds + stage * STAGE + f * 4096 + frag_at); };
    auto expand = [&](int set, int j, int f, int d) {
        const uint32_t w = codes[set][f][2 * j + (d >> 1)];
        uint32_t x = d & 1 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale[f], true))
                           : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale[f], false));
        NVFP4_PIN1(x);                                     // (where it is written: left alone it sinks to its use)
        frag[j][f][d] = x;
    };
    uint32_t word[4];
    auto take_scales = [&](int q) {                        // an E8M0 byte is the exponent of an fp32 number
#pragma unroll
        for (int f = 0; f < 4; ++f) scale[f] = __uint_as_float((word[f] >> 8 * q & 255u) << 23);
    };
    load_words(0);
#pragma unroll
    for (int f = 0; f < 4; ++f) word[f] = next_word[f];
#pragma unroll
    for (int st = 0; st < STAGES; ++st) copy(st, st);
    wait_and_join(std::integral_constant<int, 4 * (STAGES - 1)>());
#pragma unroll
    for (int f = 0; f < 4; ++f) codes[0][f] = read(0, f);
    take_scales(0);
    static_for<0, 16>([&](auto pc) { expand(0, 0, pc / 4, pc % 4); });
    // four steps (a word of scales) are one basic block, filled up with steps of zeros
    for (int s0 = 0; s0 < S; s0 += 4) {
        load_words(min(s0 + 4, (S - 1) >> 2 << 2));
        static_for<0, 8>([&](auto sub_c) {
            constexpr int q = decltype(sub_c)::value / 2, j = decltype(sub_c)::value % 2, set = q & 1;
            if constexpr (j == 0) wait_and_join(std::integral_constant<int, 4 * (STAGES - 2)>());
            else {
                if constexpr (q == 3) {
#pragma unroll
                    for (int f = 0; f < 4; ++f) word[f] = next_word[f];
                }
                take_scales((q + 1) & 3);
            }
            static_for<0, 4>([&](auto t_c) {
                constexpr int t = decltype(t_c)::value, i = t / 2, jj = t % 2;
                acc[i][jj] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8v, frag[j][i]), __builtin_bit_cast(bf16x8v, frag[j][2 + jj]), acc[i][jj], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (j == 0 && t == 0) {
#pragma unroll
                    for (int f = 0; f < 4; ++f) codes[set ^ 1][f] = read((q + 1) % STAGES, f);
                    copy(s0 + q + STAGES, q);
                }
                static_for<4 * t, 4 * t + 4>([&](auto pc) { expand(j == 0 ? set : set ^ 1, 1 - j, pc / 4, pc % 4); });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    }
    wait_and_join(std::integral_constant<int, 0>());       // (reads and copies past the end: the sums take LDS over)

    // ---- sums.  Four neighbouring columns of a row are a lane's: column 32 i + 8 q + 4 lhalf, row 32 j + lrow, of a unit (i, j, q).
    // The lane's place in the unit is moved by the column, so that sixteen threads that take a row's columns read distinct banks.
    float4v *mine = (float4v *)(lds + wave * STAGE);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                mine[((i * 2 + j) * 4 + q) * 64 + (lane ^ (i << 3 | q << 1 | lhalf))] = float4v{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __syncthreads();
    const bool whole = KIND == kE4m3F32 ? (g.ldy & 3) == 0 && ((uintptr_t)g.y & 15) == 0 : (g.ldy & 3) == 0 && ((uintptr_t)g.y & 7) == 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int at = x * 256 + (int)threadIdx.x, r = at >> 4, c = at & 15;       // row of the tile, and its columns 4 c ..
        const int unit = ((c >> 3) * 2 + (r >> 5)) * 4 + (c >> 1 & 3), from = unit * 64 + (((r & 31) | (c & 1) << 5) ^ c);
        float4v v = ((const float4v *)lds)[from];
#pragma unroll
        for (int w = 1; w < 4; ++w) v += ((const float4v *)(lds + w * STAGE))[from];
        const int64_t m = m0 + r, n = n0 + 4 * c;
        if (m >= g.M || n >= g.N) continue;
        if constexpr (KIND == kE4m3F32) {
            float *dst = (float *)g.y + m * g.ldy + n;
            if (whole && n + 4 <= g.N) *(float4v *)dst = v;
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e < g.N) dst[e] = v[e];
            }
        } else {
            uint16_t *dst = (uint16_t *)g.y + m * g.ldy + n;
            if (whole && n + 4 <= g.N) *(uint2v *)dst = uint2v{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e < g.N) dst[e] = (uint16_t)pack_bf16x2(v[e], 0.0f);
            }
        }
    }
#else
    (void)g;
#endif
}

template <int KIND>
static hipError_t launch_split(E4m3GemmArgs g, hipStream_t s)
{
    constexpr int smem = 4 * 128 * 128;
    static_assert(smem <= 64 * 1024, "dynamic LDS without raising its limit");
    g.tiles_m = (int)((g.M + 63) / 64);
    g.tiles_n = (int)((g.N + 63) / 64);
    const unsigned per_xcd = (unsigned)((g.tiles_m * (int64_t)g.tiles_n + 7) / 8);
    e4m3_split_kernel<KIND><<<8 * per_xcd, 256, smem, s>>>(g);
    return hipGetLastError();
}

hipError_t launch_e4m3_64x64(int kind, const E4m3GemmArgs &g, hipStream_t s)
{
    if (g.fast) return launch_e4m3_kind<64, 64, true>(kind, g, s);
    if (kind == kE4m3F32) return launch_split<kE4m3F32>(g, s);
    if (kind == kE4m3Bf16) return launch_split<kE4m3Bf16>(g, s);
    return hipErrorInvalidValue;
}

}  // namespace nvfp4
