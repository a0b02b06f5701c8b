// Product of 8-bit operands: the form for few rows (single tokens of some sequences) and the choice of a tile shape.
#include "nvfp4_e4m3_gemm.h"

#include <algorithm>

namespace nvfp4 {

// h of a gate and an up value, and what is kept of them
__device__ __forceinline__ float gated_value(const E4m3GemmArgs &g, int kind, int64_t m, int64_t n, float gate, float up)
{
    if (g.gate_up) {
        g.gate_up[m * g.ld_gate_up + n] = (uint16_t)pack_bf16x2(gate, 0.0f);
        g.gate_up[m * g.ld_gate_up + g.N + n] = (uint16_t)pack_bf16x2(up, 0.0f);
    }
    const float o = (kind == kE4m3Silu ? activation<kActSilu>(gate) : activation<kActGelu>(gate)) * up;
    if (g.h_bf16) g.h_bf16[m * g.ld_h + n] = (uint16_t)pack_bf16x2(o, 0.0f);
    return o;
}

// Up to 16 MT rows of A: bound by the bytes of W.  A workgroup takes 16 rows of W (GATED: 16 of the gate and the 16 of the up
// projection that belong to them), its waves cut the blocks of 128 k between them and add their sums in LDS in a fixed order.
// A wave's blocks go through a ring of DEPTH slots in LDS of its own, filled by copies that write LDS directly (eight rows of 128
// bytes each, whole lines), so waves wait for their own copies only and there is no barrier on the way.  5 x 4096 x 14336 takes 12.6 us
// (4.7 TB/s), 64 rows of it 20; 8 x 2*14336 x 4096 gated 26 with the launch behind it (20 at 5.9 TB/s, and 4.8), 64 rows 33 and 4.9.  (Loads
// straight into the instruction's operands, where neighbouring lanes hold different rows, take a cycle of the address unit for each
// lane: 14, 43, 33 and 119 us.  Gated columns by the 128 to a workgroup, which would need no second launch: 41 to 49 us for 8 rows.)
//   v_mfma_f32_16x16x32_bf16 on expanded codes, W as the row operand: lane (r = lane & 15, q = lane >> 4) holds chunks q and q + 4
//   (16 bytes each) of row r for four instructions.  Chunk c of row r stands at 128 r + 16 (c ^ (r >> 1)): no bank conflicts.
//   The lane ends up with row m = r of A and columns 4 q .. 4 q + 3.
constexpr int kFewDepth = 2;                                // slots of a wave's ring
template <int MT, bool GATED, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void e4m3_few_rows_kernel(const E4m3GemmArgs g, float *__restrict__ h, int kind)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int NW = GATED ? 2 : 1, NT = NW + MT;         // tiles of 16 rows: of W, of A
    constexpr int SLOT = NT * 2048, P = 2 * NT;             // copies of a block
    constexpr int DEPTH = kFewDepth;
    static_assert(4 % DEPTH == 0, "the four blocks of a turn go round the ring");
    typedef __attribute__((address_space(3))) void *lds_ptr_t;
    typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int K = (int)g.K, nb = (K + 127) >> 7, b0 = nb * wave / WAVES, b1 = nb * (wave + 1) / WAVES;
    uint8_t *ring = lds + wave * (DEPTH * SLOT);
    const int rows_w = (int)std::min<int64_t>(16, g.N - n0), M = (int)g.M;

    // ---- copies: rows past the operands' ends, and chunks past the end of a row or of the wave's blocks, read as zeros
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void *)g.codes_a, 0, M * K, 0x00020000);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void *)(g.codes_w + n0 * K), 0, rows_w * K, 0x00020000);
    const __amdgpu_buffer_rsrc_t ru = __builtin_amdgcn_make_buffer_rsrc((void *)(g.codes_w + (GATED ? g.N + n0 : n0) * K), 0, rows_w * K, 0x00020000);
    constexpr int kPast = 1 << 30;                          // (64 rows of at most 2^22 bytes)
    int chunk_at[2], row_at[2];                             // of the copies of rows 0 .. 7 and 8 .. 15
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        chunk_at[x] = ((lane & 7) ^ ((4 * x + (lane >> 4)) & 7)) << 4;
        row_at[x] = (8 * x + (lane >> 3)) * K;
    }
    auto copy = [&](int b, int slot) {
        const int left = b < b1 ? K - b * 128 : 0;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const bool in = chunk_at[x] < left;
            const int at = row_at[x] + chunk_at[x] + b * 128;
            uint8_t *to = ring + slot * SLOT + x * 1024;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_ptr_t)to, 16, in ? at : kPast, 0, 0, 0);
            if constexpr (GATED) __builtin_amdgcn_raw_ptr_buffer_load_lds(ru, (lds_ptr_t)(to + 2048), 16, in ? at : kPast, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < MT; ++j) __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr_t)(to + (NW + j) * 2048), 16, in ? at + 16 * j * K : kPast, 0, 0, 0);
        }
    };

    // ---- scales: a word holds those of four blocks of a tile's row (any address; moved back where it would end behind the array)
    const uint8_t *scales[NT];
    int64_t scales_left[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int64_t n = n0 + std::min(r, rows_w - 1) + (i == 1 && GATED ? g.N : 0), m = std::min(16 * (i - NW) + r, M - 1);
        const int64_t at = (i < NW ? (g.w_tiles ? n >> 7 : n) : m) * nb;
        scales[i] = (i < NW ? g.scales_w : g.scales_a) + at;
        scales_left[i] = (i < NW ? g.scales_w_bytes : g.scales_a_bytes) - at;
    }
    uint32_t next_word[NT];
    auto load_words = [&](int b) {                          // of blocks b .. b + 3; bytes behind the wave's last become 0
        typedef uint32_t any_word __attribute__((aligned(1)));
        const int mine = b1 - b;
        const uint32_t keep = mine >= 4 ? 0xFFFFFFFFu : mine > 0 ? (1u << 8 * mine) - 1u : 0u;
        const int from = min(b, nb - 1);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int at = (int)std::min<int64_t>(from, scales_left[i] - 4);       // (smaller arrays take the bytes below)
            next_word[i] = *(const any_word *)(scales[i] + at) >> 8 * (from - at) & keep;
        }
    };
    auto load_bytes = [&](int b) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            uint32_t w = 0u;
            for (int k = 0; k < 4; ++k)
                if (b + k < b1) w |= (uint32_t)scales[i][b + k] << 8 * k;
            next_word[i] = w;
        }
    };
    const bool words = g.scales_a_bytes >= 4 && g.scales_w_bytes >= 4;

    float4v acc[NW][MT];
#pragma unroll
    for (int i = 0; i < NW; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    const int at0 = r * 128 + ((q ^ (r >> 1)) << 4), at1 = r * 128 + (((q + 4) ^ (r >> 1)) << 4);
    struct Frag {
        uint4v q[2];
    };
    auto expand = [](const Frag &f, int part, uint32_t word, int k) {      // eight of the lane's codes, scale (byte k of the word) included
        const float scale = __uint_as_float((word >> 8 * k & 255u) << 23);
        uint4v o;
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const uint32_t v = f.q[part >> 1][2 * (part & 1) + d];
            o[2 * d] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, false));
            o[2 * d + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, true));
        }
        return __builtin_bit_cast(bf16x8v, o);
    };
    if (b0 < b1) {
        words ? load_words(b0) : load_bytes(b0);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) copy(b0 + d, d);
    }
    for (int b = b0; b < b1; b += 4) {
        uint32_t word[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) word[i] = next_word[i];
        if (b + 4 < b1) words ? load_words(b + 4) : load_bytes(b + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            constexpr int n = (DEPTH - 1) * P;              // the copies of the blocks behind this one stay in flight
            const uint8_t *slot = ring + (k % DEPTH) * SLOT;
            NVFP4_COMPILER_FENCE();
            __builtin_amdgcn_s_waitcnt(0x0F70 | (n & 15) | (n >> 4) << 14);
            NVFP4_COMPILER_FENCE();
            Frag f[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                f[i].q[0] = *(const uint4v *)(slot + i * 2048 + at0);
                f[i].q[1] = *(const uint4v *)(slot + i * 2048 + at1);
            }
            NVFP4_COMPILER_FENCE();
            __builtin_amdgcn_s_waitcnt(0xC07F);             // lgkmcnt(0): the slot has been read
            NVFP4_COMPILER_FENCE();
            copy(b + k + DEPTH, k % DEPTH);
#pragma unroll
            for (int part = 0; part < 4; ++part) {
                bf16x8v v[NW];
#pragma unroll
                for (int i = 0; i < NW; ++i) v[i] = expand(f[i], part, word[i], k);
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    const bf16x8v o = expand(f[NW + j], part, word[NW + j], k);
#pragma unroll
                    for (int i = 0; i < NW; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[i], o, acc[i][j], 0, 0, 0);
                }
            }
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);                     // vmcnt(0): copies past the end still write the ring, which the sums take over
    __syncthreads();
    float4v *part = (float4v *)lds;                         // [WAVES][NW][MT][64]
#pragma unroll
    for (int i = 0; i < NW; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) part[((wave * NW + i) * MT + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int at = threadIdx.x; at < MT * 64; at += 64 * WAVES) {
        const int j = at >> 6, l = at & 63;
        const int64_t m = 16 * j + (l & 15), n = n0 + 4 * (l >> 4);
        if (m >= g.M) continue;
        float4v v[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            v[i] = part[(i * MT + j) * 64 + l];
#pragma unroll
            for (int k = 1; k < WAVES; ++k) v[i] += part[((k * NW + i) * MT + j) * 64 + l];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= g.N) break;
            if constexpr (GATED) {
                const float o = gated_value(g, kind, m, n + e, v[0][e], v[1][e]);
                if (h) h[m * g.N + n + e] = o;
            } else if (kind == kE4m3F32) ((float *)g.y)[m * g.ldy + n + e] = v[0][e];
            else ((uint16_t *)g.y)[m * g.ldy + n + e] = (uint16_t)pack_bf16x2(v[0][e], 0.0f);
        }
    }
#else
    (void)g, (void)h, (void)kind;
#endif
}

// fp32 [M, F] (F % 16 == 0) -> 8 bits along F: sixteen lanes a block (8 x 14336: 4.8 us, a trip to memory and a launch)
__global__ __launch_bounds__(256) void e4m3_rows_f32_kernel(const float *__restrict__ h, int64_t F, int64_t nb, int64_t blocks, uint8_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    const int64_t block = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (block >= blocks) return;                            // (whole groups of sixteen lanes)
    const int64_t m = block / nb, col = (block - m * nb) * 128 + 8 * (threadIdx.x & 15);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.0f;
    if (col < F) {
        const float4v lo = *(const float4v *)(h + m * F + col), hi = *(const float4v *)(h + m * F + col + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = lo[i], f[4 + i] = hi[i];
    }
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = abs_max(top, f[i]);
    const uint32_t byte = e8m0_of_amax(row16_max(abs_bits(top)));
    if (col < F) {
        *(uint2v *)(codes + m * F + col) = e4m3_pack8(f, e8m0_scale(byte));
        if ((threadIdx.x & 15) == 0) scales[block] = (uint8_t)byte;
    }
}

// --------------------------------------------------------------------------
size_t e4m3_gated_workspace_bytes(int64_t M, int64_t F) { return M <= kE4m3FewRows ? (size_t)M * (size_t)F * 4 : 0; }

template <int MT, bool GATED, int WAVES>
static hipError_t launch_few(int kind, const E4m3GemmArgs &g, float *h, hipStream_t s)
{
    constexpr int NW = GATED ? 2 : 1, ring = WAVES * kFewDepth * (NW + MT) * 2048, sums = WAVES * NW * MT * 1024, smem = ring > sums ? ring : sums;
    static_assert(smem <= 160 * 1024, "LDS");
    static uint64_t attr_set = 0;                           // the dynamic LDS limit is raised once per kernel variant and device
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    if (((attr_set >> (dev & 63)) & 1u) == 0) {
        if (hipError_t e = hipFuncSetAttribute((const void *)e4m3_few_rows_kernel<MT, GATED, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, smem)) return e;
        attr_set |= 1ull << (dev & 63);
    }
    e4m3_few_rows_kernel<MT, GATED, WAVES><<<(unsigned)((g.N + 15) / 16), 64 * WAVES, smem, s>>>(g, h, kind);
    return hipGetLastError();
}

static hipError_t launch_few_rows(int kind, const E4m3GemmArgs &g, float *h, hipStream_t s)
{
    const bool gated = kind >= kE4m3Silu;
    // Eight waves where a compute unit has one workgroup; with more of them fewer waves each, so that two or three workgroups
    // share its LDS and one starts while another ends.
    const bool many = (g.N + 15) / 16 > 256;
    hipError_t e;
    if (g.M <= 16) {
        if (gated) e = many ? launch_few<1, true, 4>(kind, g, h, s) : launch_few<1, true, 8>(kind, g, h, s);
        else e = many ? launch_few<1, false, 4>(kind, g, h, s) : launch_few<1, false, 8>(kind, g, h, s);
    } else if (g.M <= 32) {
        if (gated) e = many ? launch_few<2, true, 4>(kind, g, h, s) : launch_few<2, true, 8>(kind, g, h, s);
        else e = many ? launch_few<2, false, 4>(kind, g, h, s) : launch_few<2, false, 8>(kind, g, h, s);
    } else if (gated) e = many ? launch_few<4, true, 2>(kind, g, h, s) : launch_few<4, true, 4>(kind, g, h, s);
    else e = many ? launch_few<4, false, 2>(kind, g, h, s) : launch_few<4, false, 4>(kind, g, h, s);
    if (e) return e;
    if (!h) return hipSuccess;
    const int64_t nb = (g.N + 127) / 128, blocks = g.M * nb;
    e4m3_rows_f32_kernel<<<(unsigned)((blocks + 15) / 16), 256, 0, s>>>(h, g.N, nb, blocks, g.codes, g.scales);
    return hipGetLastError();
}

hipError_t launch_e4m3_gemm(int kind, const E4m3GemmArgs &g, void *workspace, hipStream_t s)
{
    if (g.M <= kE4m3FewRows) return launch_few_rows(kind, g, g.codes ? static_cast<float *>(workspace) : nullptr, s);
    static hipError_t (*const launch[kE4m3ShapeCount])(int, const E4m3GemmArgs &, hipStream_t) = {launch_e4m3_256x256, launch_e4m3_256x128, launch_e4m3_128x256,
                                                                                             launch_e4m3_128x128, launch_e4m3_64x256, launch_e4m3_64x64};
    return launch[e4m3_shape(g.M, g.N, kind >= kE4m3Silu, g.fast)](kind, g, s);
}

}  // namespace nvfp4
