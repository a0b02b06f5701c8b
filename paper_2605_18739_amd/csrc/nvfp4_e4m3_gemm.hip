// Product of 8-bit operands: the form for few rows (single tokens of some sequences) and the choice of a tile shape.
#include "nvfp4_e4m3_gemm.h"

#include <algorithm>

namespace nvfp4 {

// Up to 16 MT rows of A: bound by the bytes of W.  A workgroup takes 16 rows of W (gated: 16 of the gate and the 16 of the up
// projection that belong to them), its waves cut the blocks of 128 k between them; nothing goes through LDS on the way:
//   v_mfma_f32_16x16x32_bf16 on expanded codes, W as the row operand: lane (r = lane & 15, g = lane >> 4) holds 32 of a block's k
//   of row r for four instructions.  Which k they are is free as long as A agrees: chunks g and g + 4 of 16 bytes, so that a load
//   instruction takes 64 neighbouring bytes of each row.
// The waves' sums are added in LDS in a fixed order.
constexpr int kFewWaves = 8, kFewAhead = 4;

template <int MT, bool GATED>
__global__ __launch_bounds__(64 * kFewWaves) void e4m3_few_rows_kernel(const E4m3GemmArgs g, float *__restrict__ h, int kind)
{
    constexpr int NW = GATED ? 2 : 1;
    __shared__ float4v part[kFewWaves][NW][MT][64];
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * 16, K = g.K;
    const int nb = (int)((K + 127) >> 7), b0 = nb * wave / kFewWaves, b1 = nb * (wave + 1) / kFewWaves;
    const uint8_t *w[NW], *ws[NW], *a[MT], *as[MT];
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const int64_t n = std::min(n0 + r, g.N - 1) + i * g.N;
        w[i] = g.codes_w + n * K + 16 * q;
        ws[i] = g.scales_w + (g.w_tiles ? n >> 7 : n) * nb;
    }
#pragma unroll
    for (int j = 0; j < MT; ++j) {
        const int64_t m = std::min<int64_t>(16 * j + r, g.M - 1);
        a[j] = g.codes_a + m * K + 16 * q;
        as[j] = g.scales_a + m * nb;
    }
    struct Frag {
        uint4v q[2];
    };
    struct Block {
        Frag w[NW], a[MT];
        uint32_t ws[NW], as[MT];
    };
    typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
    auto expand = [](const Frag &f, int part, uint32_t byte) {             // eight of the lane's codes, scale included
        const float scale = __uint_as_float(byte << 23);
        uint4v o;
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const uint32_t w = f.q[part >> 1][2 * (part & 1) + d];
            o[2 * d] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
            o[2 * d + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
        }
        return __builtin_bit_cast(bf16x8v, o);
    };
    auto fetch = [&](Block &x, int b) {
        const int64_t at = (int64_t)b * 128;
        const bool in0 = at + 16 * q < K, in1 = at + 64 + 16 * q < K;
        auto of = [&](Frag &f, const uint8_t *p) {
            f.q[0] = f.q[1] = uint4v{0u, 0u, 0u, 0u};
            if (in0) f.q[0] = *(const uint4v *)(p + at);
            if (in1) f.q[1] = *(const uint4v *)(p + at + 64);
        };
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            of(x.w[i], w[i]);
            x.ws[i] = ws[i][b];
        }
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            of(x.a[j], a[j]);
            x.as[j] = as[j][b];
        }
    };
    float4v acc[NW][MT];
#pragma unroll
    for (int i = 0; i < NW; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    for (int b = b0; b < b1; b += kFewAhead) {
        Block x[kFewAhead];
#pragma unroll
        for (int k = 0; k < kFewAhead; ++k) fetch(x[k], min(b + k, b1 - 1));
#pragma unroll
        for (int k = 0; k < kFewAhead; ++k)
            if (b + k < b1)
#pragma unroll
                for (int part = 0; part < 4; ++part) {
                    bf16x8v v[NW];
#pragma unroll
                    for (int i = 0; i < NW; ++i) v[i] = expand(x[k].w[i], part, x[k].ws[i]);
#pragma unroll
                    for (int j = 0; j < MT; ++j) {
                        const bf16x8v o = expand(x[k].a[j], part, x[k].as[j]);
#pragma unroll
                        for (int i = 0; i < NW; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[i], o, acc[i][j], 0, 0, 0);
                    }
                }
    }
#pragma unroll
    for (int i = 0; i < NW; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) part[wave][i][j][lane] = acc[i][j];
    __syncthreads();
    // lane (r, q) of a tile has row m = r and columns n = 4 q .. 4 q + 3
    for (int at = threadIdx.x; at < MT * 64; at += 64 * kFewWaves) {
        const int j = at >> 6, l = at & 63;
        const int64_t m = 16 * j + (l & 15), n = n0 + 4 * (l >> 4);
        if (m >= g.M) continue;
        float4v v[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            v[i] = part[0][i][j][l];
#pragma unroll
            for (int k = 1; k < kFewWaves; ++k) v[i] += part[k][i][j][l];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= g.N) break;
            if constexpr (GATED) {
                if (g.gate_up) {
                    g.gate_up[m * g.ld_gate_up + n + e] = (uint16_t)pack_bf16x2(v[0][e], 0.0f);
                    g.gate_up[m * g.ld_gate_up + g.N + n + e] = (uint16_t)pack_bf16x2(v[1][e], 0.0f);
                }
                const float act = kind == kE4m3Silu ? activation<kActSilu>(v[0][e]) : activation<kActGelu>(v[0][e]);
                const float o = act * v[1][e];
                if (g.h_bf16) g.h_bf16[m * g.ld_h + n + e] = (uint16_t)pack_bf16x2(o, 0.0f);
                if (h) h[m * g.N + n + e] = o;
            } else if (kind == kE4m3F32) ((float *)g.y)[m * g.ldy + n + e] = v[0][e];
            else ((uint16_t *)g.y)[m * g.ldy + n + e] = (uint16_t)pack_bf16x2(v[0][e], 0.0f);
        }
    }
}

// fp32 [M, F] (F % 16 == 0) -> 8 bits along F: sixteen lanes a block
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
constexpr int64_t kFewRows = 64;

size_t e4m3_gated_workspace_bytes(int64_t M, int64_t F) { return M <= kFewRows ? (size_t)M * (size_t)F * 4 : 0; }

static hipError_t launch_few_rows(int kind, const E4m3GemmArgs &g, float *h, hipStream_t s)
{
    const unsigned grid = (unsigned)((g.N + 15) / 16);
    const bool gated = kind >= kE4m3Silu;
    auto go = [&](auto kernel) { kernel<<<grid, 64 * kFewWaves, 0, s>>>(g, h, kind); };
    if (g.M <= 16) gated ? go(e4m3_few_rows_kernel<1, true>) : go(e4m3_few_rows_kernel<1, false>);
    else if (g.M <= 32) gated ? go(e4m3_few_rows_kernel<2, true>) : go(e4m3_few_rows_kernel<2, false>);
    else gated ? go(e4m3_few_rows_kernel<4, true>) : go(e4m3_few_rows_kernel<4, false>);
    if (hipError_t e = hipGetLastError()) return e;
    if (!h) return hipSuccess;
    const int64_t nb = (g.N + 127) / 128, blocks = g.M * nb;
    e4m3_rows_f32_kernel<<<(unsigned)((blocks + 15) / 16), 256, 0, s>>>(h, g.N, nb, blocks, g.codes, g.scales);
    return hipGetLastError();
}

hipError_t launch_e4m3_gemm(int kind, const E4m3GemmArgs &g, void *workspace, hipStream_t s)
{
    if (g.M <= kFewRows) return launch_few_rows(kind, g, g.codes ? static_cast<float *>(workspace) : nullptr, s);
    const bool gated = kind >= kE4m3Silu;
    // The shape whose rounds of tiles over the 256 compute units take least, by the time of a step (128 k) of a full round, ns:
    // 4096^3 takes exact 103 / 116 / 105 / 112 / 116 / 165 us with the shapes in this order, fast 56 / 73 / 70 / 69 / 77 / 109.
    struct Shape {
        int bm, bn, exact, fast;
        hipError_t (*launch)(int, const E4m3GemmArgs &, hipStream_t);
    };
    static const Shape kShapes[] = {{256, 256, 3150, 1750, launch_e4m3_256x256}, {256, 128, 1800, 1140, launch_e4m3_256x128}, {128, 256, 1640, 1090, launch_e4m3_128x256},
                                    {128, 128, 880, 540, launch_e4m3_128x128}, {64, 256, 910, 600, launch_e4m3_64x256}, {64, 64, 330, 215, launch_e4m3_64x64}};
    const Shape *best = nullptr;
    int64_t least = 0;
    for (const Shape &c : kShapes) {
        if (gated && c.bn != 256) continue;
        const int64_t bf = gated ? c.bn / 2 : c.bn, tiles = ((g.M + c.bm - 1) / c.bm) * ((g.N + bf - 1) / bf);
        const int64_t cost = (tiles + 255) / 256 * (g.fast ? c.fast : c.exact);
        if (!best || cost < least) best = &c, least = cost;
    }
    return best->launch(kind, g, s);
}

}  // namespace nvfp4
