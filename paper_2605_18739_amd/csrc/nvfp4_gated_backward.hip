// Backward pass of the gated activation h = act(g) u, quantized on the way: dg = dh u act'(g) and du = dh act(g) side by side
// as [T, 2F], along the features (the operand of the input's gradient) and along the tokens (that of the weights' gradient),
// and h again along the tokens.  Bound by HBM: 6 B read and 4 to 5 B written for each of the T F elements.
#include "nvfp4_e4m3.h"

#include <type_traits>

#include "nvfp4_kernels.h"

namespace nvfp4 {

// A workgroup takes 128 tokens x 128 features.  Lane (cg = t & 15, rg = t >> 4) holds eight features of four tokens: a block
// along the features is sixteen neighbouring lanes, one along the tokens goes over the lanes' rows (lane swaps) and the waves
// (LDS).  The codes along the tokens are turned in LDS: 16-byte chunks in an order that depends on the column.
constexpr int kGatedWaves = 8;

__device__ __forceinline__ uint32_t rows4_max(uint32_t v)       // over the four rows of sixteen lanes of a wave
{
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

template <int ACT, bool H>
__global__ __launch_bounds__(64 * kGatedWaves) void gated_backward_kernel(const GatedBackwardArgs a)
{
    constexpr int N = H ? 3 : 2;
    __shared__ uint32_t top[kGatedWaves][N][128];
    __shared__ __attribute__((aligned(16))) float inverse[N][128];
    __shared__ __attribute__((aligned(16))) uint8_t turned[N][128 * 128];
    const int t = threadIdx.x, cg = t & 15, rg = t >> 4, lane = t & 63, wave = t >> 6;
    const int64_t tiles_f = (a.F + 127) >> 7, tile_t = blockIdx.x / tiles_f, tile_f = blockIdx.x - tile_t * tiles_f;
    const int64_t t0 = tile_t * 128 + 4 * rg, f0 = tile_f * 128 + 8 * cg;
    uint4v g[4], u[4], d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = u[i] = d[i] = uint4v{0u, 0u, 0u, 0u};
        if (t0 + i < a.T && f0 < a.F) {
            g[i] = __builtin_nontemporal_load((const uint4v *)(a.gate_up + (t0 + i) * a.ld_gate_up + f0));
            u[i] = __builtin_nontemporal_load((const uint4v *)(a.gate_up + (t0 + i) * a.ld_gate_up + a.F + f0));
            d[i] = __builtin_nontemporal_load((const uint4v *)(a.dh + (t0 + i) * a.ld_dh + f0));
        }
    }
    float v[N][4][8];                                               // gradients of gate and up, and h
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float fg[8], fu[8], fd[8];
        unpack8(g[i], fg);
        unpack8(u[i], fu);
        unpack8(d[i], fd);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float slope;
            const float act = activation<ACT>(fg[k], slope);
            v[0][i][k] = fd[k] * fu[k] * slope;
            v[1][i][k] = fd[k] * act;
            if constexpr (H) v[2][i][k] = act * fu[k];
        }
    }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = t0 + i < a.T && f0 < a.F;
            const int64_t row = t0 + i, col = n * a.F + f0;
            if (a.d_bf16 && in) *(uint4v *)(a.d_bf16 + row * a.ld_d + col) = pack8(v[n][i]);
            if (a.codes) {
                uint32_t m = 0u;
#pragma unroll
                for (int k = 0; k < 8; ++k) m = max(m, abs_bits(v[n][i][k]));
                const uint32_t byte = e8m0_of_amax(row16_max(m));
                const uint2v c = e4m3_pack8(v[n][i], e8m0_inverse(byte));
                if (in) {
                    *(uint2v *)(a.codes + row * (2 * a.F) + col) = c;
                    if (cg == 0) a.scales[row * (a.F >> 6) + (col >> 7)] = (uint8_t)byte;
                }
            }
        }
    if (!a.codes_t && !(H && a.h_codes_t)) return;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t m = rows4_max(max(max(abs_bits(v[n][0][k]), abs_bits(v[n][1][k])), max(abs_bits(v[n][2][k]), abs_bits(v[n][3][k]))));
            if (lane < 16) top[wave][n][8 * cg + k] = m;
        }
    __syncthreads();
    const int64_t K = (a.T + 15) & ~15ll, nb = (K + 127) >> 7;
    auto of = [&](int n, uint8_t *&codes, uint8_t *&scales) {       // tensor n: its transposed rows of this tile
        codes = n < 2 ? a.codes_t + (n * a.F + tile_f * 128) * K : a.h_codes_t + tile_f * 128 * K;
        scales = n < 2 ? a.scales_t + (n * a.F + tile_f * 128) * nb : a.h_scales_t + tile_f * 128 * nb;
        return n < 2 ? a.codes_t != nullptr : a.h_codes_t != nullptr;
    };
    if (t < 128 * N) {
        const int n = t >> 7, col = t & 127;
        uint32_t m = top[0][n][col];
#pragma unroll
        for (int w = 1; w < kGatedWaves; ++w) m = max(m, top[w][n][col]);
        const uint32_t byte = e8m0_of_amax(m);
        inverse[n][col] = e8m0_inverse(byte);
        uint8_t *codes, *scales;
        if (of(n, codes, scales) && tile_f * 128 + col < a.F) scales[col * nb + tile_t] = (uint8_t)byte;
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float inv = inverse[n][8 * cg + k];
            *(uint32_t *)(turned[n] + (8 * cg + k) * 128 + ((((rg >> 2) ^ cg) & 7) << 4) + ((rg & 3) << 2)) =
                e4m3_pack4(v[n][0][k] * inv, v[n][1][k] * inv, v[n][2][k] * inv, v[n][3][k] * inv);
        }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        uint8_t *codes, *scales;
        if (!of(n, codes, scales)) continue;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int at = p * 512 + t, col = at >> 3, chunk = at & 7;
            const int64_t k = tile_t * 128 + chunk * 16;
            if (tile_f * 128 + col < a.F && k < K)
                *(uint4v *)(codes + col * K + k) = *(const uint4v *)(turned[n] + col * 128 + (((chunk ^ (col >> 3)) & 7) << 4));
        }
    }
}

hipError_t launch_gated_backward(const GatedBackwardArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)((a.T + 127) / 128 * ((a.F + 127) / 128));
    auto go = [&](auto kernel) { kernel<<<grid, 64 * kGatedWaves, 0, s>>>(a); };
    if (a.act == kActSilu) a.h_codes_t ? go(gated_backward_kernel<kActSilu, true>) : go(gated_backward_kernel<kActSilu, false>);
    else a.h_codes_t ? go(gated_backward_kernel<kActGelu, true>) : go(gated_backward_kernel<kActGelu, false>);
    return hipGetLastError();
}

}  // namespace nvfp4
