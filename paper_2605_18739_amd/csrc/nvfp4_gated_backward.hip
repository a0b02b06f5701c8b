// Backward pass of the gated activation h = act(g) u, quantized on the way: dg = dh u act'(g) and du = dh act(g) side by side
// as [T, 2F], along the features (the operand of the input's gradient) and along the tokens (that of the weights' gradient),
// and h again along the tokens.  Bound by HBM: 6 B read and 4 to 5 B written for each of the T F elements.
#include "nvfp4_e4m3.h"

#include <algorithm>

#include "nvfp4_kernels.h"

namespace nvfp4 {

// A workgroup takes 128 tokens x 128 features.  Lane (cg = t & 15, rg = t >> 4) holds eight features of two tokens: a block
// along the features is sixteen neighbouring lanes, one along the tokens goes over the lanes' rows (lane swaps) and the waves
// (LDS).  The codes along the tokens are turned in LDS: 16-byte chunks in an order that depends on the column.
// Sixteen elements a lane leave room for the next tile's inputs, in flight while this one is computed: a workgroup goes from tile
// to tile, and what it computes (45 to 60 vector instructions an element, about as long as the memory needs) hides behind its loads.
// 7040 x 11008: 194 us, 4.4 TB/s; vector instructions take 54 % of the SIMDs' cycles (GELU: 203 and 62 %).  (A workgroup of half the waves to each tile, which
// ends with it: 240; half the waves that go from tile to tile spill the loads in flight: 369.)
constexpr int kGatedWaves = 16;

// Maxima of eight columns over the four rows of sixteen lanes of a wave: each exchange halves the columns that a lane keeps.
// Row r of lanes ends up with columns k + 2 (r >> 1) + 4 (r & 1) in m[k], k = 0, 1.
__device__ __forceinline__ void columns_max(uint32_t (&m)[8])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const auto x = __builtin_amdgcn_permlane16_swap(m[k], m[k + 4], false, false);
        m[k] = max((uint32_t)x[0], (uint32_t)x[1]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto x = __builtin_amdgcn_permlane32_swap(m[k], m[k + 2], false, false);
        m[k] = max((uint32_t)x[0], (uint32_t)x[1]);
    }
}

// Addresses are 32-bit offsets from the tile's first element, checked against a range, so that rows behind T need no branches
// (loaded: zeros, stored: dropped).
constexpr int kStream = 2;                                       // (the loads' streaming bit: nothing finds the inputs cached)
constexpr uint32_t kRange = 1u << 30, kPast = 1u << 30;         // (a tile: at most 128 rows 2^22 elements apart, or 2^22 bytes)

__device__ __forceinline__ __amdgpu_buffer_rsrc_t range_at(const void *p)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)kRange, 0x00020000);
}

template <int ACT, bool H>
__global__ __launch_bounds__(64 * kGatedWaves) void gated_backward_kernel(const GatedBackwardArgs a, int64_t tiles, int64_t tiles_f)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int N = H ? 3 : 2;
    __shared__ uint32_t top[kGatedWaves][N][128];
    __shared__ __attribute__((aligned(16))) float scale_of[N][128];
    __shared__ __attribute__((aligned(16))) uint8_t turned[N][128 * 128];
    // (what follows from the lane's place is made anew in each part of a turn: kept for all of them it would cost the room of the
    //  next tile's inputs, and what is fetched back from scratch waits for those)
    int place = threadIdx.x;
    auto anew = [&] { asm volatile("" : "+v"(place)); return place; };
    const int64_t K = (a.T + 15) & ~15ll, nb = (K + 127) >> 7;
    uint4v g[2], u[2], d[2];
    auto fetch = [&](int64_t tile) {
        const int64_t tile_t = tile / tiles_f, tile_f = tile - tile_t * tiles_f;
        const int rows = (int)min<int64_t>(a.T - tile_t * 128, 128), cols = (int)min<int64_t>(a.F - tile_f * 128, 128);
        const int t = anew(), cg = t & 15, rg = t >> 4;
        const uint16_t *first = a.gate_up + tile_t * 128 * a.ld_gate_up + tile_f * 128;
        const __amdgpu_buffer_rsrc_t rg_ = range_at(first), ru = range_at(first + a.F), rd = range_at(a.dh + tile_t * 128 * a.ld_dh + tile_f * 128);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool in = 2 * rg + i < rows && 8 * cg < cols;
            const uint32_t at = in ? (uint32_t)(2 * rg + i) * (uint32_t)(2 * a.ld_gate_up) + 16 * cg : kPast;
            const uint32_t at_d = in ? (uint32_t)(2 * rg + i) * (uint32_t)(2 * a.ld_dh) + 16 * cg : kPast;
            g[i] = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(rg_, at, 0, kStream));
            u[i] = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(ru, at, 0, kStream));
            d[i] = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(rd, at_d, 0, kStream));
        }
    };
    fetch(blockIdx.x);
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t tile_t = tile / tiles_f, tile_f = tile - tile_t * tiles_f;
        const int rows = (int)min<int64_t>(a.T - tile_t * 128, 128), cols = (int)min<int64_t>(a.F - tile_f * 128, 128);
        float v[N][2][8];                                           // gradients of gate and up, and h
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float gate = k & 1 ? bf16hi_to_f32(g[i][k >> 1]) : bf16lo_to_f32(g[i][k >> 1]), up = k & 1 ? bf16hi_to_f32(u[i][k >> 1]) : bf16lo_to_f32(u[i][k >> 1]);
                const float dh = k & 1 ? bf16hi_to_f32(d[i][k >> 1]) : bf16lo_to_f32(d[i][k >> 1]);
                float slope;
                const float act = activation<ACT>(gate, slope);
                v[0][i][k] = dh * up * slope;
                v[1][i][k] = dh * act;
                if constexpr (H) v[2][i][k] = act * up;
                if (k & 1) __builtin_amdgcn_sched_barrier(0);       // (two elements at a time: a row at once would not leave room for the next tile)
            }
        }
        fetch(min(tile + (int64_t)gridDim.x, tiles - 1));           // (of the last one again: no branch around loads in flight)
        __builtin_amdgcn_sched_barrier(0);
        if (a.d_bf16) {
            const int t = anew(), cg = t & 15, rg = t >> 4;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const __amdgpu_buffer_rsrc_t r = range_at(a.d_bf16 + tile_t * 128 * a.ld_d + n * a.F + tile_f * 128);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t at = 2 * rg + i < rows && 8 * cg < cols ? (uint32_t)(2 * rg + i) * (uint32_t)(2 * a.ld_d) + 16 * cg : kPast;
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, pack8(v[n][i])), r, at, 0, 0);
                }
            }
        }
        if (a.codes) {                                              // (F is a multiple of 128)
            const int t = anew(), cg = t & 15, rg = t >> 4;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int64_t col = n * a.F + tile_f * 128;
                const __amdgpu_buffer_rsrc_t rc = range_at(a.codes + tile_t * 128 * (2 * a.F) + col), rs = range_at(a.scales + tile_t * 128 * (a.F >> 6) + (col >> 7));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float m = 0.0f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) m = abs_max(m, v[n][i][k]);
                    const uint32_t byte = e8m0_of_amax(row16_max(abs_bits(m)));
                    const bool in = 2 * rg + i < rows;
                    __builtin_amdgcn_raw_buffer_store_b64(e4m3_pack8(v[n][i], e8m0_scale(byte)), rc, in ? (uint32_t)(2 * rg + i) * (uint32_t)(2 * a.F) + 8 * cg : kPast, 0, 0);
                    __builtin_amdgcn_raw_buffer_store_b8((uint8_t)byte, rs, in && cg == 0 ? (uint32_t)(2 * rg + i) * (uint32_t)(a.F >> 6) : kPast, 0, 0);
                }
            }
        }
        if (!a.codes_t && !(H && a.h_codes_t)) continue;
        const int t = anew(), cg = t & 15, rg = t >> 4, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
        const int row = lane >> 4;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t m[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) m[k] = abs_bits(abs_max(abs_max(0.0f, v[n][0][k]), v[n][1][k]));
            columns_max(m);
#pragma unroll
            for (int k = 0; k < 2; ++k) top[wave][n][8 * cg + k + 2 * (row >> 1) + 4 * (row & 1)] = m[k];
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
        auto of = [&](int n, const uint8_t *&codes, uint8_t *&scales) {     // tensor n: its transposed rows of this tile
            codes = n < 2 ? a.codes_t + (n * a.F + tile_f * 128) * K + tile_t * 128 : a.h_codes_t + tile_f * 128 * K + tile_t * 128;
            scales = n < 2 ? a.scales_t + (n * a.F + tile_f * 128) * nb : a.h_scales_t + tile_f * 128 * nb;
            return n < 2 ? a.codes_t != nullptr : a.h_codes_t != nullptr;
        };
        if (t < 128 * N) {
            const int n = t >> 7, col = t & 127;
            uint32_t m = top[0][n][col];
#pragma unroll
            for (int w = 1; w < kGatedWaves; ++w) m = max(m, top[w][n][col]);
            const uint32_t byte = e8m0_of_amax(m);
            scale_of[n][col] = e8m0_scale(byte);
            const uint8_t *codes;
            uint8_t *scales;
            if (of(n, codes, scales) && col < cols) scales[col * nb + tile_t] = (uint8_t)byte;
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // two lanes of neighbouring rows hold four tokens of columns k and k + 4: one gets column k whole, the other k + 4
                const uint32_t lo = e4m3_pack2(v[n][0][k], v[n][1][k], scale_of[n][8 * cg + k]), hi = e4m3_pack2(v[n][0][k + 4], v[n][1][k + 4], scale_of[n][8 * cg + k + 4]);
                const auto x = __builtin_amdgcn_permlane16_swap(lo, hi, false, false);
                *(uint32_t *)(turned[n] + (8 * cg + k + (rg & 1) * 4) * 128 + ((((rg >> 3) ^ cg) & 7) << 4) + ((rg >> 1 & 3) << 2)) =
                    __builtin_amdgcn_perm((uint32_t)x[1], (uint32_t)x[0], 0x05040100u);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();                                            // (the next tile's maxima and codes: behind its own barriers)
        const int out = anew();
        const int left = (int)min<int64_t>(K - tile_t * 128, 128);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint8_t *codes;
            uint8_t *scales;
            if (!of(n, codes, scales)) continue;
            const __amdgpu_buffer_rsrc_t r = range_at(codes);
            const int col = out >> 3, chunk = out & 7;
            __builtin_amdgcn_raw_buffer_store_b128(*(const uint4v *)(turned[n] + col * 128 + (((chunk ^ (col >> 3)) & 7) << 4)), r,
                                                   col < cols && chunk * 16 < left ? (uint32_t)col * (uint32_t)K + chunk * 16 : kPast, 0, 0);
        }
    }
#else
    (void)a, (void)tiles, (void)tiles_f;
#endif
}

hipError_t launch_gated_backward(const GatedBackwardArgs &a, hipStream_t s)
{
    const int64_t tiles_f = (a.F + 127) / 128, tiles = (a.T + 127) / 128 * tiles_f;
    const unsigned grid = (unsigned)std::min<int64_t>(tiles, 256);
    auto go = [&](auto kernel) { kernel<<<grid, 64 * kGatedWaves, 0, s>>>(a, tiles, tiles_f); };
    if (a.act == kActSilu) a.h_codes_t ? go(gated_backward_kernel<kActSilu, true>) : go(gated_backward_kernel<kActSilu, false>);
    else a.h_codes_t ? go(gated_backward_kernel<kActGelu, true>) : go(gated_backward_kernel<kActGelu, false>);
    return hipGetLastError();
}

}  // namespace nvfp4
