// RMS norm of the residual stream with the residual's addition and an 8-bit output, and its gradient, for gfx950.
// Streaming kernels bound by HBM: forward 2 B (with a residual 4 B) read and 1 B (with the sum 3 B, with bf16 2 B more) written
// per element, backward 4 B (with the stream's gradient 6 B) read and 2 B written.
#include "nvfp4_e4m3.h"

#include <algorithm>
#include <type_traits>

#include "nvfp4_kernels.h"

namespace nvfp4 {

// Sums over a wave (ONE) or the workgroup of up to sixteen waves; every lane gets them, added in the same order everywhere.
// The lanes' sums (sixteen elements each) are fp32, they are added in fp64: ten more fp32 roundings in a row would be as large as
// all others of a result together, and each halves a share of the codes that lie next to a border.
constexpr int kNormMaxWaves = 16;

template <int CTRL>
__device__ __forceinline__ double dpp_add(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, true);
    return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

template <bool ONE, int N>
__device__ __forceinline__ void group_sum(const float (&lane_sum)[N], double (&v)[N], double (*part)[N])
{
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        v[k] = dpp_add<0xB1>((double)lane_sum[k]);
        v[k] = dpp_add<0x4E>(v[k]);
        v[k] = dpp_add<0x141>(v[k]);
        v[k] = dpp_add<0x140>(v[k]);
        v[k] += __shfl_xor(v[k], 16, 64);
        v[k] += __shfl_xor(v[k], 32, 64);
    }
    if constexpr (!ONE) {
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) part[wave][k] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = part[0][k];
            for (int w = 1; w < waves; ++w) v[k] += part[w][k];
        }
    }
}

// 1 / sqrt(v), the hardware's approximation (1 ulp) and one Newton step: y correct to about half an ulp
__device__ __forceinline__ float inverse_root(float v)
{
    const float y = __builtin_amdgcn_rsqf(v), e = __builtin_fmaf(-v * y, y, 1.0f);
    return __builtin_fmaf(0.5f * y, e, y);
}

// A workgroup takes a row, with as many waves as 1024 elements each ask for; rows of up to 1024 elements go a wave each (ONE),
// four to a workgroup.  Lane t of the row's L holds elements 8 (t + L j) .. + 7, so that sixteen lanes hold a block of 128.
// 17600 x 5120 takes 102 us with a residual and its sum (6.2 TB/s), 139 with a bf16 result as well (5.8), 53 without either (5.1);
// 8 x 4096 takes 3.6, a trip to memory and a launch.
template <bool ONE, int CH>
__global__ __launch_bounds__(ONE ? 256 : 64 * kNormMaxWaves) void rms_norm_kernel(const RmsNormArgs a)
{
    const int L = ONE ? 64 : blockDim.x;
    __shared__ double part[kNormMaxWaves][1];
    const int t = ONE ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = ONE ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (ONE && row >= a.T) return;
    uint4v x[CH], r[CH], w[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int e = 8 * (t + L * j);
        x[j] = r[j] = w[j] = uint4v{0u, 0u, 0u, 0u};
        if (e < a.C) {
            x[j] = *(const uint4v *)(a.x + row * a.ld + e);
            if (a.residual) r[j] = *(const uint4v *)(a.residual + row * a.ld_residual + e);
            w[j] = *(const uint4v *)(a.weight + e);
        }
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        float f[8];
        unpack8(x[j], f);
        if (a.residual) {                                            // the sum is rounded: it is what the later layers read
            float g[8];
            unpack8(r[j], g);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] += g[i];
            x[j] = pack8(f);
            const int e = 8 * (t + L * j);
            if (e < a.C) *(uint4v *)(a.sum + row * a.ld_sum + e) = x[j];
            unpack8(x[j], f);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = __builtin_fmaf(f[i], f[i], s[0]);
    }
    double sum[1];
    group_sum<ONE>(s, sum, part);
    const float rms = inverse_root((float)(sum[0] * a.inv_C + (double)a.eps));
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int e = 8 * (t + L * j);
        float f[8], g[8];
        unpack8(x[j], f);
        unpack8(w[j], g);
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float xh = f[i] * rms, low = __builtin_fmaf(f[i], rms, -xh);      // (what the product's rounding dropped comes back in the next one)
            f[i] = __builtin_fmaf(xh, g[i], low * g[i]);
            top = abs_max(top, f[i]);
        }
        if (a.y && e < a.C) *(uint4v *)(a.y + row * a.ld_y + e) = pack8(f);
        if (a.codes) {
            const uint32_t byte = e8m0_of_amax(row16_max(abs_bits(top)));
            const uint2v c = e4m3_pack8(f, e8m0_scale(byte));
            if (e < a.C) {
                *(uint2v *)(a.codes + row * a.C + e) = c;
                if ((t & 15) == 0) a.scales[row * ((a.C + 127) >> 7) + (e >> 7)] = (uint8_t)byte;
            }
        }
    }
}

// Backward: dx = dsum + r (w dy - xh mean(w dy xh)), xh = r x, and the workgroup's part of dweight = sum over rows of dy xh,
// which it keeps in registers over all of its rows: partial[workgroup][C].
// Rows that one wave holds go four to a workgroup, whose waves add up their parts at the end.
// 17600 x 5120 with the sum's gradient: 142 us, 5.1 TB/s; waves wait for memory in 70 % of their cycles.  (With loads and stores that
// keep the lines cached 155; with the next row's loads ahead of this one's sums the same 142.)
template <bool ONE, int CH>
__global__ __launch_bounds__(ONE ? 256 : 64 * kNormMaxWaves) void rms_norm_backward_kernel(const RmsNormArgs a, float *__restrict__ partial)
{
    constexpr int ROWS = ONE ? 4 : 1;
    const int L = ONE ? 64 : blockDim.x;
    __shared__ double part[2][kNormMaxWaves][2];
    __shared__ float waves_dw[ONE ? ROWS : 1][ONE ? CH * 512 : 1];
    const int t = ONE ? threadIdx.x & 63 : threadIdx.x, own = ONE ? threadIdx.x >> 6 : 0;
    uint4v w[CH];
    float dw[CH][8];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int e = 8 * (t + L * j);
        w[j] = uint4v{0u, 0u, 0u, 0u};
        if (e < a.C) w[j] = *(const uint4v *)(a.weight + e);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
    }
    uint4v x[CH], d[CH], r[CH];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int e = 8 * (t + L * j);
            x[j] = d[j] = r[j] = uint4v{0u, 0u, 0u, 0u};
            if (e < a.C) {
                x[j] = __builtin_nontemporal_load((const uint4v *)(a.x + row * a.ld + e));
                d[j] = __builtin_nontemporal_load((const uint4v *)(a.dy + row * a.ld_dy + e));
                if (a.residual) r[j] = __builtin_nontemporal_load((const uint4v *)(a.residual + row * a.ld_residual + e));
            }
        }
    };
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + own; row < a.T; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        fetch(row);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            float f[8], g[8], h[8];
            unpack8(x[j], f);
            unpack8(d[j], g);
            unpack8(w[j], h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[0] = __builtin_fmaf(f[i], f[i], s[0]);
                s[1] = __builtin_fmaf(g[i] * h[i], f[i], s[1]);
            }
        }
        double sum[2];
        group_sum<ONE>(s, sum, part[turn]);                        // (two places in turn: one barrier a row)
        const float rms = inverse_root((float)(sum[0] * a.inv_C + (double)a.eps)), mean = (float)(sum[1] * a.inv_C) * rms * rms;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int e = 8 * (t + L * j);
            float f[8], g[8], h[8], o[8];
            unpack8(x[j], f);
            unpack8(d[j], g);
            unpack8(w[j], h);
            unpack8(r[j], o);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[j][i] = __builtin_fmaf(g[i], f[i] * rms, dw[j][i]);
                o[i] = __builtin_fmaf(rms, __builtin_fmaf(-f[i], mean, g[i] * h[i]), o[i]);
            }
            if (e < a.C) __builtin_nontemporal_store(pack8(o), (uint4v *)(a.y + row * a.ld_y + e));
        }
    }
    if (!partial) return;
    if constexpr (ONE) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) waves_dw[own][(j * 8 + i) * 64 + t] = dw[j][i];
        __syncthreads();
        if (own > 0) return;
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int k = 1; k < ROWS; ++k) dw[j][i] += waves_dw[k][(j * 8 + i) * 64 + t];
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int e = 8 * (t + L * j);
        if (e < a.C) {
            *(float4v *)(partial + (int64_t)blockIdx.x * a.C + e) = float4v{dw[j][0], dw[j][1], dw[j][2], dw[j][3]};
            *(float4v *)(partial + (int64_t)blockIdx.x * a.C + e + 4) = float4v{dw[j][4], dw[j][5], dw[j][6], dw[j][7]};
        }
    }
}

// dweight = the partial sums added in a fixed order: sixteen columns a workgroup, 64 strided parts of each (768 parts of 5120: 7 us)
__global__ __launch_bounds__(1024) void rms_norm_weight_kernel(const float *__restrict__ partial, int n, int C, float *__restrict__ dweight)
{
    __shared__ float part[64][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), row = threadIdx.x >> 4;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    for (int i = row; i < n; i += 8 * 64)
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k * 64 < n) v[k] += partial[(int64_t)(i + k * 64) * C + c];
    part[row][threadIdx.x & 15] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    __syncthreads();
    if (threadIdx.x < 16) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 64; ++i) sum += part[i][threadIdx.x];
        dweight[c] = sum;
    }
}

// --------------------------------------------------------------------------
constexpr int kBackwardGrid = 1024;                    // workgroups of the backward pass at most, each with one partial sum

size_t rms_norm_workspace_bytes(int64_t T, int64_t C) { return (size_t)std::min<int64_t>(T, kBackwardGrid) * (size_t)C * sizeof(float); }

// f(a wave holds a row, chunks of eight elements a lane), waves of a workgroup
template <class F>
static void of_row(int64_t C, F &&f)
{
    using std::integral_constant;
    if (C <= 512) f(std::true_type(), integral_constant<int, 1>(), 4);
    else if (C <= 1024) f(std::true_type(), integral_constant<int, 2>(), 4);
    else f(std::false_type(), integral_constant<int, 2>(), (int)((C + 1023) / 1024));
}

hipError_t launch_rms_norm(const RmsNormArgs &a, hipStream_t s)
{
    of_row(a.C, [&](auto one, auto chunks, int waves) {
        constexpr bool ONE = decltype(one)::value;
        constexpr int CH = decltype(chunks)::value;
        rms_norm_kernel<ONE, CH><<<(unsigned)(ONE ? (a.T + 3) / 4 : a.T), 64 * waves, 0, s>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_rms_norm_backward(const RmsNormArgs &a, float *dweight, float *partial, hipStream_t s)
{
    int grid = 0;
    of_row(a.C, [&](auto one, auto chunks, int waves) {
        constexpr bool ONE = decltype(one)::value;
        constexpr int CH = decltype(chunks)::value;
        // as many workgroups as the chip holds at once (sixteen waves to a compute unit): more would be a second, emptier round
        grid = (int)std::min<int64_t>(ONE ? (a.T + 3) / 4 : a.T, 256 * std::min(16 / waves, 4));
        rms_norm_backward_kernel<ONE, CH><<<(unsigned)grid, 64 * waves, 0, s>>>(a, dweight ? partial : nullptr);
    });
    if (hipError_t e = hipGetLastError()) return e;
    if (!dweight) return hipSuccess;
    rms_norm_weight_kernel<<<(unsigned)(a.C / 16), 1024, 0, s>>>(partial, grid, (int)a.C, dweight);
    return hipGetLastError();
}

}  // namespace nvfp4
