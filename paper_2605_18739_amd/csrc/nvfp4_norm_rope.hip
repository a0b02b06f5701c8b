// RMS norm of queries and keys for each head and rotation over several position axes in one pass, and its gradient, for
// gfx950.  Streaming kernels bound by HBM: 2 B read and 2 B written per element (forward), 4 B read and 2 B written (backward).
#include "nvfp4_device.h"

#include <algorithm>
#include <type_traits>

#include "nvfp4_kernels.h"

namespace nvfp4 {

constexpr int kNormThreads = 256, kNormWaves = kNormThreads / kWave;

// Sine and cosine of position * freq.  The angle in turns is taken in fp64 (a position of 31 bits times a frequency of 24,
// rounded at 53 bits: within 2^-22 of a turn at position 2^31, 2^-33 at 10^6), reduced to an eighth of a turn either way,
// |x| <= pi/4, and evaluated by the Taylor polynomials in fp32: the terms left out are below x^11/11! = 2e-9 and
// x^10/10! = 2.5e-8, less than half an fp32 ulp of the result's scale.
__device__ __forceinline__ void turn(double position, float freq, float &c, float &s)
{
    const double turns = position * (double)freq * 0.15915494309189535;
    const double quarters = 4.0 * __builtin_amdgcn_fract(turns);
    const double nearest = __builtin_rint(quarters);
    const uint32_t quadrant = (uint32_t)(int)nearest;
    const float x = (float)(quarters - nearest) * 1.57079632679f, x2 = x * x;
    float sp = __builtin_fmaf(x2, 2.7557319e-6f, -1.9841270e-4f);
    sp = __builtin_fmaf(x2, sp, 8.3333333e-3f);
    sp = __builtin_fmaf(x2, sp, -1.6666667e-1f);
    sp = __builtin_fmaf(x * x2, sp, x);
    float cp = __builtin_fmaf(x2, 2.4801587e-5f, -1.3888889e-3f);
    cp = __builtin_fmaf(x2, cp, 4.1666667e-2f);
    cp = __builtin_fmaf(x2, cp, -0.5f);
    cp = __builtin_fmaf(x2, cp, 1.0f);
    const bool odd = (quadrant & 1u) != 0u;
    const float a = odd ? sp : cp, b = odd ? cp : sp;
    c = __uint_as_float(__float_as_uint(a) ^ (((quadrant + 1u) & 2u) << 30));      // cos: negative in quadrants 1, 2
    s = __uint_as_float(__float_as_uint(b) ^ ((quadrant & 2u) << 30));             // sin: negative in quadrants 2, 3
}

// Sum over the LPR neighbouring lanes that hold a row (LPR a power of two up to 32); every lane gets it.
template <int LPR>
__device__ __forceinline__ float row_sum(float v)
{
    if constexpr (LPR > 1) v += dpp_f32<0xB1>(v);      // lane ^ 1
    if constexpr (LPR > 2) v += dpp_f32<0x4E>(v);      // lane ^ 2
    if constexpr (LPR > 4) v += dpp_f32<0x141>(v);     // the other half of eight
    if constexpr (LPR > 8) v += dpp_f32<0x140>(v);     // the other half of sixteen
    if constexpr (LPR > 16) v += __shfl_xor(v, 16, kWave);
    return v;
}

__device__ __forceinline__ void unpack8(uint4v v, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16lo_to_f32(v[i]);
        f[2 * i + 1] = bf16hi_to_f32(v[i]);
    }
}
__device__ __forceinline__ uint4v pack8(const float (&f)[8])
{
    return uint4v{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}

// What a lane knows of the rotation of its eight elements at one token.
// INTER: four pairs of neighbours, cos and sin of each.  Otherwise element e is paired with e + P (or e - P), which the
// lane `partner` holds at the same place; the sign of the sine says which of the two an element is.
template <bool INTER>
struct Turns {
    float c[INTER ? 4 : 8], s[INTER ? 4 : 8];
    int partner;
    int turned;                                          // pairs (INTER) or elements of the lane that turn, the first ones; the others pass

    // e: the lane's first element; pos: this token's positions
    __device__ __forceinline__ void load(const NormRopeArgs &a, int e, int lane, int64_t t)
    {
        constexpr int N = INTER ? 4 : 8;
        const int P = a.pairs;
        const int first = INTER ? e >> 1 : (e < P ? e : e - P);
        partner = INTER ? lane : (e < P ? lane + (P >> 3) : lane - (P >> 3));
        turned = INTER ? min(max(P - first, 0), 4) : e < 2 * P ? 8 : 0;
        if (turned == 0) partner = lane;
        double pos[kRopeMaxAxes];
#pragma unroll
        for (int x = 0; x < kRopeMaxAxes; ++x) pos[x] = x < a.axes ? (double)a.positions[t * a.axes + x] : 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = first + i;
            c[i] = 1.0f;
            s[i] = 0.0f;
            if (i < turned) {
                double p = pos[0];                       // the axis of pair j: the last one that starts at or before it
#pragma unroll
                for (int x = 1; x < kRopeMaxAxes; ++x) p = j >= a.axis_start[x] ? pos[x] : p;
                turn(p, a.freqs[j], c[i], s[i]);
                if (!INTER && e < P) s[i] = -s[i];       // (first of its pair: a cos - b sin)
            }
        }
    }
    // y -> R y, or R^T y
    template <bool TRANSPOSED>
    __device__ __forceinline__ void apply(float (&y)[8], bool any) const
    {
        if (!any) return;                                // (the same for every lane: no pairs at all)
        if constexpr (INTER) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float sn = TRANSPOSED ? -s[i] : s[i], p = y[2 * i], q = y[2 * i + 1];
                y[2 * i] = i < turned ? __builtin_fmaf(p, c[i], -(q * sn)) : p;
                y[2 * i + 1] = i < turned ? __builtin_fmaf(p, sn, q * c[i]) : q;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float o = __shfl(y[i], partner, kWave), sn = TRANSPOSED ? -s[i] : s[i];
                y[i] = turned != 0 ? __builtin_fmaf(y[i], c[i], o * sn) : y[i];
            }
        }
    }
};

// A wave takes a token and some of its heads, kWave / LPR of them at a time: LPR lanes of eight elements hold a row, so the
// sines and cosines (an fp64 product and two polynomials a pair) are made once and serve every head of the token.
// Queries come first, then keys; a turn of the loop is all queries or all keys, the next turn's loads in flight.
// Measured (17600 tokens, 24 + 24 heads of 128, three axes): 90 us, 4.8 TB/s; 8 tokens of 32 + 8 heads: 4.4 us, latency (launch,
// positions, angles, rows).
struct Unit {
    int64_t t;
    int g0, g1;
    __device__ __forceinline__ Unit(const NormRopeArgs &a, int64_t u)
    {
        t = divide(u, a.parts, a.by_parts);
        const int part = (int)(u - t * a.parts);
        g0 = part * a.groups_per_part;
        g1 = min(g0 + a.groups_per_part, a.groups_q + a.groups_k);
    }
};

template <int LPR, bool INTER>
__global__ __launch_bounds__(kNormThreads) void norm_rope_kernel(const NormRopeArgs a)
{
    constexpr int RPT = kWave / LPR;                               // rows a turn
    const int lane = threadIdx.x & (kWave - 1), col = lane & (LPR - 1), sub = lane / LPR, e = col * 8;
    const int64_t unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * kNormWaves + threadIdx.x / kWave));
    if (unit >= a.units) return;
    const Unit u(a, unit);
    const bool in_row = e < a.d;
    auto fetch = [&](int g) {
        const bool is_k = g >= a.groups_q;
        const NormRopeTensor &x = is_k ? a.k : a.q;
        const int h = (is_k ? g - a.groups_q : g) * RPT + sub;
        uint4v v = {0u, 0u, 0u, 0u};
        if (in_row && h < x.H) v = *(const uint4v *)(x.x + u.t * x.ld + (int64_t)h * a.d + e);
        return v;
    };
    uint4v next = fetch(u.g0);                                     // in flight while the angles are made
    uint4v wq = {0u, 0u, 0u, 0u}, wk = wq;
    if (in_row && a.q.weight) wq = *(const uint4v *)(a.q.weight + e);
    if (in_row && a.k.weight) wk = *(const uint4v *)(a.k.weight + e);
    Turns<INTER> turns;
    turns.load(a, e, lane, u.t);
    const float inv_d = 1.0f / (float)a.d;
    for (int g = u.g0; g < u.g1; ++g) {
        const bool is_k = g >= a.groups_q;
        const NormRopeTensor &x = is_k ? a.k : a.q;
        const int h = (is_k ? g - a.groups_q : g) * RPT + sub;
        float y[8];
        unpack8(next, y);
        if (g + 1 < u.g1) next = fetch(g + 1);
        if (x.weight) {
            float w[8], ss = 0.0f;
            unpack8(is_k ? wk : wq, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(y[i], y[i], ss);
            const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<LPR>(ss), inv_d, a.eps));
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = y[i] * r * w[i];
        }
        turns.template apply<false>(y, a.pairs > 0);
        if (in_row && h < x.H) *(uint4v *)(x.out + u.t * x.ld_out + (int64_t)h * a.d + e) = pack8(y);
    }
}

// Backward: the same units, but a workgroup takes one after another, because each leaves its sum of the weights' gradients:
// partial[workgroup][q, k][d], added in order by norm_rope_weights_kernel.  Measured (17600 tokens, 24 + 24 heads of 128): 133 us,
// 4.9 TB/s.
// WAVES: sixteen to a workgroup where that leaves a unit to a wave, four otherwise.  (777 tokens of 16 + 4 heads of 64: 146
// partial sums instead of 583, 10.6 us and 3.8 to add them instead of 9.1 and 6.4; 17600 of 24 + 24 heads of 128, where the
// workgroups go round: 142 and 5 instead of 134 and 8.)
template <int LPR, bool INTER, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void norm_rope_backward_kernel(const NormRopeArgs a, float *__restrict__ partial)
{
    constexpr int RPT = kWave / LPR;
    __shared__ float sums[WAVES][2][LPR * 8];
    const int lane = threadIdx.x & (kWave - 1), col = lane & (LPR - 1), sub = lane / LPR, e = col * 8;
    const int wave = threadIdx.x / kWave;
    const bool in_row = e < a.d;
    uint4v wq = {0u, 0u, 0u, 0u}, wk = wq;
    if (in_row && a.q.weight) wq = *(const uint4v *)(a.q.weight + e);
    if (in_row && a.k.weight) wk = *(const uint4v *)(a.k.weight + e);
    const float inv_d = 1.0f / (float)a.d;
    float dw[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[0][i] = dw[1][i] = 0.0f;
    for (int64_t n = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * WAVES + wave)); n < a.units; n += (int64_t)gridDim.x * WAVES) {
        const Unit u(a, n);
        auto fetch = [&](int g, uint4v &vx, uint4v &vd) {
            const bool is_k = g >= a.groups_q;
            const NormRopeTensor &x = is_k ? a.k : a.q;
            const int h = (is_k ? g - a.groups_q : g) * RPT + sub;
            vx = vd = uint4v{0u, 0u, 0u, 0u};
            if (in_row && h < x.H) {
                vd = *(const uint4v *)(x.dy + u.t * x.ld_dy + (int64_t)h * a.d + e);
                if (x.weight) vx = *(const uint4v *)(x.x + u.t * x.ld + (int64_t)h * a.d + e);
            }
        };
        uint4v nx, nd;
        fetch(u.g0, nx, nd);
        Turns<INTER> turns;
        turns.load(a, e, lane, u.t);
        for (int g = u.g0; g < u.g1; ++g) {
            const bool is_k = g >= a.groups_q;
            const NormRopeTensor &x = is_k ? a.k : a.q;
            const int h = (is_k ? g - a.groups_q : g) * RPT + sub;
            float y[8], xh[8];
            unpack8(nd, y);
            unpack8(nx, xh);
            if (g + 1 < u.g1) fetch(g + 1, nx, nd);
            turns.template apply<true>(y, a.pairs > 0);
            if (x.weight) {
                float w[8], ss = 0.0f, dot = 0.0f;
                unpack8(is_k ? wk : wq, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(xh[i], xh[i], ss);
                const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<LPR>(ss), inv_d, a.eps));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    xh[i] *= r;
                    const float gx = y[i] * xh[i];
                    if (is_k) dw[1][i] += gx;                      // (the same for the whole wave)
                    else dw[0][i] += gx;
                    dot = __builtin_fmaf(w[i], gx, dot);
                }
                const float mean = row_sum<LPR>(dot) * inv_d;
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = r * __builtin_fmaf(w[i], y[i], -(xh[i] * mean));
            }
            if (in_row && h < x.H) *(uint4v *)(x.out + u.t * x.ld_out + (int64_t)h * a.d + e) = pack8(y);
        }
    }
    if (!partial) return;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v = dw[which][i];
#pragma unroll
            for (int m = LPR; m < kWave; m <<= 1) v += __shfl_xor(v, m, kWave);
            if (sub == 0) sums[wave][which][e + i] = v;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.d; i += 64 * WAVES) {
        const int which = i >= a.d, c = i - which * a.d;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[w][which][c];
        partial[(int64_t)blockIdx.x * (2 * a.d) + i] = v;
    }
}

// dweight = the sum of the workgroups' partial sums: sixteen columns a workgroup, each in 64 strided parts (eight loads of
// one in flight) that are added in order.  Bound by latency: 1024 partial sums of d = 64 (0.5 MB) take 6 us, of d = 128 8 us;
// sixteen parts with one load in flight each took 15 and 21 us.
constexpr int kWeightParts = 64;

__global__ __launch_bounds__(16 * kWeightParts) void norm_rope_weights_kernel(const float *__restrict__ partial, int n, int d, float *__restrict__ dwq,
                                                                              float *__restrict__ dwk)
{
    __shared__ float part[kWeightParts][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), row = threadIdx.x >> 4;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    for (int i = row; i < n; i += 8 * kWeightParts)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int at = i + k * kWeightParts;
            if (at < n) v[k] += partial[(int64_t)at * (2 * d) + c];      // (2 d is a multiple of 16)
        }
    part[row][threadIdx.x & 15] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    __syncthreads();
    if (threadIdx.x < 16) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kWeightParts; ++i) sum += part[i][threadIdx.x];
        float *dw = c < d ? dwq : dwk;
        if (dw) dw[c < d ? c : c - d] = sum;
    }
}

// --------------------------------------------------------------------------
constexpr int kNormUnits = 4096;              // waves that fill the chip: sixteen to a compute unit
constexpr int kNormBackwardGrid = 1024;       // workgroups of the backward pass at most, each with one partial sum

size_t norm_rope_workspace_bytes(int64_t, int64_t d) { return (size_t)kNormBackwardGrid * (size_t)(2 * d) * sizeof(float); }

// heads of a token split into parts where whole tokens would be too few waves
static void plan_units(NormRopeArgs &a, int lpr, int64_t T)
{
    const int rpt = kWave / lpr;
    a.groups_q = (a.q.H + rpt - 1) / rpt;
    a.groups_k = (a.k.H + rpt - 1) / rpt;
    const int64_t groups = a.groups_q + a.groups_k;
    const int64_t parts = std::max<int64_t>(1, std::min(groups, (kNormUnits + T - 1) / T));
    a.groups_per_part = (int)((groups + parts - 1) / parts);
    a.parts = (groups + a.groups_per_part - 1) / a.groups_per_part;
    a.units = T * a.parts;
    a.by_parts = Divisor(a.parts, a.units);
}

static int lanes_per_row(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }

hipError_t launch_norm_rope(NormRopeArgs a, int64_t T, hipStream_t s)
{
    const int lpr = lanes_per_row(a.d);
    plan_units(a, lpr, T);
    const unsigned grid = (unsigned)((a.units + kNormWaves - 1) / kNormWaves);
    auto go = [&](auto kernel) { kernel<<<grid, kNormThreads, 0, s>>>(a); };
    if (lpr == 8) a.interleaved ? go(norm_rope_kernel<8, true>) : go(norm_rope_kernel<8, false>);
    else if (lpr == 16) a.interleaved ? go(norm_rope_kernel<16, true>) : go(norm_rope_kernel<16, false>);
    else a.interleaved ? go(norm_rope_kernel<32, true>) : go(norm_rope_kernel<32, false>);
    return hipGetLastError();
}

hipError_t launch_norm_rope_backward(NormRopeArgs a, int64_t T, float *dwq, float *dwk, float *partial, hipStream_t s)
{
    const int lpr = lanes_per_row(a.d);
    plan_units(a, lpr, T);
    const bool weights = dwq || dwk;
    const int waves = a.units <= kNormUnits ? 16 : 4, grid = (int)std::min<int64_t>((a.units + waves - 1) / waves, kNormBackwardGrid);
    float *p = weights ? partial : nullptr;
    auto go = [&](auto kernel) { kernel<<<grid, 64 * waves, 0, s>>>(a, p); };
    auto of_waves = [&](auto number) {
        constexpr int W = decltype(number)::value;
        if (lpr == 8) a.interleaved ? go(norm_rope_backward_kernel<8, true, W>) : go(norm_rope_backward_kernel<8, false, W>);
        else if (lpr == 16) a.interleaved ? go(norm_rope_backward_kernel<16, true, W>) : go(norm_rope_backward_kernel<16, false, W>);
        else a.interleaved ? go(norm_rope_backward_kernel<32, true, W>) : go(norm_rope_backward_kernel<32, false, W>);
    };
    if (waves == 16) of_waves(std::integral_constant<int, 16>());
    else of_waves(std::integral_constant<int, 4>());
    if (hipError_t e = hipGetLastError()) return e;
    if (!weights) return hipSuccess;
    norm_rope_weights_kernel<<<2 * a.d / 16, 16 * kWeightParts, 0, s>>>(partial, grid, a.d, dwq, dwk);
    return hipGetLastError();
}

}  // namespace nvfp4
