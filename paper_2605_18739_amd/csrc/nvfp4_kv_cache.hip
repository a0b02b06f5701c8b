// The paged NVFP4 KV cache as it is written and read back, for gfx950.  Streaming kernels bound by HBM: 2 B read and
// 0.5625 B written per element on the way in, the reverse on the way out.
#include "nvfp4_device.h"

#include "nvfp4_kernels.h"

namespace nvfp4 {

constexpr int kCacheThreads = 256, kCacheWaves = kCacheThreads / kWave;

// Measured (3520 tokens of 24 heads of 128): writing 10.6 us, 5.2 TB/s, the rate of a copy; with the search 13.7, smoothed keys 12.6, both
// 16.6, the instructions of the one and the exchange of the other (a row's loads wait for its slot in all four); reading 13 us, and
// 18480 tokens 61 us, 4.8 TB/s; 33 tokens of 8 heads 2.8 and 3.1 us, latency.
// A wave works on one token of one tensor (keys or values), so the slot, the page and the page's scale with its tie tests
// are the same for all its lanes: unit = (token, tensor, part of the token's row of H * d elements).
struct CacheUnits {
    int64_t units;
    int tensors, first;                      // 2 and 0: keys and values; 1 and 0 or 1: keys or values alone
    int parts;                               // parts of a token's row
    Divisor by_parts, by_tensors, by_page;
};
struct CacheUnit {
    int64_t t, slot, page;
    int part;
    bool is_v, there, live;                  // there: a unit; live: its slot is one of the cache
    __device__ __forceinline__ CacheUnit(const CacheUnits &n, const KvPages &c, const int64_t *__restrict__ slots)
    {
        const int64_t u = (int64_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * kCacheWaves + threadIdx.x / kWave));
        there = u < n.units;
        const int64_t v = divide(there ? u : 0, n.parts, n.by_parts);
        part = (int)((there ? u : 0) - v * n.parts);
        t = divide(v, n.tensors, n.by_tensors);
        is_v = (int)(v - t * n.tensors) + n.first != 0;
        slot = slots[t];
        live = there && slot >= 0 && slot < c.n_pages * c.page_tokens;
        page = live ? divide(slot, c.page_tokens, n.by_page) : 0;
    }
};

template <bool SEARCH, bool SMOOTH>
__global__ __launch_bounds__(kCacheThreads) void kv_cache_write_kernel(const KvPages c, const CacheUnits n, const uint16_t *__restrict__ k, int64_t ldk,
                                                                       const uint16_t *__restrict__ v, int64_t ldv, const int64_t *__restrict__ slots)
{
    const int lane = threadIdx.x & (kWave - 1);
    const CacheUnit u(n, c, slots);
    if (!u.live) return;                                            // (the whole wave)
    const int nb = c.H * (c.d >> 4), b = u.part * kWave + lane;     // blocks of the row, this lane's
    const bool mine = b < nb;
    uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (mine) {
        const uint4v *p = (const uint4v *)((u.is_v ? v + u.t * ldv : k + u.t * ldk) + (b << 4));
        const uint4v v0 = p[0], v1 = p[1];
        w[0] = v0.x; w[1] = v0.y; w[2] = v0.z; w[3] = v0.w;
        w[4] = v1.x; w[5] = v1.y; w[6] = v1.z; w[7] = v1.w;
    }
    const TensorScale ts = tensor_scale(u.is_v ? c.v_global[u.page] : c.k_global[u.page]);
    if (SMOOTH && !u.is_v) {
        const int nb_row = c.d >> 4;
        const uint32_t mean = row_mean_bits(w, nb_row);
        smooth_block16(w, __uint_as_float(mean << 16));
        if (mine && (b & (nb_row - 1)) == 0) c.k_mean[u.slot * c.H + b / nb_row] = (uint16_t)mean;
    }
    if (__builtin_expect(ts.shift != 1.0f, 0)) rescale_block16(w, ts.shift);
    uint32_t sbyte, c0, c1;
    if constexpr (SEARCH) quantize_block16_4over6(w, ts, sbyte, c0, c1);
    else quantize_block16(w, ts, sbyte, c0, c1);
    if (mine) {
        const int64_t at = u.slot * nb + b;
        *(uint2v *)((u.is_v ? c.v_codes : c.k_codes) + (at << 3)) = uint2v{c0, c1};
        (u.is_v ? c.v_scales : c.k_scales)[at] = (uint8_t)sbyte;
    }
}

// A lane per half block (eight codes in, sixteen bytes out), kReadUnroll of them in flight.
constexpr int kReadUnroll = 4;
__global__ __launch_bounds__(kCacheThreads) void kv_cache_read_kernel(const KvPages c, const CacheUnits n, const int64_t *__restrict__ slots,
                                                                      uint16_t *__restrict__ k_out, uint16_t *__restrict__ v_out, int clear)
{
    const int lane = threadIdx.x & (kWave - 1);
    const CacheUnit u(n, c, slots);
    const int nb_row = c.d >> 4, nh = c.H * (c.d >> 3);             // half blocks of the row
    if (!u.live) {                                                  // (the whole wave)
        if (!u.there || !clear) return;
        uint16_t *const out = (u.is_v ? v_out : k_out) + u.t * (int64_t)(nh << 3);
        const int h0 = u.part * (kWave * kReadUnroll) + lane;
        for (int h = h0; h < min(nh, h0 + kWave * kReadUnroll); h += kWave) *(uint4v *)(out + (h << 3)) = uint4v{0u, 0u, 0u, 0u};
        return;
    }
    const int64_t at = u.slot * (int64_t)nh;
    const uint32_t *codes = (const uint32_t *)(u.is_v ? c.v_codes : c.k_codes) + at;
    const uint8_t *scales = (u.is_v ? c.v_scales : c.k_scales) + (at >> 1);
    const uint16_t *means = u.is_v || !c.k_mean ? nullptr : c.k_mean + u.slot * c.H;
    const float sg = u.is_v ? c.v_global[u.page] : c.k_global[u.page];
    uint16_t *out = (u.is_v ? v_out : k_out) + u.t * (int64_t)(nh << 3);
    const int h0 = u.part * (kWave * kReadUnroll) + lane;
    uint32_t cw[kReadUnroll], sb[kReadUnroll], mu[kReadUnroll];
#pragma unroll
    for (int i = 0; i < kReadUnroll; ++i) {
        const int h = min(h0 + i * kWave, nh - 1);
        cw[i] = codes[h];
        sb[i] = scales[h >> 1] & 0x7Fu;
        // (no mean: -0, which leaves every sum as it is, signs of zeros included)
        mu[i] = means ? (uint32_t)means[(unsigned)(h >> 1) / (unsigned)nb_row] : 0x8000u;
    }
    const bool mid = scale_is_mid(sg);
#pragma unroll
    for (int i = 0; i < kReadUnroll; ++i) {
        const int h = h0 + i * kWave;
        if (h >= nh) continue;
        const float mean = __uint_as_float(mu[i] << 16);
        uint32_t o[4];
        dequant_half_mean(cw[i], e4m3_to_f32(sb[i]), sg, mid & mean_is_mid(fabsf(mean)), mean, o);
        *(uint4v *)(out + (h << 3)) = uint4v{o[0], o[1], o[2], o[3]};
    }
}

// --------------------------------------------------------------------------
static CacheUnits cache_units(const KvPages &c, int64_t T, bool k, bool v, int parts)
{
    CacheUnits n{};
    n.tensors = (k ? 1 : 0) + (v ? 1 : 0);
    n.first = k ? 0 : 1;
    n.parts = parts;
    n.units = T * n.tensors * parts;
    n.by_parts = Divisor(parts, n.units);
    n.by_tensors = Divisor(n.tensors, n.units);
    n.by_page = Divisor(c.page_tokens, c.n_pages * c.page_tokens);
    return n;
}

hipError_t launch_kv_cache_write(const KvPages &c, const uint16_t *k, int64_t ldk, const uint16_t *v, int64_t ldv, const int64_t *slots,
                                 int64_t T, bool scale_search, hipStream_t s)
{
    const CacheUnits n = cache_units(c, T, k, v, (c.H * (c.d >> 4) + kWave - 1) / kWave);
    const unsigned grid = (unsigned)((n.units + kCacheWaves - 1) / kCacheWaves);
    const bool smooth = k && c.k_mean;
    auto go = [&](auto kernel) { kernel<<<grid, kCacheThreads, 0, s>>>(c, n, k, ldk, v, ldv, slots); };
    if (scale_search) smooth ? go(kv_cache_write_kernel<true, true>) : go(kv_cache_write_kernel<true, false>);
    else smooth ? go(kv_cache_write_kernel<false, true>) : go(kv_cache_write_kernel<false, false>);
    return hipGetLastError();
}

hipError_t launch_kv_cache_read(const KvPages &c, const int64_t *slots, int64_t T, uint16_t *k_out, uint16_t *v_out, bool clear, hipStream_t s)
{
    constexpr int per = kWave * kReadUnroll;
    const CacheUnits n = cache_units(c, T, k_out, v_out, (c.H * (c.d >> 3) + per - 1) / per);
    kv_cache_read_kernel<<<(unsigned)((n.units + kCacheWaves - 1) / kCacheWaves), kCacheThreads, 0, s>>>(c, n, slots, k_out, v_out, clear);
    return hipGetLastError();
}

}  // namespace nvfp4
