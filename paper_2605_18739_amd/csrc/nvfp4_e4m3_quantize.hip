// Quantizers to E4M3 with one power-of-two scale for each 128 elements: along the rows, along the columns (transposed, for
// products contracted over the rows), and with a scale for each 128 x 128 tile (weights, both orders in one pass).
// Streaming kernels bound by HBM: 2 B read and 1 B (tiles with both orders: 2 B) written per element.
#include "nvfp4_e4m3.h"

#include <algorithm>

#include "nvfp4_kernels.h"

namespace nvfp4 {

// Along the rows.  A wave takes pieces of 512 neighbouring elements of a row, 8 a lane, sixteen lanes to a block; the loads of
// its kRowPieces pieces are all in flight before the first is encoded.  (3520 x 14336: 26 us, 5.8 TB/s; 17600 x 4096: 35, 6.1.)
constexpr int kRowPieces = 4;

__global__ __launch_bounds__(256) void e4m3_rows_kernel(const uint16_t *__restrict__ x, int64_t ld, int64_t C, int64_t pieces, int64_t per_row, Divisor by_per_row,
                                                        uint8_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    const int lane = threadIdx.x & 63;
    const int64_t first = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * kRowPieces, nb = (C + kE4m3Block - 1) / kE4m3Block;
    int64_t row[kRowPieces], col[kRowPieces];
    uint4v v[kRowPieces];
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const int64_t u = min(first + i, pieces - 1);
        row[i] = divide(u, per_row, by_per_row);
        col[i] = (u - row[i] * per_row) * 512 + 8 * lane;
        v[i] = uint4v{0u, 0u, 0u, 0u};
        if (col[i] < C) v[i] = __builtin_nontemporal_load((const uint4v *)(x + row[i] * ld + col[i]));
    }
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t byte = e8m0_of_amax(row16_max(absmax8_bits(v[i])));
        const uint2v c = e4m3_pack8(v[i], e8m0_scale(byte));
        if (first + i < pieces && col[i] < C) {
            *(uint2v *)(codes + row[i] * C + col[i]) = c;
            if ((lane & 15) == 0) scales[row[i] * nb + (col[i] >> 7)] = (uint8_t)byte;
        }
    }
}

// Along the columns, and by tiles: a workgroup takes 128 x 128 elements.  Lane (cg = t & 15, rg = t >> 4) holds eight columns of
// eight neighbouring rows, so its codes of a column are eight neighbouring bytes of the transposed row: they go through LDS
// (16-byte chunks in an order that depends on the column, so that neighbouring columns fall on different banks) and leave in
// whole rows of 128 bytes.
// TILES: one scale for the tile, the codes also leave in the order of x.
// (17600 x 4096 along the columns: 42 us, 5.2 TB/s; 14336 x 4096 by tiles, both orders 40 us, 5.9 TB/s, one order 30.)
template <bool TILES>
__global__ __launch_bounds__(256, 4) void e4m3_tile_kernel(const uint16_t *__restrict__ x, int64_t ld, int64_t R, int64_t C, int64_t tiles_c, int64_t K_t,
                                                        uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, uint8_t *__restrict__ codes_t,
                                                        uint8_t *__restrict__ scales_t)
{
    __shared__ __attribute__((aligned(16))) uint8_t turned[128 * 128];
    __shared__ uint32_t top[4][16][4];
    const int t = threadIdx.x, cg = t & 15, rg = t >> 4, lane = t & 63, wave = t >> 6;
    const int64_t tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x - tile_r * tiles_c, r0 = tile_r * 128 + 8 * rg, c0 = tile_c * 128 + 8 * cg;
    uint4v v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = uint4v{0u, 0u, 0u, 0u};
        if (r0 + i < R && c0 < C) v[i] = __builtin_nontemporal_load((const uint4v *)(x + (r0 + i) * ld + c0));
    }
    uint32_t m[4] = {0u, 0u, 0u, 0u};                       // largest magnitudes of the eight columns, two to a word
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) m[k] = pk_absmax_u16(m[k], v[i][k]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        m[k] = pk_absmax_u16(m[k], (uint32_t)__shfl_xor((int)m[k], 16, 64));
        m[k] = pk_absmax_u16(m[k], (uint32_t)__shfl_xor((int)m[k], 32, 64));
    }
    if (lane < 16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) top[wave][lane][k] = m[k];
    }
    __syncthreads();
    uint32_t byte[8];
    float scale[8];
    if constexpr (TILES) {
        uint32_t all = 0u;
#pragma unroll
        for (int w = 0; w < 4; ++w) all = pk_absmax_u16(all, top[w][lane >> 2][lane & 3]);
        byte[0] = e8m0_of_amax(wave_max_u32(pk_hmax_u16(all)) << 16);
        scale[0] = e8m0_scale(byte[0]);
#pragma unroll
        for (int k = 1; k < 8; ++k) scale[k] = scale[0];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t all = top[0][cg][k];
#pragma unroll
            for (int w = 1; w < 4; ++w) all = pk_absmax_u16(all, top[w][cg][k]);
            byte[2 * k] = e8m0_of_amax(all << 16);
            byte[2 * k + 1] = e8m0_of_amax(all & 0xFFFF0000u);
            scale[2 * k] = e8m0_scale(byte[2 * k]);
            scale[2 * k + 1] = e8m0_scale(byte[2 * k + 1]);
        }
    }
    uint32_t c[8][2];                                       // TILES: of a row; otherwise of a column
    if constexpr (TILES) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint2v w = e4m3_pack8(v[i], scale[0]);
            c[i][0] = w.x, c[i][1] = w.y;
            if (r0 + i < R && c0 < C) *(uint2v *)(codes + (r0 + i) * C + c0) = w;
        }
        if (t == 0) scales[tile_r * tiles_c + tile_c] = (uint8_t)byte[0];
        if (!codes_t) return;
        if (t == 0) scales_t[tile_c * ((R + 127) >> 7) + tile_r] = (uint8_t)byte[0];
        // 8 x 8 bytes turned: 4 x 4 at a time
        uint32_t d[8][2];
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint32_t w0 = c[4 * a][b], w1 = c[4 * a + 1][b], w2 = c[4 * a + 2][b], w3 = c[4 * a + 3][b];
                const uint32_t lo01 = __builtin_amdgcn_perm(w1, w0, 0x05010400u), hi01 = __builtin_amdgcn_perm(w1, w0, 0x07030602u);
                const uint32_t lo23 = __builtin_amdgcn_perm(w3, w2, 0x05010400u), hi23 = __builtin_amdgcn_perm(w3, w2, 0x07030602u);
                d[4 * b][a] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
                d[4 * b + 1][a] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
                d[4 * b + 2][a] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
                d[4 * b + 3][a] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
            }
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k][0] = d[k][0], c[k][1] = d[k][1];
    } else {
        if (rg == 0 && c0 < C) {
            const int64_t nb = (K_t + 127) >> 7;
#pragma unroll
            for (int k = 0; k < 8; ++k) scales_t[(c0 + k) * nb + tile_r] = (uint8_t)byte[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            uint32_t pair[4];                               // rows 2 i, 2 i + 1 of column k
#pragma unroll
            for (int i = 0; i < 4; ++i) pair[i] = __builtin_amdgcn_perm(v[2 * i + 1][k >> 1], v[2 * i][k >> 1], k & 1 ? 0x07060302u : 0x05040100u);
            c[k][0] = e4m3_pack4(pair[0], pair[1], scale[k]);
            c[k][1] = e4m3_pack4(pair[2], pair[3], scale[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        *(uint2v *)(turned + (8 * cg + k) * 128 + ((((rg >> 1) ^ cg) & 7) << 4) + ((rg & 1) << 3)) = uint2v{c[k][0], c[k][1]};
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int at = p * 256 + t, col = at >> 3, chunk = at & 7;
        const int64_t k = tile_r * 128 + chunk * 16;
        if (tile_c * 128 + col < C && k < K_t)
            *(uint4v *)(codes_t + (tile_c * 128 + col) * K_t + k) = *(const uint4v *)(turned + col * 128 + (((chunk ^ (col >> 3)) & 7) << 4));
    }
}

hipError_t launch_e4m3_rows(const uint16_t *x, int64_t R, int64_t C, int64_t ld, uint8_t *codes, uint8_t *scales, hipStream_t s)
{
    const int64_t per_row = (C + 511) / 512, pieces = R * per_row;
    e4m3_rows_kernel<<<(unsigned)((pieces + 4 * kRowPieces - 1) / (4 * kRowPieces)), 256, 0, s>>>(x, ld, C, pieces, per_row, Divisor(per_row, pieces), codes, scales);
    return hipGetLastError();
}

hipError_t launch_e4m3_columns(const uint16_t *x, int64_t R, int64_t C, int64_t ld, uint8_t *codes, uint8_t *scales, hipStream_t s)
{
    const int64_t tiles_c = (C + 127) / 128, tiles = (R + 127) / 128 * tiles_c;
    e4m3_tile_kernel<false><<<(unsigned)tiles, 256, 0, s>>>(x, ld, R, C, tiles_c, (R + 15) / 16 * 16, nullptr, nullptr, codes, scales);
    return hipGetLastError();
}

hipError_t launch_e4m3_tiles(const uint16_t *x, int64_t R, int64_t C, int64_t ld, uint8_t *codes, uint8_t *scales, uint8_t *codes_t, uint8_t *scales_t, hipStream_t s)
{
    const int64_t tiles_c = (C + 127) / 128, tiles = (R + 127) / 128 * tiles_c;
    e4m3_tile_kernel<true><<<(unsigned)tiles, 256, 0, s>>>(x, ld, R, C, tiles_c, R, codes, scales, codes_t, scales_t);
    return hipGetLastError();
}

}  // namespace nvfp4
