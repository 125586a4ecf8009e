// Experts' products where an expert has few rows: single tokens and batches of them.
#pragma once

#include "dn_ffn_few.h"

namespace dn {

// Sixteen rows of one expert a workgroup, as few_kernel's: sixteen columns, its waves every eighth piece of 128 bytes of k.  GROUP: as the
// tiles' (G_TOKENS: rows of X by the lists).
template <class T, int EPI, int WAVES, bool WHOLE, int GROUP>
__global__ __launch_bounds__(WAVES * 64) void experts_few_kernel(const ProductArgs a)
{
    constexpr int PLANES = EPI == E_GATED ? 2 : 1, E = 16 / (int)sizeof(T), BK = 128 / (int)sizeof(T), AHEAD = 4;
    __shared__ v4f part[WAVES][PLANES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, h = lane >> 4;
    const uint32_t columns = ((uint32_t)a.N + 15) / 16;
    const GroupTile tile = tile_in_group(a.group, tiles_of(a.group, 0, 16, lane), (int)(blockIdx.x / columns), 16, lane);
    if (tile.first >= tile.end) return;
    const int n0 = (int)(blockIdx.x % columns) * 16, row = min(tile.first + i, tile.end - 1);
    const int64_t from = GROUP == G_TOKENS ? token_of(a.group, row) : row;
    const T *w[PLANES], *x = reinterpret_cast<const T *>(static_cast<const char *>(a.a[0]) + from * a.lda) + h * 2 * E;
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
        w[p] = reinterpret_cast<const T *>(static_cast<const char *>(a.b[p]) + tile.expert * a.group.b_stride + min(n0 + i, a.N - 1) * a.ldb) + h * 2 * E;
    v4f acc[PLANES][1] = {};
    const bool odd_x = odd_rows(a.a[0], a.a[0], a.lda), odd_w = odd_rows(w[0], w[PLANES - 1], a.ldb);
    for (int k0 = wave * BK; k0 < a.K; k0 += WAVES * BK * AHEAD) {
        const bool ends = !WHOLE && k0 + ((AHEAD - 1) * WAVES + 1) * BK > a.K, last = ends && (a.K & 1);   // then a row's last pieces are odd
        const bool ox = odd_x || last, ow = odd_w || last;
        Piece<T, WHOLE, !WHOLE && sizeof(T) == 2, E> fw[AHEAD][PLANES], fx[AHEAD];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            const int k = k0 + s * WAVES * BK, left = a.K - k - h * 2 * E;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) fw[s][p].load(w[p] + k, left, ow);
            fx[s].load(x + k, left, ox);
        }
        if constexpr (!WHOLE) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                const int left = a.K - (k0 + s * WAVES * BK) - h * 2 * E;
#pragma unroll
                for (int p = 0; p < PLANES; ++p) fw[s][p].settle(w[p], left, ow, ends);
                fx[s].settle(x, left, ox, ends);
            }
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
                    const v4u rows[1] = {fx[s].x[c]};
                    mfma_row<T, true>(rows, fw[s][p].x[c], acc[p]);
                }
    }
#pragma unroll
    for (int p = 0; p < PLANES; ++p) part[wave][p][lane] = acc[p][0];
    __syncthreads();
    // a thread: eight columns of one row, the lanes of two h
    const int t = threadIdx.x, m = tile.first + (t >> 1), n = n0 + 8 * (t & 1);
    if (t >= 32 || m >= tile.end || n >= a.N) return;
    Beside<T, EPI> side;
    float v[8] = {}, u[8] = {};
#pragma unroll 4
    for (int s = 0; s < WAVES; ++s)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int at = (2 * (t & 1) + q) * 16 + (t >> 1);
            const v4f y = part[s][0][at], z = part[s][PLANES - 1][at];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[4 * q + j] += y[j];
                u[4 * q + j] += z[j];
            }
        }
    finish8<T, EPI, false>(a.f, side, m, n, a.N - n, v, u);
}

}  // namespace dn
