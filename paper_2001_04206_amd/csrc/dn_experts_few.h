// Experts' products where an expert has few rows: single tokens and batches of them.
#pragma once

#include "dn_experts.h"
#include "dn_ffn_few.h"
#include "dn_wave.h"

namespace dn {

// Sixteen rows of one expert a workgroup, as few_kernel's: sixteen columns, its waves every fourth or eighth piece of 128 bytes of k.  GROUP: as
// the tiles' (G_TOKENS: rows of X by the lists).  Bound by reading the matrices: 64 tokens through 8 of 64 experts, 2048 wide with 1024 hidden, bf16,
// 106 us for 537 MB (5.1 TB/s); one token 14.8 us for 67 MB, of which a third are the waits for lists, rows and matrices one after the other.
// 37 rows of 16 experts at odd widths, 1021 with 555, f16: 14.0 us with four waves, 25 with eight.
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
    Beside<T, EPI> side{};
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

// Few tokens: the last product and the sum over a row's choices in one, Y_t = R_t + sum of w (H Wd[e]^T).  A workgroup takes eight columns
// of one row, a wave every eighth choice: it reads eight rows of that expert's matrix, a kilobyte at a time, and multiplies on the vector
// unit.  Experts that several rows share are read by each of them.  One token, 8 experts of 1024 by 2048, bf16: 8.6 us (3.9 TB/s); with the
// matrix instructions, sixteen columns a workgroup, 11.7, and in two launches 9.9 and 5.2.
template <class T, bool WHOLE>
__global__ __launch_bounds__(512) void few_down_kernel(const FewDown a)
{
    constexpr int E = 16 / (int)sizeof(T), ROWS = 8;
    constexpr int OWN = WHOLE ? E : 2 * E;    // elements of a kilobyte, of two where they lie at odd places, that are a lane's
    __shared__ float part[8][ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t columns = ((uint32_t)a.N + ROWS - 1) / ROWS;
    const int t = (int)(blockIdx.x / columns), n0 = (int)(blockIdx.x % columns) * ROWS;
    float sum = 0.f;   // lane c: of column c
    for (int j = wave; j < a.k; j += 8) {
        const int p = a.place[(int64_t)t * a.k + j];
        if ((uint32_t)p >= (uint32_t)a.pairs) continue;
        int e = 0;   // the last expert that begins at or before the place
        for (int e0 = 0; e0 < a.experts; e0 += 64) {
            const int n = __popcll(__ballot(e0 + lane < a.experts && a.starts[e0 + lane] <= p));
            e += n;
            if (n < 64) break;
        }
        e = max(e - 1, 0);
        const T *x = reinterpret_cast<const T *>(static_cast<const char *>(a.h) + p * a.ldh) + lane * OWN, *w[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            w[r] = reinterpret_cast<const T *>(static_cast<const char *>(a.w) + e * a.w_stride + min(n0 + r, a.N - 1) * a.ldw) + lane * OWN;
        float acc[ROWS] = {};
        for (int k0 = 0; k0 < a.K; k0 += 128 * E) {
            Piece<T, WHOLE, false, 64 * E> fw[ROWS], fx;
            const int left = a.K - k0 - lane * OWN;
            fx.load(x + k0, left, false);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) fw[r].load(w[r] + k0, left, false);
            if constexpr (!WHOLE) {
                __builtin_amdgcn_sched_barrier(0);
                const bool ends = k0 + 128 * E > a.K;
                fx.settle(x, left, false, ends);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) fw[r].settle(w[r], left, false, ends);
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int c = 0; c < 2; ++c) acc[r] = dot(fw[r].x[c], fx.x[c], acc[r], T());
        }
        const float by = a.weight[(int64_t)t * a.k + j];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float v = wave_sum(acc[r]);
            sum += lane == r ? by * v : 0.f;
        }
    }
    if (lane < ROWS) part[wave][lane] = sum;
    __syncthreads();
    const int left = a.N - n0;
    if (threadIdx.x != 0) return;
    float v[8] = {};
    if (a.r) load8<T>(v, a.r, t * a.ldr + n0, left);
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += part[s][j];
    store8<T>(a.y, t * a.ldy + n0, v, left);
}

}  // namespace dn
