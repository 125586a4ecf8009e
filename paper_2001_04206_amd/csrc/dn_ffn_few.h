// Matrix products of few rows (at most 64): single tokens and short prompts.  All there is to do is to read the weights
// once, so nothing is staged: a workgroup takes sixteen columns (rows of W), its waves every NW-th piece of 128 bytes of k,
// fragments come from memory in the lanes that multiply them, and the waves' sums meet in LDS.
#pragma once

#include "dn_ffn_tile.h"

namespace dn {

constexpr int kFewWaves = 8;

// sixteen bytes of a row of which `left` elements exist from here on
template <class T, bool WHOLE>
__device__ __forceinline__ v4u chunk(const T *p, int left)
{
    constexpr int E = 16 / (int)sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(E), aligned(WHOLE ? 16 : sizeof(T))));
    if (left >= E) return __builtin_bit_cast(v4u, *reinterpret_cast<const Piece *>(p));
    if (WHOLE || left <= 0) return v4u{};
    Piece x;
#pragma unroll
    for (int j = 0; j < E; ++j) x[j] = j < left ? p[j] : (T)0.f;
    return __builtin_bit_cast(v4u, x);
}

// MB: blocks of sixteen rows.  The matrix instructions work on sixteen rows at least; rows that do not exist repeat the last.
template <class T, int EPI, int MB, bool WHOLE>
__global__ __launch_bounds__(kFewWaves * 64) void few_kernel(const ProductArgs a)
{
    constexpr int PLANES = EPI == E_GATED ? 2 : 1, E = 16 / (int)sizeof(T), BK = 128 / (int)sizeof(T), AHEAD = MB == 1 ? 4 : 2;
    __shared__ v4f part[kFewWaves][PLANES * MB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, h = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const T *w[PLANES], *x[MB];
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
        w[p] = reinterpret_cast<const T *>(static_cast<const char *>(a.b[p]) + min(n0 + i, a.N - 1) * a.ldb) + h * E;
#pragma unroll
    for (int b = 0; b < MB; ++b)
        x[b] = reinterpret_cast<const T *>(static_cast<const char *>(a.a[0]) + min(b * 16 + i, a.M - 1) * a.lda) + h * E;
    v4f acc[PLANES][MB] = {};
    for (int k0 = wave * BK; k0 < a.K; k0 += kFewWaves * BK * AHEAD) {
        v4u fw[AHEAD][2][PLANES], fx[AHEAD][2][MB];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int k = k0 + s * kFewWaves * BK + c * (BK / 2), left = a.K - k - h * E;
#pragma unroll
                for (int p = 0; p < PLANES; ++p) fw[s][c][p] = chunk<T, WHOLE>(w[p] + k, left);
#pragma unroll
                for (int b = 0; b < MB; ++b) fx[s][c][b] = chunk<T, WHOLE>(x[b] + k, left);
            }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int p = 0; p < PLANES; ++p)
#pragma unroll
                    for (int b = 0; b < MB; ++b) acc[p][b] = mfma(fw[s][c][p], fx[s][c][b], acc[p][b], T());
    }
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
#pragma unroll
        for (int b = 0; b < MB; ++b) part[wave][p * MB + b][lane] = acc[p][b];
    __syncthreads();
    // a thread: eight columns of one row, the lanes of two h
    const int t = threadIdx.x, m = t >> 1, n = n0 + 8 * (t & 1);
    if (t >= 32 * MB || m >= a.M || n >= a.N) return;
    Beside<T, EPI> side;
    side.template get<false>(a.f, m, n, a.N - n);
    float v[8] = {}, u[8] = {};
#pragma unroll
    for (int s = 0; s < kFewWaves; ++s)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int from = (2 * (t & 1) + q) * 16 + (m & 15);
            const v4f y = part[s][m >> 4][from], z = part[s][(PLANES - 1) * MB + (m >> 4)][from];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[4 * q + j] += y[j];
                u[4 * q + j] += z[j];
            }
        }
    finish8<T, EPI, false>(a.f, side, m, n, a.N - n, v, u);
}

}  // namespace dn
