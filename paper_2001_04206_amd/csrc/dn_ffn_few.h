// Matrix products of few rows (at most 64): single tokens and short prompts.  All there is to do is to read the weights
// once, so nothing is staged: a workgroup takes sixteen columns (rows of W), its waves every eighth piece of 128 bytes of k,
// fragments come from memory in the lanes that multiply them, and the waves' sums meet in LDS.
#pragma once

#include "dn_ffn_tile.h"

namespace dn {

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

constexpr int kFewWaves = 8;
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
                for (int p = 0; p < PLANES; ++p) mfma_row<T, true>(fx[s][c], fw[s][c][p], acc[p]);
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

// Up to four rows: single tokens.  Vector instructions suffice, so a wave reads whole rows of W, a kilobyte at a time, and every
// line of memory is asked for once: four waves of two rows, eight columns a workgroup.  (The matrix instructions' layout asks for
// sixteen rows, 64 bytes of each, in one load.)
__device__ __forceinline__ float dot(const v4u &a, const v4u &b, float c, bf16)
{
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = a[j], y = b[j];
        c = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2b, x), __builtin_bit_cast(v2b, y), c, false);
    }
    return c;
}
__device__ __forceinline__ float dot(const v4u &a, const v4u &b, float c, f16)
{
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = a[j], y = b[j];
        c = __builtin_amdgcn_fdot2(__builtin_bit_cast(v2h, x), __builtin_bit_cast(v2h, y), c, false);
    }
    return c;
}
__device__ __forceinline__ float dot(const v4u &a, const v4u &b, float c, float)
{
    const v4f x = __builtin_bit_cast(v4f, a), y = __builtin_bit_cast(v4f, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = fmaf(x[j], y[j], c);
    return c;
}

template <class T, int EPI, int M, bool WHOLE>
__global__ __launch_bounds__(256) void token_kernel(const ProductArgs a)
{
    constexpr int PLANES = EPI == E_GATED ? 2 : 1, E = 16 / (int)sizeof(T), ROWS = 2 * PLANES, AHEAD = ROWS + M <= 4 ? 8 : 4;
    __shared__ float share[PLANES][M][8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n0 = blockIdx.x * 8;
    const T *w[ROWS], *x[M];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        w[r] = reinterpret_cast<const T *>(static_cast<const char *>(a.b[r / 2]) + min(n0 + wave * 2 + r % 2, a.N - 1) * a.ldb) + lane * E;
#pragma unroll
    for (int m = 0; m < M; ++m) x[m] = reinterpret_cast<const T *>(static_cast<const char *>(a.a[0]) + min(m, a.M - 1) * a.lda) + lane * E;
    float acc[ROWS][M] = {};
    for (int k0 = 0; k0 < a.K; k0 += 64 * E * AHEAD) {
        v4u fw[AHEAD][ROWS], fx[AHEAD][M];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            const int k = k0 + s * 64 * E, left = a.K - k - lane * E;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) fw[s][r] = chunk<T, WHOLE>(w[r] + k, left);
#pragma unroll
            for (int m = 0; m < M; ++m) fx[s][m] = chunk<T, WHOLE>(x[m] + k, left);
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int m = 0; m < M; ++m) acc[r][m] = dot(fw[s][r], fx[s][m], acc[r][m], T());
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) {
            float v = acc[r][m];
#pragma unroll
            for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
            if (lane == 0) share[r / 2][m][wave * 2 + r % 2] = v;
        }
    __syncthreads();
    const int m = threadIdx.x;
    if (m >= a.M || m >= M) return;
    float v[8], u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] = share[0][m][j];
        u[j] = share[PLANES - 1][m][j];
    }
    Beside<T, EPI> side;
    side.template get<false>(a.f, m, n0, a.N - n0);
    finish8<T, EPI, false>(a.f, side, m, n0, a.N - n0, v, u);
}

}  // namespace dn
