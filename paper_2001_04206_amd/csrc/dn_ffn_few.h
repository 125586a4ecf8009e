// Matrix products of few rows (at most 64): single tokens and short prompts.  All there is to do is to read the weights
// once, so nothing is staged: a workgroup takes sixteen columns (rows of W), its waves every eighth (or sixteenth) piece of 128 bytes of
// k, fragments come from memory in the lanes that multiply them, and the waves' sums meet in LDS.
#pragma once

#include "dn_ffn_tile.h"

namespace dn {

// A lane's 32 bytes of a row (which has as many), `left` elements of which exist from here on: two times sixteen, APART elements apart
// where the row is WHOLE, at a multiple of 16 bytes with all or none of the sixteen there, and else on end.  Those are settled once
// all loads of a step are out, so that no branch or wait lies between them.  Where the row ends inside, its last 32 bytes are taken,
// and zeros put in place of the elements that the piece before holds: both operands are read alike, so their products stay paired.
// WORDS: 16-bit rows may begin in the middle of a word, and the memory path then takes several cycles for each lane; the nine words
// are loaded that hold the piece (each holds some element of it), and shifted.  37 rows of 2731 by 1024, f16: 30 us as they lie, 14 so
// (11 where every row begins at a word).  A single row, whose lanes are neighbours, takes 5.5 us as it lies and 6.3 so.
template <class T> struct Any { typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T)))); };
template <class T, bool WHOLE, bool WORDS, int APART> struct Piece {
    static constexpr int E = 16 / (int)sizeof(T);
    v4u x[2];
    uint32_t more;
    // odd: whether pieces may begin in the middle of a word
    __device__ __forceinline__ void load(const T *p, int left, bool odd)
    {
        if constexpr (WHOLE) {
#pragma unroll
            for (int c = 0; c < 2; ++c) x[c] = left >= c * APART + E ? *reinterpret_cast<const v4u *>(p + c * APART) : v4u{};
        } else {
            const uintptr_t at = reinterpret_cast<uintptr_t>(p - (left >= 2 * E ? 0 : 2 * E - left));
            const uintptr_t from = WORDS ? at & ~(uintptr_t)3 : at;
#pragma unroll
            for (int c = 0; c < 2; ++c) x[c] = __builtin_bit_cast(v4u, reinterpret_cast<const typename Any<T>::type *>(from)[c]);
            if (WORDS && odd) more = reinterpret_cast<const uint32_t *>(from)[at & 2 ? 8 : 7];
        }
    }
    __device__ __forceinline__ void settle(const T *row, int left, bool odd, bool ends)
    {
        const int back = left >= 2 * E ? 0 : 2 * E - left;
        if (WORDS && odd) {
            const uint32_t by = (((uint32_t)(reinterpret_cast<uintptr_t>(row) >> 1) + back) & 1) * 16;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j / 4][j % 4] = __builtin_amdgcn_alignbit(j < 7 ? x[(j + 1) / 4][(j + 1) % 4] : more, x[j / 4][j % 4], by);
        }
        if (ends) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t v = x[j / 4][j % 4];
                if (sizeof(T) == 4) x[j / 4][j % 4] = back <= j ? v : 0u;
                else x[j / 4][j % 4] = back <= 2 * j ? v : back == 2 * j + 1 ? v & 0xffff0000u : 0u;
            }
        }
    }
};
// whether 16-bit rows may begin in the middle of a word
__device__ __forceinline__ bool odd_rows(const void *p, const void *q, int64_t ld) { return ((uintptr_t)p | (uintptr_t)q | (uintptr_t)ld) & 2; }

// MB: blocks of sixteen rows.  The matrix instructions work on sixteen rows at least; rows that do not exist repeat the last.  Bound by
// reading the weights, and past some rows by reading those again in every workgroup: 8 rows by 4096 x 8192 x 2, bf16, 29 us (4.6 TB/s), 64
// rows 58.
template <class T, int EPI, int MB, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES * 64) void few_kernel(const ProductArgs a)
{
    constexpr int PLANES = EPI == E_GATED ? 2 : 1, E = 16 / (int)sizeof(T), BK = 128 / (int)sizeof(T);
    // pieces in flight: what the registers hold, 128 where there are sixteen waves
    constexpr int AHEAD = WAVES == 8 ? (MB == 1 ? 4 : 2) : MB + PLANES <= 2 ? 4 : MB + PLANES <= 4 ? 2 : 1;
    __shared__ v4f part[WAVES][PLANES * MB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, h = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const T *w[PLANES], *x[MB];
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
        w[p] = reinterpret_cast<const T *>(static_cast<const char *>(a.b[p]) + min(n0 + i, a.N - 1) * a.ldb) + h * 2 * E;
#pragma unroll
    for (int b = 0; b < MB; ++b)
        x[b] = reinterpret_cast<const T *>(static_cast<const char *>(a.a[0]) + min(b * 16 + i, a.M - 1) * a.lda) + h * 2 * E;
    v4f acc[PLANES][MB] = {};
    const bool odd_x = odd_rows(a.a[0], a.a[0], a.lda), odd_w = odd_rows(a.b[0], a.b[PLANES - 1], a.ldb);
    for (int k0 = wave * BK; k0 < a.K; k0 += WAVES * BK * AHEAD) {
        const bool ends = !WHOLE && k0 + ((AHEAD - 1) * WAVES + 1) * BK > a.K, last = ends && (a.K & 1);   // then a row's last pieces are odd
        const bool ox = odd_x || last, ow = odd_w || last;
        Piece<T, WHOLE, !WHOLE && sizeof(T) == 2, E> fw[AHEAD][PLANES], fx[AHEAD][MB];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            const int k = k0 + s * WAVES * BK, left = a.K - k - h * 2 * E;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) fw[s][p].load(w[p] + k, left, ow);
#pragma unroll
            for (int b = 0; b < MB; ++b) fx[s][b].load(x[b] + k, left, ox);
        }
        if constexpr (!WHOLE) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                const int left = a.K - (k0 + s * WAVES * BK) - h * 2 * E;
#pragma unroll
                for (int p = 0; p < PLANES; ++p) fw[s][p].settle(w[p], left, ow, ends);
#pragma unroll
                for (int b = 0; b < MB; ++b) fx[s][b].settle(x[b], left, ox, ends);
            }
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
                    v4u rows[MB];
#pragma unroll
                    for (int b = 0; b < MB; ++b) rows[b] = fx[s][b].x[c];
                    mfma_row<T, true>(rows, fw[s][p].x[c], acc[p]);
                }
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
    side.template columns<false>(a.f, n, a.N - n);
    side.template get<false>(a.f, m, n, a.N - n);
    float v[8] = {}, u[8] = {};
#pragma unroll 4
    for (int s = 0; s < WAVES; ++s)
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
// sixteen rows, 64 bytes of each, in one load.)  Bound by memory: one row by 4096 x 8192 x 2, bf16, 27.5 us (4.9 TB/s; the matrix
// instructions' kernel 33), four rows 32, and at 4095 x 8191 x 2 27.8.
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
    constexpr int PLANES = EPI == E_GATED ? 2 : 1, E = 16 / (int)sizeof(T), ROWS = 2 * PLANES, AHEAD = ROWS + M <= 4 ? 4 : 2;
    constexpr int OWN = WHOLE ? E : 2 * E;    // elements of a kilobyte, of two where they lie at odd places, that are a lane's
    __shared__ float share[PLANES][M][8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n0 = blockIdx.x * 8;
    const T *w[ROWS], *x[M];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        w[r] = reinterpret_cast<const T *>(static_cast<const char *>(a.b[r / 2]) + min(n0 + wave * 2 + r % 2, a.N - 1) * a.ldb) + lane * OWN;
#pragma unroll
    for (int m = 0; m < M; ++m) x[m] = reinterpret_cast<const T *>(static_cast<const char *>(a.a[0]) + min(m, a.M - 1) * a.lda) + lane * OWN;
    float acc[ROWS][M] = {};
    for (int k0 = 0; k0 < a.K; k0 += 128 * E * AHEAD) {
        Piece<T, WHOLE, false, 64 * E> fw[AHEAD][ROWS], fx[AHEAD][M];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            const int k = k0 + s * 128 * E, left = a.K - k - lane * OWN;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) fw[s][r].load(w[r] + k, left, false);
#pragma unroll
            for (int m = 0; m < M; ++m) fx[s][m].load(x[m] + k, left, false);
        }
        if constexpr (!WHOLE) {
            __builtin_amdgcn_sched_barrier(0);
            const bool ends = k0 + 128 * E * AHEAD > a.K;
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                const int left = a.K - (k0 + s * 128 * E) - lane * 2 * E;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) fw[s][r].settle(w[r], left, false, ends);
#pragma unroll
                for (int m = 0; m < M; ++m) fx[s][m].settle(x[m], left, false, ends);
            }
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) acc[r][m] = dot(fw[s][r].x[c], fx[s][m].x[c], acc[r][m], T());
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
    side.template columns<false>(a.f, n0, a.N - n0);
    side.template get<false>(a.f, m, n0, a.N - n0);
    finish8<T, EPI, false>(a.f, side, m, n0, a.N - n0, v, u);
}

}  // namespace dn
