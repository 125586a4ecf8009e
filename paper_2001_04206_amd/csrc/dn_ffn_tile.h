// Matrix products in tiles on the matrix instructions, 32-bit, f16 and bf16 operands, with the block's epilogues.
//
// The geometry is one in bytes: a stage holds 128 bytes of k (64 16-bit numbers, 32 fp32 ones) of every row of both tiles,
// a lane's fragment is 16 bytes (eight k of v_mfma_f32_16x16x32, or four of v_mfma_f32_16x16x4_f32 in four instructions).
// The matrix instruction's first operand is the N side, so that a lane holds four consecutive columns of one row of C:
// lane = 16 h + i: D register r is column 4 h + r, row i.
//
// Bound by the matrix instructions and, as the chip's power limit sets its clock, by what feeds them.  Measured: a gated block of 8192 rows,
// 4096 wide with 8192 hidden, bf16, 831 + 410 us forward (1330 TFLOP/s; a library product of 8192 x 8192 x 8192 reaches 1500; by card and
// warmth up to 897 + 438), its four products backward 509 + 763 + 750 + 379 (1440 to 1470 but for the first, whose epilogue moves 655 MB);
// fp32 2048 x 1024 x 4096 at 115 of the library's 154.
#pragma once

#include <type_traits>

#include "dn_ffn.h"

namespace dn {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

__device__ __forceinline__ v4f mfma(const v4u &a, const v4u &b, v4f c, bf16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
}
__device__ __forceinline__ v4f mfma(const v4u &a, const v4u &b, v4f c, f16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}
// a row of N blocks: their products with one fragment.  fp32's four instructions a block go round the blocks: one that adds to
// the sums of the one before would wait for it.  SECOND: the blocks' fragments are the second operand.
template <class T, bool SECOND, int N>
__device__ __forceinline__ void mfma_row(const v4u (&b)[N], const v4u &a, v4f (&c)[N])
{
    if constexpr (sizeof(T) == 4) {
        const v4f y = __builtin_bit_cast(v4f, a);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const v4f x = __builtin_bit_cast(v4f, b[j]);
                c[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(SECOND ? y[q] : x[q], SECOND ? x[q] : y[q], c[j], 0, 0, 0);
            }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) c[j] = SECOND ? mfma(a, b[j], c[j], T()) : mfma(b[j], a, c[j], T());
    }
}
// c plus the sum of a fragment's elements
__device__ __forceinline__ float add_all(const v4u &a, float c, bf16)
{
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t two = a[j];   // (a cast of a[j] itself reads a[0])
        c = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2b, two), v2b{(bf16)1.f, (bf16)1.f}, c, false);
    }
    return c;
}
__device__ __forceinline__ float add_all(const v4u &a, float c, f16)
{
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t two = a[j];
        c = __builtin_amdgcn_fdot2(__builtin_bit_cast(v2h, two), v2h{(f16)1.f, (f16)1.f}, c, false);
    }
    return c;
}
__device__ __forceinline__ float add_all(const v4u &a, float c, float)
{
    const v4f x = __builtin_bit_cast(v4f, a);
    return c + ((x[0] + x[1]) + (x[2] + x[3]));
}

// ---- epilogues -------------------------------------------------------------------------------------------------------

// What the epilogue of row m, columns n .. n + 7 of N (n a multiple of 8, n < N) reads: the residual; G and U.  Apart from
// finish8 so that a thread's reads of several rows can be under way together.  ALL: all eight columns exist.
template <class T, int EPI>
struct Beside {
    typename Eight<T>::type r, u;    // a row's
    typename Eight<T>::type b, b2;   // its columns'
    template <bool ALL>
    __device__ __forceinline__ void columns(const Finish &e, int n, int left)
    {
        if ((EPI == E_LINEAR || EPI == E_GATED) && e.bias) b = get8<T, ALL>(e.bias, n, left);
        if (EPI == E_GATED && e.bias2) b2 = get8<T, ALL>(e.bias2, n, left);
    }
    template <bool ALL>
    __device__ __forceinline__ void get(const Finish &e, int m, int n, int left)
    {
        if (EPI == E_LINEAR && e.r) r = get8<T, ALL>(e.r, m * e.ldr + n, left);
        if (EPI == E_DGATED) {
            r = get8<T, ALL>(e.r, m * e.ldr + n, left);
            u = get8<T, ALL>(e.r, m * e.ldr + n + e.half, left);
        }
    }
};

// The epilogue: `v` the sums, E_GATED: `w` those of the second matrix.  All of it is fp32, and each result is rounded once.  H, dG and dU
// are rounded to T because the next product reads them as operands of the 16-bit matrix instruction: one more rounding in what comes of
// them, the biases' gradients among it, which are sums of the same operands.  The activation's derivative is taken of G and U as the
// forward call stored them.  Whole tiles' results other than Y stream past the L2, which leaves it to the operands: backward of 1024 rows,
// 2048 wide with 4096 hidden, 170 -> 162 us; not those of the gated product, whose rows of 64 bytes are half lines (903 -> 945 us at 8192
// rows, 4096 wide with 8192 hidden).
template <class T, int EPI, bool ALL>
__device__ __forceinline__ void finish8(const Finish &e, const Beside<T, EPI> &side, int m, int n, int left, float (&v)[8], float (&w)[8])
{
    constexpr bool FAST = sizeof(T) == 2;
    if constexpr (EPI == E_LINEAR) {
        if (e.bias)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += (float)side.b[j];
        if (e.y2) store8<T, ALL, ALL>(e.y2, m * e.ldy2 + n, v, left);
        float f[8], df[8];
        act8<FAST>(e.act, v, f, df);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = f[j];
        if (e.drop.t) drop8(e.drop, m, n, v);
        if (e.r)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += (float)side.r[j];
        store8<T, ALL>(e.y, m * e.ldy + n, v, left);
    } else if constexpr (EPI == E_GATED) {
        if (e.bias)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += (float)side.b[j];
        if (e.bias2)
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] += (float)side.b2[j];
        if (e.y2) {
            store8<T, ALL>(e.y2, m * e.ldy2 + n, v, left);
            store8<T, ALL>(e.y2, m * e.ldy2 + n + e.half, w, left);
        }
        float f[8], df[8];
        act8<FAST>(e.act, v, f, df);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = !ALL && j >= left ? 0.f : f[j] * w[j];
        store8<T, ALL>(e.y, m * e.ldy + n, v, left + e.zeros);
    } else if constexpr (EPI == E_DGATED) {
        float g[8], f[8], df[8], h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = (float)side.r[j];
        act8<FAST>(e.act, g, f, df);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] *= e.alpha;
            w[j] = v[j] * f[j];
            v[j] *= (float)side.u[j] * df[j];
            h[j] = (float)side.u[j] * f[j];
            if (!ALL && j >= left) v[j] = w[j] = h[j] = 0.f;
        }
        store8<T, ALL, ALL>(e.y, m * e.ldy + n, v, left + e.zeros);
        store8<T, ALL, ALL>(e.y, m * e.ldy + n + e.half_y, w, left + e.zeros);
        store8<T, ALL, ALL>(e.y2, m * e.ldy2 + n, h, left + e.zeros);
    } else {
        const int row = m < e.m_split ? m : m - e.m_split;
        if (row >= e.m_valid) return;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= e.alpha;
        void *y = m < e.m_split ? e.y : e.y2;
        const int64_t at = row * (m < e.m_split ? e.ldy : e.ldy2) + n;
        if (e.f32_out) store8<float, ALL, ALL>(y, at, v, left);
        else store8<T, ALL, ALL>(y, at, v, left);
    }
}
template <class T>
__device__ __forceinline__ void finish_sum(const Finish &e, int m, float v)
{
    void *p = m < e.m_split ? e.sums : e.sums2;
    const int at = m < e.m_split ? m : m - e.m_split;
    if (at >= e.m_valid || !p) return;
    if (e.f32_out) static_cast<float *>(p)[at] = v * e.alpha;
    else static_cast<T *>(p)[at] = (T)(v * e.alpha);
}

// ---- operands ----------------------------------------------------------------------------------------------------------

// One operand's stage of R rows in LDS, R * 128 bytes, filled by NW waves in pieces of 1024 bytes (wave w: pieces w, w + NW, ..).
//   KC: row r at 128 r, its 16-byte chunk c at c ^ ((r >> 1) & 7).
//   MC, fp32: k at k R 4, its 64-byte units u at u ^ ((k >> 2) & 3).
//   MC, 16-bit, 128 rows: k at k 256, its 32-byte units u at u ^ ((k & 3) + 4 ((k >> 3) & 1)).
//   MC, 16-bit, 256 rows (PAD): 32 bytes more after every piece, which is two k, and the units of odd k at u ^ 2.
// Each spreads what the lanes of one read touch over all banks; the last one's reads have their blocks at constant
// distances of two addresses, where an exclusive-or of three bits would take an address register for each of eight blocks.
// PAIR (KC): rows 0..15, 32..47, .. are of the first matrix, the rows between them of the second.
template <class T, int R, int NW, bool MC, bool PAIR>
struct Operand {
    static constexpr bool MC_ = MC;
    static constexpr int Q = R / 8 / NW;             // pieces of a wave
    static constexpr int BK = 128 / (int)sizeof(T);  // k of a stage
    static constexpr int RB = R * (int)sizeof(T);    // MC: bytes of a k
    static constexpr bool PAD = MC && sizeof(T) == 2 && R == 256;
    static constexpr int PIECE = PAD ? 1056 : 1024, STAGE = R / 8 * PIECE;
    static constexpr int READS = MC ? (sizeof(T) == 2 ? 2 : 4) : 1;   // LDS instructions of a fragment
    static_assert(!MC || RB >= 256, "the exclusive-or of MC needs rows of 256 bytes");
    static constexpr bool HOP = !MC || sizeof(T) == 2;   // the lane's chunks lie one distance apart
    uint32_t off[HOP ? 1 : Q], hop;   // byte offsets of the lane's chunks in the first stage of a segment
    uint32_t kbyte;    // KC: its byte within the stage's k
    const char *base, *next;   // first row of the tile, in this segment and the second one
    int64_t ld;
    int rows;          // rows of the tile that exist

    __device__ __forceinline__ uint32_t offset(int q) const { return HOP ? off[0] + q * hop : off[HOP ? 0 : q]; }

    // `wave` and everything but `lane` are uniform
    __device__ __forceinline__ void init(const void *const (&p)[2], int64_t ld_, int row0, int total, int wave, int lane)
    {
        ld = ld_;
        rows = min(total - row0, PAIR ? R / 2 : R);
        const int64_t at = MC ? (int64_t)row0 * (int)sizeof(T) : row0 * ld;
        const bool second = PAIR && ((wave >> 1) & 1);
        base = static_cast<const char *>(second ? p[1] : p[0]) + at;
        next = PAIR ? base : static_cast<const char *>(p[1]) + at;
        if (MC) {
#pragma unroll
            for (int q = 0; q < (HOP ? 1 : Q); ++q) {
                const int byte = (wave + q * NW) * 1024 + lane * 16, k = byte / RB;
                int x = byte % RB;
                x ^= PAD ? (k & 1) << 6 : sizeof(T) == 2 ? ((k & 3) + 4 * ((k >> 3) & 1)) << 5 : ((k >> 2) & 3) << 6;
                off[q] = (uint32_t)(k * ld) + (uint32_t)x;
            }
            static_assert(!MC || !HOP || NW * 1024 / RB % 16 == 0, "the exclusive-or repeats after sixteen k");
            hop = (uint32_t)(NW * 1024 / RB * ld);
            kbyte = 0;
        } else {
            const int r = 8 * (wave & 1) + (lane >> 3);   // within a block of 16 rows
            kbyte = (uint32_t)(((lane & 7) ^ ((r >> 1) & 7)) * 16);
            const int block = wave >> 1;   // of sixteen rows; the lane's next chunk is NW / 2 blocks further on
            off[0] = (uint32_t)((r + 16 * (PAIR ? block >> 1 : block)) * ld) + kbyte;
            hop = (uint32_t)(16 * (PAIR ? NW / 4 : NW / 2) * ld);
        }
    }

    // Stage `step` of a segment (K elements long) from memory straight into LDS (zeros if it is not `valid`).  What lies outside
    // the matrix becomes zero or (columns of MC beyond the tile) a number that no result depends on.  Pieces of 16 bytes lie inside
    // or outside whole.  aim() holds the arithmetic, so that it is out of the way when the loads are due.
    struct Aim {
        const char *from;
        int bytes;
        uint32_t first;   // offset of the lane's first chunk, past every resource if it is not to be read
    };
    __device__ __forceinline__ Aim aim(bool valid, bool second, int step, int K) const
    {
        const int k0 = step * BK, kleft = K - k0;
        const char *b = (second ? next : base) + (MC ? (int64_t)k0 * ld : (int64_t)k0 * (int)sizeof(T));
        const int64_t bytes = MC ? (int64_t)(min(kleft, BK) - 1) * ld + rows * (int)sizeof(T) : (int64_t)(rows - 1) * ld + kleft * (int)sizeof(T);
        const bool in = valid && (MC || (int)kbyte < kleft * (int)sizeof(T));
        return {b, valid ? (int)bytes : 0, in ? off[0] : 0x80000000u};
    }
    __device__ __forceinline__ void fetch(lds_char *lds, const Aim &at, int wave) const
    {
        const __amdgpu_buffer_rsrc_t res = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at.from), 0, at.bytes, 0x00020000);
#pragma unroll
        for (int q = 0; q < Q; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(res, (__attribute__((address_space(3))) void *)(lds + (wave + q * NW) * PIECE), 16,
                                                     (int)(HOP ? at.first + q * hop : offset(q)), 0, 0, 0);
    }

    // Fragments: sixteen rows from 16 block on, half kk (64 bytes of k) of the stage.  `at` from start(), block a constant
    // below the number of blocks that the wave's rows start at a multiple of.
    struct At { uint32_t x, y; };   // y: PAD, blocks whose bit 1 is set
    static __device__ __forceinline__ At start(int row0, int lane)
    {
        const int i = lane & 15, h = lane >> 4;
        if (!MC) return {(uint32_t)((row0 + i) * 128 + ((h ^ ((i >> 1) & 7)) * 16)), 0};
        if (PAD) {
            const uint32_t odd = (i >> 2) & 1, x = (4 * h + (i >> 3)) * PIECE + odd * RB + row0 * 2 + (i & 3) * 8;
            return {x + odd * 64, x - odd * 64};
        }
        if (sizeof(T) == 2) return {(uint32_t)((8 * h + (i >> 2)) * RB + (((row0 >> 4) ^ ((i >> 2) + 4 * (h & 1))) << 5) + (i & 3) * 8), 0};
        return {(uint32_t)(4 * h * RB + (((row0 >> 4) ^ h) << 6) + i * 4), 0};
    }
    static __device__ __forceinline__ v4u read(const lds_char *lds, const At &at, int block, int kk)
    {
        if (!MC) {   // chunk 4 kk + h
            const lds_char *p = lds + ((at.x ^ (uint32_t)(kk * 64)) + block * 2048);
            return *(const __attribute__((address_space(3))) v4u *)p;
        }
        if (sizeof(T) == 2) {
            // ds_read_b64_tr_b16: of each sixteen lanes, lanes 4 r .. 4 r + 3 read row r of a 4 x 16 block, lane i gets column i
            const lds_char *p = PAD ? lds + (block & 2 ? at.y : at.x) + block * 32 + kk * 16 * PIECE : lds + ((at.x ^ (uint32_t)(block << 5)) + kk * 32 * RB);
            typedef __attribute__((address_space(3))) v4s *P;
            const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds_char *)p);
            const v4s y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds_char *)(p + (PAD ? 2 * PIECE : 4 * RB)));
            return __builtin_bit_cast(v4u, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        const lds_char *p = lds + ((at.x ^ (uint32_t)(block << 6)) + kk * 16 * RB);
        v4u v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = *(const __attribute__((address_space(3))) uint32_t *)(p + j * RB);
        return v;
    }
};

// Workgroup b of n runs on XCD b mod 8: each XCD gets a run of consecutive tiles, and they go down bands of four tile rows, so
// that the workgroups of an XCD share operands in its L2.
__device__ __forceinline__ void tile_of(int b, int tiles_m, int tiles_n, int &tm, int &tn)
{
    const int n = tiles_m * tiles_n, each = n / 8, more = n % 8, x = b % 8;
    const int t = x * each + min(x, more) + b / 8;
    const int band = t / (4 * tiles_n), first = band * 4, high = min(4, tiles_m - first), in = t - band * 4 * tiles_n;
    tm = first + in % high;
    tn = in / high;
}

// All but the wave's last LATER loads into LDS are there, and every wave is done with what it read and has come here.
template <int LATER>
__device__ __forceinline__ void arrived()
{
    static_assert(LATER < 64, "the counter has six bits");
    __asm__ volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LATER) : "memory");
    __builtin_amdgcn_s_barrier();
    __asm__ volatile("" ::: "memory");
}

// What a wave's lanes have written to LDS is what its other lanes read next, and what they have read may be written over: a wave's LDS
// instructions run in order, so all that this takes is that the compiler, which sees one lane, leaves them in it.
__device__ __forceinline__ void exchanged()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// The order of a half stage's instructions.  First half: its TM rows of TN blocks (EACH matrix instructions a block) and the
// reads of the second half's fragments, READS_B and READS_A instructions each, those of a row of A after the row whose
// registers they can take.
template <int READS_B, int READS_A, int TN, int TM, int EACH>
__device__ __forceinline__ void order_first()
{
    constexpr int LDS = 0x100, MATRIX = 0x008;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        __builtin_amdgcn_sched_group_barrier(LDS, READS_B, 0);
        __builtin_amdgcn_sched_group_barrier(MATRIX, EACH, 0);
    }
#pragma unroll
    for (int i = 1; i < TM; ++i) {
        __builtin_amdgcn_sched_group_barrier(LDS, READS_A, 0);
        __builtin_amdgcn_sched_group_barrier(MATRIX, EACH * TN, 0);
    }
    __builtin_amdgcn_sched_group_barrier(LDS, READS_A, 0);
    __builtin_amdgcn_sched_barrier(0);
}
// Second half, from row FROM on: the reads of the next stage's first fragments likewise, and the LOADS from memory evenly, one for
// every three blocks of a large tile.  (In a burst they hold up the waves that issue them: two for every two blocks made 8192 x
// 8192 x 8192 take 845 us instead of 800.  Without any loads the loop's matrix instructions are busy 95 % of its time, with them
// 73 %.)
template <int READS_B, int READS_A, int LOADS, int TN, int TM, int EACH, int FROM>
__device__ __forceinline__ void order_second()
{
    constexpr int LDS = 0x100, MEMORY = 0x010, MATRIX = 0x008;
    // those of all of B and of the rows that are past, then those of two rows of A after each row
    constexpr int N = (TM - FROM) * TN, READS = READS_B * TN + READS_A * FROM, SOME = (READS + N / 2 - 1) / (N / 2);
    constexpr int THIRDS = (N + 2) / 3, TOGETHER = (LOADS + THIRDS - 1) / THIRDS;
#pragma unroll
    for (int g = 0; g < N; ++g) {
        if (g < N / 2 && g * SOME < READS) __builtin_amdgcn_sched_group_barrier(LDS, SOME, 0);
        if (g >= N / 2 && g % TN == 0) __builtin_amdgcn_sched_group_barrier(LDS, 2 * READS_A, 0);
        if (g % 3 == 0) __builtin_amdgcn_sched_group_barrier(MEMORY, TOGETHER, 0);
        __builtin_amdgcn_sched_group_barrier(MATRIX, EACH, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
}

// WM x WN waves, each TM x TN blocks of 16 x 16; NB stages in LDS
template <int WM_, int WN_, int TM_, int TN_, int NB_>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, NB = NB_, NW = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16;
};
typedef Shape<2, 4, 8, 4, 2> Large;    // 256 x 256, 8 waves
typedef Shape<2, 4, 4, 4, 3> Medium;   // 128 x 256, 8 waves; the third stage makes up for the shorter time of one
typedef Shape<2, 2, 4, 4, 2> Small;    // 128 x 128, 4 waves, two workgroups a compute unit
typedef Shape<2, 2, 2, 4, 2> Tiny;     // 64 x 128, 4 waves, three

template <class T, int P, int EPI, class S, bool SUMS>
__global__ __launch_bounds__(S::NW * 64, 2) void product_kernel(const ProductArgs a)
{
    constexpr bool PAIR = EPI == E_GATED;
    typedef Operand<T, S::BM, S::NW, P == P_GRAD, false> OpA;
    typedef Operand<T, S::BN, S::NW, P != P_FWD, PAIR> OpB;
    constexpr int COLS = PAIR ? S::BN / 2 : S::BN;
    constexpr int A_BYTES = OpA::STAGE;
    constexpr int LOADS = OpA::Q + OpB::Q;   // of a wave and stage
    __shared__ __attribute__((aligned(1024))) char stage0[A_BYTES + OpB::STAGE];
    __shared__ __attribute__((aligned(1024))) char stage1[A_BYTES + OpB::STAGE];
    __shared__ __attribute__((aligned(1024))) char stage2[S::NB == 3 ? A_BYTES + OpB::STAGE : 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tm, tn;
    tile_of(blockIdx.x, a.tiles_m, a.tiles_n, tm, tn);
    const int m0 = tm * S::BM, n0 = tn * COLS;
    const int wm = wave / S::WN, wn = wave % S::WN;

    OpA oa;
    OpB ob;
    oa.init(a.a, a.lda, m0, OpA::MC_ ? a.a_ext : a.M, wave, lane);
    ob.init(a.b, a.ldb, n0, OpB::MC_ ? a.b_ext : a.N, wave, lane);
    const int per_seg = (a.K + OpA::BK - 1) / OpA::BK, all = per_seg * a.segments;
    const int t0 = blockIdx.y * a.steps, t1 = min(all, t0 + a.steps);

    v4f acc[S::TM][S::TN] = {};
    float sum[SUMS ? S::TM : 1] = {};   // the lane's part of A's sums over k
    const bool sums = SUMS && tn == 0 && wn == 0;
    const typename OpA::At ra = OpA::start(wm * S::TM * 16, lane);
    const typename OpB::At rb = OpB::start(wn * S::TN * 16, lane);

    struct Half { v4u a[S::TM], b[S::TN]; };   // a wave's fragments of half a stage
    auto read = [&](Half &f, const char *stage, int kk) {
        const lds_char *l = (const lds_char *)stage;
        typename OpA::At pa = ra;
        typename OpB::At pb = rb;
        if (OpB::MC_ && !OpB::PAD) __asm__("" : "+v"(pa.x), "+v"(pb.x));   // the blocks' addresses are formed anew: the registers are the fragments'
#pragma unroll
        for (int j = 0; j < S::TN; ++j) f.b[j] = OpB::read(l + A_BYTES, pb, j, kk);
#pragma unroll
        for (int i = 0; i < S::TM; ++i) f.a[i] = OpA::read(l, pa, i, kk);
    };
    auto multiply = [&](const Half &f, int from, int to) {
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
            if (i >= from && i < to) {
                mfma_row<T, false>(f.b, f.a[i], acc[i]);
                if (SUMS) sum[i] = add_all(f.a[i], sum[i], T());
            }
    };

    // NB stages in LDS, and in registers the fragments of the half stage at work.  Each row of blocks (TN matrix
    // instructions) is followed by the read of its next fragment, which can go where the last one was; the other operand's
    // fragments, which every row needs, come beforehand and into registers of their own.  The loads from memory have the time of
    // NB - 1 stages.
    Half f0, f1;
    typename OpA::Aim aim_a;
    typename OpB::Aim aim_b;
    auto prepare = [&](int t) {
        const bool second = t >= per_seg;
        aim_a = oa.aim(t < t1, second, second ? t - per_seg : t, OpA::MC_ ? a.K : a.a_ext);
        aim_b = ob.aim(t < t1, second, second ? t - per_seg : t, OpB::MC_ ? a.K : a.b_ext);
    };
    auto fetch = [&](char *stage) {
        oa.fetch((lds_char *)stage, aim_a, wave);
        ob.fetch((lds_char *)stage + A_BYTES, aim_b, wave);
    };
    constexpr int EACH = sizeof(T) == 4 ? 4 : 1, AHEAD = S::TM == 8 ? 2 : 0;   // matrix instructions of a block; rows before the barrier
    auto stage = [&](char *cur, char *next, int t) {
        prepare(t + S::NB);
        read(f1, cur, 1);
        multiply(f0, 0, S::TM);
        order_first<OpB::READS, OpA::READS, S::TN, S::TM, EACH>();
        multiply(f1, 0, AHEAD);
        __builtin_amdgcn_sched_barrier(0);
        arrived<(S::NB - 2) * LOADS>();   // `next` has come, and every wave has read all of `cur`
        __builtin_amdgcn_sched_barrier(0);
        fetch(cur);
        read(f0, next, 0);
        multiply(f1, AHEAD, S::TM);
        order_second<OpB::READS, OpA::READS, LOADS, S::TN, S::TM, EACH, AHEAD>();
    };
    prepare(t0);
    fetch(stage0);
    prepare(t0 + 1);
    fetch(stage1);
    if (S::NB == 3) {
        prepare(t0 + 2);
        fetch(stage2);
    }
    arrived<(S::NB - 1) * LOADS>();
    read(f0, stage0, 0);
    int t = t0;
    if constexpr (S::NB == 3) {
        for (; t + 2 < t1; t += 3) {
            stage(stage0, stage1, t);
            stage(stage1, stage2, t + 1);
            stage(stage2, stage0, t + 2);
        }
        if (t < t1) stage(stage0, stage1, t);
        if (t + 1 < t1) stage(stage1, stage2, t + 1);
    } else {
        // Large tiles: a stage past the last one is zeros.  (A loop's tail of its own costs registers that they do not have.)
        for (; t + (S::TM == 8 ? 0 : 1) < t1; t += 2) {
            stage(stage0, stage1, t);
            stage(stage1, stage0, t + 1);
        }
        if (S::TM != 8 && t < t1) stage(stage0, stage1, t);
    }
    arrived<0>();

    // Epilogue.  A wave turns its sums through its own 16 KB of LDS, sixty-four rows (or all it has) at a time, so that a lane gets eight
    // neighbouring columns of a row: rows of 256 bytes, their 16-byte units u at u ^ (row mod 16).  No bank conflicts but a pair's: sixteen of its
    // lanes read eight units twice (2.1e6 cycles over the chip at 8192 x 8192, of 8.4e8 that its waves live).
    const int i16 = lane & 15, h = lane >> 4;
    const int64_t plane = (int64_t)a.M * a.N;
    const int row0 = m0 + wm * S::TM * 16;
    if (SUMS && sums)
#pragma unroll
        for (int i = 0; i < S::TM; ++i) {
            const int m = row0 + i * 16 + i16;
            float v = sum[i] + __shfl_xor(sum[i], 16);
            v += __shfl_xor(v, 32);
            if (h == 0 && m < a.M) {
                if (a.split > 1) a.ws[a.split * plane + (int64_t)blockIdx.y * a.M + m] = v;
                else finish_sum<T>(a.f, m, v);
            }
        }
    float *part = a.ws + blockIdx.y * plane * (PAIR ? 2 : 1);
    constexpr int EACH_STAGE = (S::NW + S::NB - 1) / S::NB;   // waves
    constexpr int BLOCKS = S::TM < 4 ? S::TM : 4, ROWS = BLOCKS * 16;   // at a time
    static_assert(EACH_STAGE * ROWS * 256 <= A_BYTES + OpB::STAGE, "a wave's own part of a stage");
    char *own = (wave < EACH_STAGE ? stage0 : wave < 2 * EACH_STAGE ? stage1 : stage2) + wave % EACH_STAGE * ROWS * 256;
    constexpr int LANES = PAIR ? 4 : 8;   // of a row
    const int c = lane % LANES, n = n0 + wn * (PAIR ? 32 : 64) + c * 8;
    static_assert(S::TN == 4, "a wave's 64 columns");
    auto unit = [&](int row, int u) { return reinterpret_cast<v4f *>(own + row * 256 + ((u ^ (row & 15)) << 4)); };
    auto sums_of = [&](int r, float (&v)[8], float (&w)[8]) {
        const v4f x = *unit(r, 2 * c), y = *unit(r, 2 * c + 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = x[j];
            v[4 + j] = y[j];
        }
        if (PAIR) {
            const v4f p = *unit(r, 8 + 2 * c), q = *unit(r, 9 + 2 * c);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] = p[j];
                w[4 + j] = q[j];
            }
        }
    };
    auto turn = [&](int i0) {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)   // a pair's blocks alternate: those of the first matrix first
                *unit(i * 16 + i16, (PAIR ? (j >> 1) + (j & 1) * 2 : j) * 4 + h) = acc[i0 + i][j];
    };
    constexpr int STEP = 64 / LANES;   // rows apart
    // Sixty-four rows at a time; what lies beside the result is read once for the columns, and a round ahead for the rows.  ALL: the tile
    // lies inside the result.
    auto finish = [&](auto all) {
        constexpr bool ALL = decltype(all)::value;
        constexpr int TOGETHER = ALL && EPI != E_GATED ? 4 : 2;   // rows whose reads go together
        const int last = ALL ? row0 + S::TM * 16 - 1 : a.M - 1, left = ALL ? 8 : a.N - n;
        Beside<T, EPI> next[TOGETHER];
        next[0].template columns<ALL>(a.f, n, left);
#pragma unroll
        for (int q = 0; q < TOGETHER; ++q) {
            next[q].b = next[0].b;
            next[q].b2 = next[0].b2;
            next[q].template get<ALL>(a.f, min(row0 + lane / LANES + q * STEP, last), n, left);
        }
#pragma unroll
        for (int i0 = 0; i0 < S::TM; i0 += BLOCKS) {
            turn(i0);
            exchanged();
            const int first = row0 + i0 * 16;
#pragma unroll 1
            for (int r = lane / LANES; r < ROWS; r += STEP * TOGETHER) {
                Beside<T, EPI> side[TOGETHER];
#pragma unroll
                for (int q = 0; q < TOGETHER; ++q) {
                    side[q] = next[q];
                    next[q].template get<ALL>(a.f, min(first + r + (TOGETHER + q) * STEP, last), n, left);
                }
#pragma unroll
                for (int q = 0; q < TOGETHER; ++q) {
                    const int m = first + r + q * STEP;
                    float v[8], w[8];
                    sums_of(r + q * STEP, v, w);
                    if (ALL || (m < a.M && n < a.N)) finish8<T, EPI, ALL>(a.f, side[q], m, n, left, v, w);
                }
            }
            exchanged();
        }
    };
    if (a.split > 1) {
#pragma unroll
        for (int i0 = 0; i0 < S::TM; i0 += BLOCKS) {
            turn(i0);
            exchanged();
#pragma unroll 1
            for (int r = lane / LANES; r < ROWS; r += STEP) {
                const int m = row0 + i0 * 16 + r;
                if (m >= a.M || n >= a.N) break;
                float v[8], w[8];
                sums_of(r, v, w);
                store8<float>(part, (int64_t)m * a.N + n, v, a.N - n);
                if (PAIR) store8<float>(part, plane + (int64_t)m * a.N + n, w, a.N - n);
            }
            exchanged();
        }
    } else if (m0 + S::BM <= a.M && n0 + COLS <= a.N) {
        finish(std::true_type());
    } else {
        finish(std::false_type());
    }
}

// A's sums over k for a product in large tiles, whose registers have no room for them: a workgroup takes 256 columns of the
// rows of one part, eight columns a thread, and leaves the part's sums in the workspace.  Bound by launches at ordinary sizes: 1024 x 8192,
// bf16, 6.4 us, and 4.7 to join the parts.
template <class T>
__global__ __launch_bounds__(256) void sum_parts_kernel(const ProductArgs a)
{
    __shared__ float share[8][256];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5, m = blockIdx.x * 256 + c * 8;
    const int each = (a.K + kSumParts - 1) / kSumParts, from = blockIdx.y * each, to = min(a.K, from + each);
    float v[8] = {};
    if (m < a.M)
        for (int k = from + r; k < to; k += 8) {
            float x[8];
            load8<T>(x, static_cast<const char *>(a.a[0]) + k * a.lda, m, a.M - m);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += x[j];
        }
#pragma unroll
    for (int j = 0; j < 8; ++j) share[r][c * 8 + j] = v[j];
    __syncthreads();
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= a.M) return;
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) s += share[q][threadIdx.x];
    a.ws[(int64_t)blockIdx.y * a.M + n] = s;
}
template <class T>
__global__ __launch_bounds__(256) void sum_join_kernel(const ProductArgs a)
{
    const int m = blockIdx.x * 256 + threadIdx.x;
    if (m >= a.M) return;
    float v = 0.f;
    for (int p = 0; p < kSumParts; ++p) v += a.ws[(int64_t)p * a.M + m];
    finish_sum<T>(a.f, m, v);
}

// The parts of a product whose k was split, added in order (so that results repeat), and its epilogue.  A thread takes eight columns of one
// row, four parts loaded at a time.  Bound by reading the parts: 32 rows by 4096, eight parts, 4.2 us (a part at a time: 6.2).
template <class T, int EPI>
__global__ __launch_bounds__(256) void join_kernel(const ProductArgs a, int sums)
{
    constexpr int PLANES = EPI == E_GATED ? 2 : 1, AT_ONCE = 4;
    // the workgroup's first eight columns by one uniform division, the thread's by a short one
    const uint32_t eights = ((uint32_t)a.N + 7) / 8;
    const int64_t first = (int64_t)blockIdx.x * 256, plane = (int64_t)a.M * a.N;
    const uint32_t row0 = (uint32_t)((uint64_t)first / eights), c0 = (uint32_t)((uint64_t)first % eights) + threadIdx.x, more = c0 / eights;
    const int64_t row = (int64_t)row0 + more;
    if (row < a.M) {
        const int m = (int)row, n = (int)(c0 - more * eights) * 8;
        Beside<T, EPI> side;
        side.template columns<false>(a.f, n, a.N - n);
        side.template get<false>(a.f, m, n, a.N - n);
        float v[8] = {}, w[8] = {};
        const float *p = a.ws + row * a.N + n;
        for (int s = 0; s < a.split; s += AT_ONCE) {
            float x[AT_ONCE][PLANES][8] = {};
#pragma unroll
            for (int q = 0; q < AT_ONCE; ++q)
                if (s + q < a.split) {
#pragma unroll
                    for (int c = 0; c < PLANES; ++c) load8<float>(x[q][c], p, ((int64_t)(s + q) * PLANES + c) * plane, a.N - n);
                }
#pragma unroll
            for (int q = 0; q < AT_ONCE; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] += x[q][0][j];
                    w[j] += x[q][PLANES - 1][j];
                }
        }
        finish8<T, EPI, false>(a.f, side, m, n, a.N - n, v, w);
    }
    const int64_t at = first + threadIdx.x;
    if (EPI == E_STORE && sums && at < a.M) {
        float v = 0.f;
        for (int s = 0; s < a.split; ++s) v += a.ws[a.split * plane + (int64_t)s * a.M + at];
        finish_sum<T>(a.f, (int)at, v);
    }
}

}  // namespace dn
