// Operators of the residual feed-forward block: what their kernels share.  Internal; the entry points are in include/dn.h.
#pragma once

#include "dn_internal.h"

namespace dn {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef _Float16 f16;
typedef __bf16 bf16;

// eight elements as they lie in memory, at any alignment of theirs
template <class T> struct Eight { typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T)))); };

// elements from p[at] on; those from `left` on are zero, and not stored.  ALL: left is 8 or more.
template <class T, bool ALL = false>
__device__ __forceinline__ typename Eight<T>::type get8(const void *p, int64_t at, int left)
{
    const T *q = static_cast<const T *>(p) + at;
    if (ALL || left >= 8) return *reinterpret_cast<const typename Eight<T>::type *>(q);
    typename Eight<T>::type x;
    if (left <= 0) return typename Eight<T>::type{};   // without this a wave whose lanes have all or nothing would take what follows too
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? q[j] : (T)0.f;
    return x;
}
template <class T, bool ALL = false>
__device__ __forceinline__ void load8(float (&v)[8], const void *p, int64_t at, int left)
{
    const auto x = get8<T, ALL>(p, at, left);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)x[j];
}
// STREAM: past the caches' own order, for results that nothing near reads again
template <class T, bool ALL = false, bool STREAM = false>
__device__ __forceinline__ void store8(void *p, int64_t at, const float (&v)[8], int left)
{
    T *q = static_cast<T *>(p) + at;
    if (ALL || left >= 8) {
        typename Eight<T>::type x;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (T)v[j];
        if (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<typename Eight<T>::type *>(q));
        else *reinterpret_cast<typename Eight<T>::type *>(q) = x;
    } else if (left > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) q[j] = (T)v[j];
    }
}

// fp32 numbers in 24 bits, the upper 16 and the next 8 apart: rounded to 16 significant bits, which is 2^-17 of a number.  For what is
// added up and then rounded to 16 bits: a third less to write and read.
__device__ __forceinline__ uint32_t upper24(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    return v == v ? u + 0x80 : (u & 0xffffff00u) | 0x400000u;   // (a carry of NaN's would make a number of it)
}
template <bool ALL>
__device__ __forceinline__ void store24(void *high, void *low, int64_t at, const float (&v)[8], int left)
{
    typedef uint16_t v8s __attribute__((ext_vector_type(8), aligned(16)));
    typedef uint8_t v8b __attribute__((ext_vector_type(8), aligned(8)));
    v8s h;
    v8b l;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t u = ALL || j < left ? upper24(v[j]) : 0;
        h[j] = (uint16_t)(u >> 16);
        l[j] = (uint8_t)(u >> 8);
    }
    // rows are padded to multiples of eight
    __builtin_nontemporal_store(h, reinterpret_cast<v8s *>(static_cast<uint16_t *>(high) + at));
    __builtin_nontemporal_store(l, reinterpret_cast<v8b *>(static_cast<uint8_t *>(low) + at));
}
__device__ __forceinline__ void load24(float (&v)[8], const void *high, const void *low, int64_t at)
{
    typedef uint16_t v8s __attribute__((ext_vector_type(8), aligned(16)));
    typedef uint8_t v8b __attribute__((ext_vector_type(8), aligned(8)));
    const v8s h = *reinterpret_cast<const v8s *>(static_cast<const uint16_t *>(high) + at);
    const v8b l = *reinterpret_cast<const v8b *>(static_cast<const uint8_t *>(low) + at);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(float, (uint32_t)h[j] << 16 | (uint32_t)l[j] << 8);
}

// ---- dropout --------------------------------------------------------------------------------------------------
// Philox 4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two
// 32 x 32 -> 64 bit products over a 128-bit counter.  One call gives the eight 16-bit numbers of eight neighbouring columns
// of a row, which is what a thread of every kernel here has in hand: twenty products for eight numbers.  (With 32-bit
// numbers it would be forty, and the numbers a third of a wide layer's epilogue.)
struct Dropout {
    uint32_t t = 0;          // numbers below t are dropped; 0: none are
    float scale = 1.f;       // 65536 / (65536 - t)
    uint32_t k0 = 0, k1 = 0; // seed
    uint32_t o0 = 0, o1 = 0; // offset
};

__device__ __forceinline__ v4u philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)q;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return v4u{c0, c1, c2, c3};
}

// v[j] of row m, columns n .. n + 7 (n a multiple of 8) as dropout leaves them
__device__ __forceinline__ void drop8(const Dropout &d, int m, int n, float (&v)[8])
{
    const v4u w = philox((uint32_t)n >> 3, (uint32_t)m, d.o0, d.o1, d.k0, d.k1);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t u = j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xffff;
        v[j] = u >= d.t ? v[j] * d.scale : 0.f;
    }
}

// ---- activations ------------------------------------------------------------------------------------------------
// fp32 results come from the library's functions.  Results that are rounded to 16 bits come from the hardware's exp2 and
// reciprocal (1 ulp each), and their error function from Abramowitz and Stegun 7.1.26 (|error| <= 1.5e-7): a few
// instructions instead of some sixty, which would be a quarter of a wide layer's time.  A 16-bit GELU is so within 2.2e-7 everywhere before
// it is rounded; of its own size it is off by up to 0.05 % above -4, 0.4 % above -6 and 1.5 % above -9, where it is 10^-4, 10^-8 and 10^-18.
template <bool FAST> struct Math;
template <> struct Math<false> {
    static __device__ __forceinline__ float exp(float x) { return expf(x); }
    static __device__ __forceinline__ float inv(float x) { return 1.f / x; }
    static __device__ __forceinline__ void tanh(float x, float &f, float &df)
    {
        const float e = exp(-2.f * fabsf(x)), q = inv(1.f + e);
        f = tanhf(x);
        df = 4.f * e * q * q;
    }
    // the normal distribution's function and density
    static __device__ __forceinline__ void normal(float x, float &cdf, float &pdf)
    {
        // 1 + erf would lose the tail, 5 % of it at -5.  1 to 2 % of a layer's time; of a short product's, 8192 x 256 by 4096, 166 -> 177 us
        cdf = 0.5f * erfcf(x * -0.70710678f);
        pdf = 0.39894228f * expf(-0.5f * x * x);
    }
};
template <> struct Math<true> {
    static __device__ __forceinline__ float exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
    static __device__ __forceinline__ float inv(float x) { return __builtin_amdgcn_rcpf(x); }
    static __device__ __forceinline__ void tanh(float x, float &f, float &df)
    {
        // 1 - 2 / (e^2x + 1) loses the leading bits of small results: their series instead
        const float e = exp(2.f * x), q = inv(e + 1.f), big = 1.f - 2.f * q, s = x * x;
        f = s < 0.01f ? x * (1.f + s * (-0.33333333f + s * 0.13333333f)) : big;
        df = 4.f * q * (x < 0.f ? e * q : 1.f - q);
    }
    static __device__ __forceinline__ void normal(float x, float &cdf, float &pdf)
    {
        const float y = fabsf(x) * 0.70710678f, t = inv(1.f + 0.3275911f * y), e = exp(-y * y);
        const float poly = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
        const float half = 0.5f * poly * e;   // (1 - erf y) / 2
        cdf = x < 0.f ? half : 1.f - half;
        pdf = 0.39894228f * e;
    }
};

// f(z), and f'(z) with it.  1 - f of a unit that is all but 1 would be rounding: a sigmoid's comes of exp(-z), which is small there, and so
// do both ends of a tanh's derivative, 4 q (1 - q) with q = 1 / (1 + exp(2 z)).
template <int ACT, bool FAST>
__device__ __forceinline__ void act_one(float z, float &f, float &df)
{
    typedef Math<FAST> K;
    if (ACT == DN_ACT_SIGMOID) {
        const float e = K::exp(-z);
        f = K::inv(1.f + e);
        df = f * (z > 0.f ? e * f : 1.f - f);
    } else if (ACT == DN_ACT_TANH) {
        K::tanh(z, f, df);
    } else if (ACT == DN_ACT_RELU) {   // a comparison that a NaN fails would hide it
        f = z < 0.f ? 0.f : z;
        df = z > 0.f ? 1.f : 0.f;
    } else if (ACT == DN_ACT_SILU) {
        const float s = K::inv(1.f + K::exp(-z));
        const bool far = fabsf(z) > 1e4f;   // where s is 0 or 1: inf * 0
        f = far && z < 0.f ? 0.f : z * s;
        df = far ? s : s * (1.f + z * (1.f - s));
    } else if (ACT == DN_ACT_GELU) {
        float c, p;
        K::normal(z, c, p);
        f = z < -30.f ? 0.f : z * c;
        df = fabsf(z) > 30.f ? c : c + z * p;   // inf * 0
    } else {
        f = z;
        df = 1.f;
    }
}
// of eight, the choice made once for all
template <int ACT, bool FAST>
__device__ __forceinline__ void act_each(const float (&z)[8], float (&f)[8], float (&df)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) act_one<ACT, FAST>(z[j], f[j], df[j]);
}
template <bool FAST>
__device__ __forceinline__ void act8(int act, const float (&z)[8], float (&f)[8], float (&df)[8])
{
    switch (act) {
    case DN_ACT_SIGMOID: act_each<DN_ACT_SIGMOID, FAST>(z, f, df); break;
    case DN_ACT_TANH: act_each<DN_ACT_TANH, FAST>(z, f, df); break;
    case DN_ACT_RELU: act_each<DN_ACT_RELU, FAST>(z, f, df); break;
    case DN_ACT_SILU: act_each<DN_ACT_SILU, FAST>(z, f, df); break;
    case DN_ACT_GELU: act_each<DN_ACT_GELU, FAST>(z, f, df); break;
    default: act_each<DN_ACT_LINEAR, FAST>(z, f, df);
    }
}

// ---- matrix products ---------------------------------------------------------------------------------------------
// C[m][n] = sum_k A(m, k) B(n, k).  An operand is stored with k contiguous ("KC": [m][k] or [n][k]) or with its own index
// contiguous ("MC": [k][m] or [k][n]).
enum Product : int {
    P_FWD = 0,    // A = X [rows][n_in] KC, B = W [n_out][n_in] KC
    P_DELTA = 1,  // A = delta [rows][n_out] KC, B = W [n_out][n_in] MC
    P_GRAD = 2    // A = delta [rows][n_out] MC, B = X [rows][n_in] MC
};
enum Epilogue : int {
    E_LINEAR = 0,  // P_FWD: + bias, activation, dropout, residual; the net input too
    E_GATED = 1,   // P_FWD of two matrices B: f(g) u; g and u too
    E_DGATED = 2,  // P_DELTA: d(f(g) u) from its derivative: dG, dU, and f(g) u again
    E_STORE = 3,   // alpha times the sum, as T or as fp32
    E_DEXPERT = 4, // as E_DGATED, each row times its weight; and the weight's derivative
    E_PAIR = 5     // the sum, in 24 bits
};

struct Finish {
    void *y = nullptr;          // result [M][ldy]; E_DGATED: dG [M][ldy] with dU `half_y` columns further on
    int64_t ldy = 0;
    void *y2 = nullptr;         // E_LINEAR: net inputs; E_GATED: G and U; E_DGATED: f(g) u; E_STORE: rows from m_split on; E_PAIR: low bytes
    int64_t ldy2 = 0;
    const void *r = nullptr;    // E_LINEAR: residual; E_DGATED: G and U
    int64_t ldr = 0;
    const void *bias = nullptr, *bias2 = nullptr;
    void *sums = nullptr, *sums2 = nullptr;   // P_GRAD: alpha times A's sums over k, [M] (from m_split on: sums2)
    int32_t zeros = 0;          // E_GATED, E_DGATED: columns of zeros that follow the results' rows, to a multiple of eight
    int64_t half = 0, half_y = 0;   // columns between G and U; between dG and dU
    int32_t m_split = 0x7fffffff;
    int32_t m_valid = 0x7fffffff;   // rows of either side of m_split that exist
    int32_t act = 0;
    int32_t f32_out = 0;        // E_STORE: results are fp32 whatever T is
    float alpha = 1.f;
    const float *weight = nullptr;      // E_DEXPERT: of row m, weight[order[m]] of `pairs`
    const int32_t *order = nullptr;
    uint32_t pairs = 1;
    float *dots = nullptr;              // E_DEXPERT: parts of the weights' derivatives, [64 columns each][rows], rows dots_ld apart
    int64_t dots_ld = 0;
    Dropout drop;
};

// Rows that are pairs of a row and one of several experts, by expert
struct Group {
    const int32_t *starts = nullptr, *order = nullptr;   // an expert's first pair, [experts + 1]; the pair at a place
    int32_t experts = 0, k = 1, pairs = 0, rows = 0;     // k: pairs of a row
    int64_t b_stride = 0, c_stride = 0;                  // bytes between two experts' matrices; between their results (P_GRAD), those of parts of k
};

__device__ __forceinline__ int bounded(const Group &g, int e) { return min(max(g.starts[e], 0), g.pairs); }
// the row of X that the pair at place m is of; whatever the lists hold, a row that exists
__device__ __forceinline__ int token_of(const Group &g, int m)
{
    return (int)min((uint32_t)max(g.order[m], 0) / (uint32_t)g.k, (uint32_t)g.rows - 1);
}

struct ProductArgs {
    const void *a[2], *b[2];    // operands; the second ones: of the second segment of k, or (E_GATED) of the second matrix
    int64_t lda, ldb;           // bytes between stored rows
    int32_t a_ext, b_ext;       // elements of a stored row that may be read: the row and zeros up to a multiple of 16 bytes
    int32_t M, N, K;            // K: of one segment
    int32_t segments;           // 1 or 2
    float *ws;                  // split > 1: partial sums [split][planes][M][N], then [split][M] of E_STORE's sums
    int32_t split, steps;       // k steps of each part
    int32_t tiles_m, tiles_n;
    Finish f;
    Group group;
};

constexpr int kFewRows = 64;    // most rows of the kernel that stages nothing
constexpr int kSumParts = 32;   // parts of k that a launch of its own adds A's columns in

// How a product is run.  `ws_bytes`: workspace that it needs.
enum ProductKernel : int { K_FEW, K_TINY, K_SMALL, K_MEDIUM, K_LARGE };   // K_TINY: fp32, K_MEDIUM and K_LARGE: 16 bits
struct ProductPlan {
    ProductKernel kernel = K_SMALL;
    int split = 1, steps = 0;
    size_t ws_bytes = 0;
};
ProductPlan plan_product(int type, Product p, Epilogue e, int M, int N, int K, int segments, bool sums);
hipError_t launch_product_f32(Product p, Epilogue e, const ProductPlan &plan, ProductArgs a, hipStream_t s);
hipError_t launch_product_f16(Product p, Epilogue e, const ProductPlan &plan, ProductArgs a, hipStream_t s);
hipError_t launch_product_bf16(Product p, Epilogue e, const ProductPlan &plan, ProductArgs a, hipStream_t s);

// ---- elementwise ------------------------------------------------------------------------------------------------
// Y = D(X), or (act >= 0) Y = kept(X) f'(Z) without D's scale, which the products that follow multiply their sums by
struct MaskArgs {
    const void *x, *z;
    void *y;
    int64_t ldx, ldz, ldy;
    int32_t rows, cols, act;
    int32_t zeros;   // columns of zeros that follow Y's rows
    Dropout drop;
};

// Matrices whose rows do not lie at multiples of 16 bytes, or end between two, copied to where they do, zeros following.
struct PackArgs {
    struct { const void *x; void *y; int64_t ldx; int32_t rows, cols; int64_t first; } m[5];   // first: its first group of eight
    int32_t n;
    int64_t groups;
};
// either or both; `a` may be NULL, and `p` may hold none
hipError_t launch_mask_pack(int type, const MaskArgs *a, const PackArgs &p, hipStream_t s);

// ---- norms ------------------------------------------------------------------------------------------------------
struct NormArgs {
    // forward: x' = x + scale gate post(b), n = pre(x'); backward: x is x'
    const void *x, *b, *gate, *post_w, *post_b, *pre_w, *pre_b;
    void *x_out, *n_out;
    const void *dx_out, *dn;
    void *dx, *db, *dgate, *dpost_w, *dpost_b, *dpre_w, *dpre_b;
    float *ws;
    int32_t rows, d, group;   // rows that share a gate
    int32_t post, pre;        // dn_norm_kind
    int32_t f32_out;          // parameter gradients are fp32
    float scale, eps;
    // backward: rows of a part, parts of a group (1 where a part is whole groups), and how many parts there are
    int32_t part_rows, group_parts, parts;
};
hipError_t launch_norm_forward(int type, const NormArgs &a, hipStream_t s);
hipError_t launch_norm_backward(int type, const NormArgs &a, hipStream_t s);
constexpr int kNormWidth = 16384;   // largest d
// how the backward pass is divided, and its workspace
size_t norm_backward_plan(int type, NormArgs &a);

}  // namespace dn
