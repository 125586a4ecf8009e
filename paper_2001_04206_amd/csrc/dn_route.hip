// Routing of rows to experts: choices and weights from logits, the lists of rows by expert, and the logits' gradient.
//
// Bound by instructions, about 900 a row of 256 experts with groups and eight choices: 16384 rows in 24 us with a bias and groups (scores in
// 64 bits take 7 of them, groups 4; scores in 32, with rows that come close done again, were no faster), 14 without, 7 for one choice.  The lists
// take 4.8 and 6.6 us more for 131072 pairs.  One row of 128 experts with its lists: one launch, 5.4 us.  Backward, 16384 rows of 128: 8.8 us.
#include <type_traits>

#include "dn_ffn_host.h"
#include "dn_wave.h"

namespace dn {
namespace {

constexpr int kMostExperts = 1024, kMostChoices = 32, kWaves = 4;
constexpr int64_t kMostRows = (int64_t)1 << 25, kMostPairs = (int64_t)1 << 30;

struct RouteArgs {
    const void *l;
    const float *bias;
    int32_t *expert;
    float *weight;
    const int32_t *chosen;    // backward: expert
    const float *dweight;
    void *dl;
    int64_t ldl;
    int32_t rows, experts, k;
    int32_t groups, each, top_groups, best;   // each: experts of a group
    int32_t score, renorm;
    float scale;
};

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ double dpp_move64(double v, double identity)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v), i = __builtin_bit_cast(uint64_t, identity);
    const uint32_t lo = __builtin_amdgcn_update_dpp((int)(uint32_t)i, (int)(uint32_t)b, CTRL, ROW_MASK, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp((int)(uint32_t)(i >> 32), (int)(uint32_t)(b >> 32), CTRL, ROW_MASK, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double last_lane(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ float highest(float v) { return wave_max(v); }
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ int higher(int v)
{
    return max(v, __builtin_amdgcn_update_dpp(v, v, CTRL, ROW_MASK, 0xf, ROW_MASK == 0xf));   // (lanes that are not moved to keep v)
}
__device__ __forceinline__ int highest(int v)
{
    v = higher<0xB1, 0xf>(v);    // as wave_max()
    v = higher<0x4E, 0xf>(v);
    v = higher<0x141, 0xf>(v);
    v = higher<0x140, 0xf>(v);
    v = higher<0x142, 0xa>(v);
    v = higher<0x143, 0xc>(v);
    return __builtin_amdgcn_readlane(v, 63);
}
// fp32 numbers as whole numbers of the same order, -0 as 0; kNone is that of -inf
__device__ __forceinline__ int in_order(float v)
{
    const int u = __builtin_bit_cast(int, v + 0.f);
    return u ^ (int)((uint32_t)(u >> 31) >> 1);
}
constexpr int kNone = (int)0x807fffff;
__device__ __forceinline__ double highest(double v)
{
    const double ninf = -INFINITY;
    v = fmax(v, dpp_move64<0xB1, 0xf>(v, ninf));
    v = fmax(v, dpp_move64<0x4E, 0xf>(v, ninf));
    v = fmax(v, dpp_move64<0x141, 0xf>(v, ninf));
    v = fmax(v, dpp_move64<0x140, 0xf>(v, ninf));
    v = fmax(v, dpp_move64<0x142, 0xa>(v, ninf));
    v = fmax(v, dpp_move64<0x143, 0xc>(v, ninf));
    return last_lane(v);
}
__device__ __forceinline__ double total(double v)
{
    v += dpp_move64<0xB1, 0xf>(v, 0.);
    v += dpp_move64<0x4E, 0xf>(v, 0.);
    v += dpp_move64<0x141, 0xf>(v, 0.);
    v += dpp_move64<0x140, 0xf>(v, 0.);
    v += dpp_move64<0x142, 0xa>(v, 0.);
    v += dpp_move64<0x143, 0xc>(v, 0.);
    return last_lane(v);
}

// a lane's logits, -inf behind the last
template <class T, int V> struct Several { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
template <class T, int V>
__device__ __forceinline__ void load_logits(float (&l)[V], const T *p, int first, int experts)
{
    if (first + V <= experts) {
        const auto x = *reinterpret_cast<const typename Several<T, V>::type *>(p + first);
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = first + i < experts ? (float)p[first + i] : -INFINITY;
    }
}

// 1 / x of an x from 1 to 1e300: the hardware's estimate and two Newton steps
__device__ __forceinline__ double inverse64(double x)
{
    double r = __builtin_amdgcn_rcp(x);
    r = fma(fma(-x, r, 1.), r, r);
    return fma(fma(-x, r, 1.), r, r);
}

// sigmoid(l) e^-low, low <= 0 and not below the largest of the logits that are compared (or 0): ratios of small scores keep their bits
__device__ __forceinline__ float sigmoid_above(float l, float low)
{
    const float e = expf(-fabsf(l)), q = 1.f / (1.f + e);
    return l >= 0.f ? q : l == l ? expf(l - low) * q : l;
}

// The weights of choices, lane j the one of logit l where it is `mine`: m, sum are the row's (softmax without renorm).
__device__ __forceinline__ float weight_of(const RouteArgs &a, float l, bool mine, float m, float sum)
{
    float x;
    if (a.score == DN_SCORE_SOFTMAX) {
        if (a.renorm) m = wave_max(mine ? l : -INFINITY);
        x = expf(l - m);
    } else {
        x = sigmoid_above(l, a.renorm ? fminf(0.f, wave_max(mine ? l : -INFINITY)) : 0.f);
    }
    if (a.renorm) sum = wave_sum(mine ? x : 0.f);
    if (a.renorm || a.score == DN_SCORE_SOFTMAX) x /= sum;
    return x * a.scale;
}

// The two highest of p and q (p >= q) and of another lane's, whose lane the move names
template <int CTRL>
__device__ __forceinline__ void best_two(double &p, double &q)
{
    const double x = dpp_move64<CTRL, 0xf>(p, p), y = dpp_move64<CTRL, 0xf>(q, q);
    q = fmax(fmin(p, x), fmax(q, y));
    p = fmax(p, x);
}
template <int CTRL>
__device__ __forceinline__ void best_two(float &p, float &q)
{
    const float x = dpp_move<CTRL, 0xf>(p, p), y = dpp_move<CTRL, 0xf>(q, q);
    q = fmaxf(fminf(p, x), fmaxf(q, y));
    p = fmaxf(p, x);
}
__device__ __forceinline__ double from_lane(double v, int lane)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ float from_lane(float v, int lane)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// A wave takes a row, a lane V neighbouring experts of it.  The highest of all lanes, k times: of equal ones the lowest lane holds the
// lowest expert.  WIDE: ranks are scores in 64 bits plus the bias; otherwise the logits themselves.  WIDE without a bias: groups are chosen by
// sums of two scores, experts by their logits all the same, as scores run together where logits do not (a sigmoid is 1 from 37 on).
template <class T, int V, bool WIDE>
__device__ __forceinline__ void route_row(const RouteArgs &a, int row, int lane)
{
    typedef typename std::conditional<WIDE, double, float>::type Rank;
    const int first = lane * V;
    const Rank ninf = -INFINITY;
    const T *p = static_cast<const T *>(a.l) + row * a.ldl;
    float l[V], high = -INFINITY;
    Rank c[V];
    load_logits<T, V>(l, p, first, a.experts);
#pragma unroll
    for (int i = 0; i < V; ++i) high = fmaxf(high, l[i]);
    float m = -INFINITY, sum = 1.f;
    if (a.score == DN_SCORE_SOFTMAX) m = wave_max(high);
    if constexpr (WIDE) {
        if (a.score == DN_SCORE_SOFTMAX) {
            double s = 0.;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                c[i] = l[i] == -INFINITY ? 0. : exp((double)l[i] - (double)m);
                s += c[i];
            }
            s = total(s);
            sum = (float)s;
#pragma unroll
            for (int i = 0; i < V; ++i) c[i] *= inverse64(s);   // (of NaN, or of the 0 of a row of padding: no expert of it is ranked by it)
        } else {
            bool far = false;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                c[i] = 1. + exp(-(double)l[i]);
                far = far || (c[i] >= 1e300 && l[i] > -INFINITY);
            }
            // below -690 the steps fail.  One branch for all of a lane's: one for each takes 1.3 us more of 33 (16384 rows of 256 experts)
            if (__ballot(far))
#pragma unroll
                for (int i = 0; i < V; ++i) c[i] = 1. / c[i];
            else
#pragma unroll
                for (int i = 0; i < V; ++i) c[i] = inverse64(c[i]);
        }
        if (a.bias)
#pragma unroll
            for (int i = 0; i < V; ++i) c[i] += first + i < a.experts ? (double)a.bias[first + i] : 0.;
    } else {
        if (a.score == DN_SCORE_SOFTMAX && !a.renorm) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) s += l[i] == -INFINITY ? 0.f : expf(l[i] - m);
            sum = wave_sum(s);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = l[i];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = l[i] == -INFINITY ? ninf : c[i] == c[i] ? c[i] : (Rank)INFINITY;
    const int lanes = a.each / V;   // of a group, where it is whole lanes and a power of two of them
    if (a.top_groups < a.groups && a.each % V == 0 && (lanes & (lanes - 1)) == 0) {
        // every lane forms its group's score with the others, and then counts the groups before its own
        Rank p = ninf, q = ninf;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            q = c[i] > p ? p : c[i] > q ? c[i] : q;
            p = c[i] > p ? c[i] : p;
        }
        if (lanes > 1) best_two<0xB1>(p, q);     // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
        if (lanes > 2) best_two<0x4E>(p, q);
        if (lanes > 4) best_two<0x141>(p, q);
        if (lanes > 8) best_two<0x140>(p, q);
        for (int o = 16; o < lanes; o <<= 1) {
            const Rank x = __shfl_xor(p, o), y = __shfl_xor(q, o), low = x < p ? x : p, high = y > q ? y : q;
            p = x > p ? x : p;
            q = low > high ? low : high;
        }
        if (a.best == 2 && q > ninf) p += q;
        int before = 0;
        const int mine = lane / lanes;
        for (int g = 0; g < a.groups; ++g) {
            const Rank other = from_lane(p, g * lanes);
            before += other > p || (other == p && g < mine);
        }
        if (before >= a.top_groups)
#pragma unroll
            for (int i = 0; i < V; ++i) c[i] = ninf;
    } else if (a.top_groups < a.groups) {
        Rank score = ninf;   // lane g: group g's
        for (int g = 0; g < a.groups; ++g) {
            const int from = g * a.each, to = from + a.each;
            Rank b = ninf;
#pragma unroll
            for (int i = 0; i < V; ++i) b = first + i >= from && first + i < to && c[i] > b ? c[i] : b;
            Rank best = highest(b);
            if (a.best == 2 && best > ninf) {
                const int f = __builtin_ctzll(__ballot(b == best));
                bool skip = lane == f;
                b = ninf;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (first + i >= from && first + i < to) {
                        if (skip && c[i] == best) skip = false;   // once
                        else b = c[i] > b ? c[i] : b;
                    }
                const Rank second = highest(b);
                if (second > ninf) best += second;
            }
            if (lane == g) score = best;
        }
        uint64_t stay = 0;
        for (int n = 0; n < a.top_groups; ++n) {
            const Rank best = highest(score);
            if (!(best > ninf)) break;
            const int f = __builtin_ctzll(__ballot(score == best));
            stay |= (uint64_t)1 << f;
            if (lane == f) score = ninf;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (!(stay >> min((first + i) / a.each, 63) & 1)) c[i] = ninf;
    }
    if (WIDE && !a.bias)
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = c[i] == ninf ? ninf : l[i] == l[i] ? (Rank)l[i] : (Rank)INFINITY;
    int chosen = -1;
    float logit = -INFINITY;   // lane j: of choice j
    // Ranks in 32 bits: rounding keeps their order, so one that is alone the highest there is the highest; only equals are told apart in 64.  As
    // whole numbers of the same order: a step of the wave's maximum is one instruction, where fp32's is five.  Which of the lane's
    // experts it is, and taking it out, is a matter of one lane: its ranks are read into scalar registers, whose instructions go beside the
    // other waves' vector ones.
    int key[V], b = kNone;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        key[i] = in_order((float)c[i]);
        b = max(b, key[i]);
    }
    for (int j = 0; j < a.k; ++j) {
        const int best = highest(b);
        if (best == kNone) break;
        const uint64_t have = __ballot(b == best);
        int f = __builtin_ctzll(have), at = 0, equal = 0;
#pragma unroll
        for (int i = V - 1; i >= 0; --i)
            if (__builtin_amdgcn_readlane(key[i], f) == best) {
                at = i;
                ++equal;
            }
        if constexpr (WIDE) {
            if (have & (have - 1) || equal > 1) {   // (every lane takes part)
                Rank r = ninf;
                int mine = 0;
#pragma unroll
                for (int i = V - 1; i >= 0; --i)
                    if (key[i] == best && c[i] >= r) {
                        r = c[i];
                        mine = i;
                    }
                const Rank top = highest(r);
                f = __builtin_ctzll(__ballot(b == best && r == top));
                at = __builtin_amdgcn_readlane(mine, f);
            }
        }
        int le = 0;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (at == i) {
                le = __builtin_amdgcn_readlane(__builtin_bit_cast(int, l[i]), f);
                key[i] = lane == f ? kNone : key[i];
            }
        if (lane == j) {
            chosen = f * V + at;
            logit = __builtin_bit_cast(float, le);
        }
        b = key[0];
#pragma unroll
        for (int i = 1; i < V; ++i) b = max(b, key[i]);
    }
    float w = weight_of(a, logit, chosen >= 0, m, sum);
    if (!(sum == sum)) w = sum;   // a softmax of NaN or +inf, whose ranks name any expert
    if (lane < a.k) {
        a.expert[(int64_t)row * a.k + lane] = chosen;
        a.weight[(int64_t)row * a.k + lane] = chosen >= 0 ? w : 0.f;
    }
}

// With u = w / scale the weights without their scale and g = scale dw:
//   softmax, renorm: dl_j = u_j (g_j - sum g u);  sigmoid, renorm: the same times 1 - s_j (chosen experts only, as every s drops out of
//   the others' ratio);  sigmoid: dl_j = g_j s_j (1 - s_j);  softmax: dl = s (g - sum g s) over all of a row, g 0 but where chosen.
template <class T, int V, bool WIDE>
__global__ __launch_bounds__(kWaves * 64) void route_kernel(const RouteArgs a)
{
    const int row = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row < a.rows) route_row<T, V, WIDE>(a, row, threadIdx.x & 63);
}

template <class T, int V>
__global__ __launch_bounds__(kWaves * 64) void route_back_kernel(const RouteArgs a)
{
    const int lane = threadIdx.x & 63, row = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = lane * V;
    if (row >= a.rows) return;
    const T *p = static_cast<const T *>(a.l) + row * a.ldl;
    const int e = lane < a.k ? a.chosen[(int64_t)row * a.k + lane] : -1;
    const bool mine = (uint32_t)e < (uint32_t)a.experts;
    const float g = mine ? a.dweight[(int64_t)row * a.k + lane] * a.scale : 0.f, l = mine ? (float)p[e] : -INFINITY;
    const bool dense = a.score == DN_SCORE_SOFTMAX && !a.renorm;
    float s[V], m = 0.f, sum = 1.f, d;
    if (dense) {
        float high = -INFINITY, t = 0.f;
        load_logits<T, V>(s, p, first, a.experts);
#pragma unroll
        for (int i = 0; i < V; ++i) high = fmaxf(high, s[i]);
        m = wave_max(high);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[i] = s[i] == -INFINITY ? 0.f : expf(s[i] - m);
            t += s[i];
        }
        sum = 1.f / wave_sum(t);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = t == 0.f && m == -INFINITY ? 0.f : s[i] * sum;
        d = g;
    } else {
        RouteArgs one = a;
        one.scale = 1.f;
        float u = weight_of(one, l, mine, m, sum);   // (every lane takes part)
        if (!mine) u = 0.f;
        d = a.renorm ? u * (g - wave_sum(g * u)) : g * u;
        if (a.score == DN_SCORE_SIGMOID) d *= sigmoid_above(-l, 0.f);   // 1 - s
        if (!mine) d = 0.f;
    }
    float v[V] = {};
    for (int j = 0; j < a.k; ++j) {
        const int ej = __builtin_amdgcn_readlane(e, j);
        const float dj = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, d), j));
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += first + i == ej ? dj : 0.f;
    }
    if (dense) {
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) dot = fmaf(v[i], s[i], dot);
        dot = wave_sum(dot);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = s[i] * (v[i] - dot);
    }
    T *q = static_cast<T *>(a.dl) + (int64_t)row * a.experts + first;
    if (first + V <= a.experts) {
        typename Several<T, V>::type x;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (T)v[i];
        *reinterpret_cast<typename Several<T, V>::type *>(q) = x;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (first + i < a.experts) q[i] = (T)v[i];
    }
}

// ---- lists -----------------------------------------------------------------------------------------------------------
// A stable counting sort of the pairs by expert: workgroups count chunks, and then each adds up what lies before its own (every expert
// before, and its own expert's pairs in earlier chunks) and gives its pairs their places in order.  Counts are whole numbers: the LDS
// atomics that make them leave no order behind.
struct ListArgs {
    const int32_t *expert;
    int32_t *starts, *order, *place, *counts;   // counts [chunks][experts]
    int32_t pairs, experts, chunk, chunks;      // pairs of a chunk, a multiple of 1024
};

constexpr int kPlaceWaves = 16;

__global__ __launch_bounds__(256) void count_kernel(const ListArgs a)
{
    __shared__ int32_t count[kMostExperts];
    for (int e = threadIdx.x; e < a.experts; e += 256) count[e] = 0;
    __syncthreads();
    const int from = blockIdx.x * a.chunk, to = min(a.pairs - from, a.chunk);
    for (int i = threadIdx.x; i < to; i += 256) {
        const int e = a.expert[from + i];
        if ((uint32_t)e < (uint32_t)a.experts) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += 256) a.counts[blockIdx.x * a.experts + e] = count[e];
}

// one chunk: it counts itself
template <int WAVES>
__device__ __forceinline__ void place_chunk(const ListArgs &a, int block)
{
    constexpr int THREADS = WAVES * 64, EACH = kMostExperts / THREADS;   // EACH: experts of a thread
    __shared__ int32_t next[WAVES][kMostExperts], all[kMostExperts], earlier[kMostExperts], sums[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int from = block * a.chunk + wave * (a.chunk / WAVES), to = min(from + a.chunk / WAVES, a.pairs);   // the wave's pairs
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
        for (int e = threadIdx.x; e < a.experts; e += THREADS) next[w][e] = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) all[threadIdx.x + i * THREADS] = earlier[threadIdx.x + i * THREADS] = 0;
    // the first 256 pairs of the wave stay in registers: most often all of them
    int mine_of[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) mine_of[q] = from + q * 64 + lane < to ? a.expert[from + q * 64 + lane] : -1;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if ((uint32_t)mine_of[q] < (uint32_t)a.experts) atomicAdd(&next[wave][mine_of[q]], 1);
    for (int i = from + 256 + lane; i < to; i += 64) {
        const int e = a.expert[i];
        if ((uint32_t)e < (uint32_t)a.experts) atomicAdd(&next[wave][e], 1);
    }
    if (a.chunks > 1) {
        // all chunks' counts: as many threads to an expert as there are, each a run of chunks with its loads under way together
        const int wide = a.experts <= THREADS / 4 ? THREADS / 4 : a.experts <= THREADS / 2 ? THREADS / 2 : THREADS;
        const int run = (a.chunks * wide + THREADS - 1) / THREADS, first = (int)threadIdx.x / wide * run, last = min(first + run, a.chunks);
        for (int e = (int)threadIdx.x % wide; e < a.experts; e += wide) {
            int before = 0, sum = 0;
            for (int b0 = first; b0 < last; b0 += 16) {
                int n[16];
#pragma unroll
                for (int q = 0; q < 16; ++q) n[q] = a.counts[min(b0 + q, a.chunks - 1) * a.experts + e];
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    before += b0 + q < min(last, block) ? n[q] : 0;
                    sum += b0 + q < last ? n[q] : 0;
                }
            }
            atomicAdd(&all[e], sum);
            atomicAdd(&earlier[e], before);
        }
    }
    __syncthreads();
    // `all`: an expert's pairs; next[w]: those of earlier chunks and of earlier waves of this one
    for (int e = threadIdx.x; e < a.experts; e += THREADS) {
        int own = earlier[e];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int n = next[w][e];
            next[w][e] = own;
            own += n;
        }
        if (a.chunks == 1) all[e] = own;
    }
    __syncthreads();
    // where each expert's pairs begin
    int n[EACH], mine = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        n[i] = mine;
        mine += all[threadIdx.x * EACH + i];
    }
    int until = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(until, o);
        until += lane >= o ? v : 0;
    }
    if (lane == 63) sums[wave] = until;
    __syncthreads();
    int before = until - mine, total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int e = threadIdx.x * EACH + i;
        if (e >= a.experts) break;
        const int start = before + n[i];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) next[w][e] += start;
        if (block == 0) a.starts[e] = start;
    }
    if (block == 0 && threadIdx.x == 0) a.starts[a.experts] = total;
    __syncthreads();
    // sixty-four pairs at a time: a pair's place is its expert's next one and how many lanes below have the same expert
    auto put = [&](int i, int e) {
        const int q = i + lane;
        const bool has = (uint32_t)e < (uint32_t)a.experts;
        uint64_t same = __ballot(has);
#pragma unroll
        for (int b = 0; b < 10; ++b) {
            const uint64_t set = __ballot(has && (e >> b & 1));
            same &= e >> b & 1 ? set : ~set;
        }
        const int below = __popcll(same & (((uint64_t)1 << lane) - 1));
        int p = -1;
        if (has) {
            p = next[wave][e] + below;
            a.order[p] = q;
        }
        if (q < to) a.place[q] = p;
        // every lane has read before one of each expert writes
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
        if (has && below == 0) next[wave][e] = p + __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    };
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (from + q * 64 < to) put(from + q * 64, mine_of[q]);
    for (int i = from + 256; i < to; i += 64) put(i, i + lane < to ? a.expert[i + lane] : -1);
    for (int p = max(from, total) + lane; p < to; p += 64) a.order[p] = -1;
}

__global__ __launch_bounds__(kPlaceWaves * 64) void place_kernel(const ListArgs a)
{
    place_chunk<kPlaceWaves>(a, blockIdx.x);
}

// Few rows: choices and lists in one launch of one workgroup, a wave a row at a time.
template <class T, int V, bool WIDE>
__global__ __launch_bounds__(256) void route_few_kernel(const RouteArgs a, const ListArgs lists)
{
    for (int row = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); row < a.rows; row += 4) route_row<T, V, WIDE>(a, row, threadIdx.x & 63);
    __threadfence_block();
    __syncthreads();
    place_chunk<4>(lists, 0);
}

// Up to 8192 pairs are one workgroup's, which counts them itself (5204 pairs of 60 experts: 9.0 us, in chunks 3.4 and 5.8); of more, chunks of at
// least 1024, and at most 128 of them, as each workgroup reads all counts.
constexpr int kMostChunks = 128, kOneChunk = 8192;
int chunk_of(int pairs)
{
    const int n = pairs <= kOneChunk ? 1 : kMostChunks;
    return (pairs + 1024 * n - 1) / (1024 * n) * 1024;
}

dn_status sizes(int32_t rows, int32_t experts, int32_t k)
{
    return rows < 1 || experts < 1 || k < 1 || experts > kMostExperts || k > kMostChoices || rows >= kMostRows || (int64_t)rows * k >= kMostPairs
               ? DN_ERR_SHAPE
               : DN_OK;
}

size_t lists_bytes(int32_t rows, int32_t experts, int32_t k)
{
    const int pairs = rows * k, chunk = chunk_of(pairs), chunks = (pairs + chunk - 1) / chunk;
    return chunks == 1 ? 0 : up256((size_t)chunks * experts * sizeof(int32_t));
}

hipError_t launch_lists(ListArgs a, hipStream_t s)
{
    a.chunk = chunk_of(a.pairs);
    a.chunks = (a.pairs + a.chunk - 1) / a.chunk;
    if (a.chunks > 1) launch_kernel(count_kernel, dim3(a.chunks), dim3(256), 0, s, a);
    launch_kernel(place_kernel, dim3(a.chunks), dim3(kPlaceWaves * 64), 0, s, a);
    return hipGetLastError();
}

dn_status route_of(const dn_route_desc *d, RouteArgs &a)
{
    a = RouteArgs{};
    if (!d || !type_ok(d->type) || (d->score != DN_SCORE_SOFTMAX && d->score != DN_SCORE_SIGMOID)) return DN_ERR_INVALID_ARG;
    if (!isfinite(d->scale) || (d->group_best != 1 && d->group_best != 2) || (d->renorm != 0 && d->renorm != 1)) return DN_ERR_INVALID_ARG;
    const dn_status s = sizes(d->rows, d->experts, d->k);
    if (s != DN_OK) return s;
    if (d->groups < 1 || d->groups > 64 || d->experts % d->groups || d->top_groups < 1 || d->top_groups > d->groups) return DN_ERR_SHAPE;
    a.each = d->experts / d->groups;
    if (d->k > a.each * d->top_groups || (d->groups > 1 && d->group_best > a.each)) return DN_ERR_SHAPE;
    a.ldl = d->ldl;
    const dn_status r = row_length(d->type, a.ldl, d->experts);
    if (r != DN_OK) return r;
    a.rows = d->rows;
    a.experts = d->experts;
    a.k = d->k;
    a.groups = d->groups;
    a.top_groups = d->top_groups;
    a.best = d->group_best;
    a.score = d->score;
    a.renorm = d->renorm;
    a.scale = d->scale;
    return DN_OK;
}

// Rows of one workgroup, a wave a row at a time.  So, and in launches of their own, us: up to four rows 8.2 and 10.8 (128 experts, 8 choices; 256 with a
// bias; 16), 20.3 to 21.0 and 21.0 to 21.7 (1024 experts, 16 choices, a bias); eight rows 8.1 and 10.7, 11.7 and 11.0, 8.1 and 10.8, 37.4 and 22.2: five to
// eight rows of many experts lose by it.  Sixteen: 12.3 and 10.8, 20.1 and 11.0, 7.9 and 10.8, 70 and 22.
constexpr int kOneLaunchRows = 8;

template <class T, int V, bool WIDE>
void choose_as(const RouteArgs &a, const ListArgs *lists, hipStream_t s)
{
    if (lists) launch_kernel(route_few_kernel<T, V, WIDE>, dim3(1), dim3(256), 0, s, a, *lists);
    else launch_kernel(route_kernel<T, V, WIDE>, dim3((unsigned)((a.rows + kWaves - 1) / kWaves)), dim3(kWaves * 64), 0, s, a);
}
template <class T, int V>
void forward_as(const RouteArgs &a, const ListArgs *lists, hipStream_t s)
{
    if (a.bias || (a.top_groups < a.groups && a.best == 2)) choose_as<T, V, true>(a, lists, s);
    else choose_as<T, V, false>(a, lists, s);
}
template <class T, int V>
void backward_as(const RouteArgs &a, hipStream_t s)
{
    launch_kernel(route_back_kernel<T, V>, dim3((unsigned)((a.rows + kWaves - 1) / kWaves)), dim3(kWaves * 64), 0, s, a);
}
template <class T>
hipError_t run(const RouteArgs &a, bool back, const ListArgs *lists, hipStream_t s)
{
    if (a.experts <= 64) back ? backward_as<T, 1>(a, s) : forward_as<T, 1>(a, lists, s);
    else if (a.experts <= 128) back ? backward_as<T, 2>(a, s) : forward_as<T, 2>(a, lists, s);
    else if (a.experts <= 256) back ? backward_as<T, 4>(a, s) : forward_as<T, 4>(a, lists, s);
    else if (a.experts <= 512) back ? backward_as<T, 8>(a, s) : forward_as<T, 8>(a, lists, s);
    else back ? backward_as<T, 16>(a, s) : forward_as<T, 16>(a, lists, s);
    return hipGetLastError();
}
hipError_t launch_route(int type, const RouteArgs &a, bool back, const ListArgs *lists, hipStream_t s)
{
    return type == DN_F32 ? run<float>(a, back, lists, s) : type == DN_F16 ? run<f16>(a, back, lists, s) : run<bf16>(a, back, lists, s);
}

template <class... P>
bool words(const P *...p)
{
    return multiples(DN_F32, p...);
}

}  // namespace
}  // namespace dn

using namespace dn;

extern "C" {

size_t dn_route_workspace_bytes(int32_t rows, int32_t experts, int32_t k)
{
    return sizes(rows, experts, k) == DN_OK ? lists_bytes(rows, experts, k) : kBad;
}

dn_status dn_route_lists(const int32_t *expert_dev, int32_t rows, int32_t experts, int32_t k, int32_t *starts_dev, int32_t *order_dev,
                         int32_t *place_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!expert_dev || !starts_dev || !order_dev || !place_dev || !words(expert_dev, starts_dev, order_dev, place_dev)) return DN_ERR_INVALID_ARG;
    dn_status s = sizes(rows, experts, k);
    if (s != DN_OK) return s;
    if ((s = workspace(lists_bytes(rows, experts, k), workspace_dev, workspace_bytes)) != DN_OK) return s;
    return device(launch_lists({expert_dev, starts_dev, order_dev, place_dev, static_cast<int32_t *>(workspace_dev), rows * k, experts, 0, 0},
                               (hipStream_t)hip_stream));
}

dn_status dn_route_forward(const dn_route_desc *d, const void *L_dev, const float *bias_dev, int32_t *expert_dev, float *weight_dev,
                           int32_t *starts_dev, int32_t *order_dev, int32_t *place_dev, void *workspace_dev,
                           size_t workspace_bytes, void *hip_stream)
{
    RouteArgs a;
    dn_status s = route_of(d, a);
    if (s != DN_OK) return s;
    const bool lists = starts_dev || order_dev || place_dev;
    if (!L_dev || !expert_dev || !weight_dev || (lists && !(starts_dev && order_dev && place_dev))) return DN_ERR_INVALID_ARG;
    if (!multiples(d->type, L_dev) || !words(bias_dev, expert_dev, weight_dev, starts_dev, order_dev, place_dev)) return DN_ERR_INVALID_ARG;
    if (lists && (s = workspace(lists_bytes(d->rows, d->experts, d->k), workspace_dev, workspace_bytes)) != DN_OK) return s;
    a.l = L_dev;
    a.bias = bias_dev;
    a.expert = expert_dev;
    a.weight = weight_dev;
    const hipStream_t stream = (hipStream_t)hip_stream;
    ListArgs l{expert_dev, starts_dev, order_dev, place_dev, static_cast<int32_t *>(workspace_dev), d->rows * d->k, d->experts, 0, 0};
    if (lists && d->rows <= kOneLaunchRows) {
        l.chunk = chunk_of(l.pairs);
        l.chunks = 1;
        return device(launch_route(d->type, a, false, &l, stream));
    }
    if (launch_route(d->type, a, false, nullptr, stream) != hipSuccess) return DN_ERR_DEVICE;
    return lists ? device(launch_lists(l, stream)) : DN_OK;
}

dn_status dn_route_backward(const dn_route_desc *d, const void *L_dev, const int32_t *expert_dev, const float *dweight_dev,
                            void *dL_dev, void *hip_stream)
{
    RouteArgs a;
    const dn_status s = route_of(d, a);
    if (s != DN_OK) return s;
    if (!L_dev || !expert_dev || !dweight_dev || !dL_dev) return DN_ERR_INVALID_ARG;
    if (!multiples(d->type, L_dev, dL_dev) || !words(expert_dev, dweight_dev)) return DN_ERR_INVALID_ARG;
    a.l = L_dev;
    a.chosen = expert_dev;
    a.dweight = dweight_dev;
    a.dl = dL_dev;
    return device(launch_route(d->type, a, true, nullptr, (hipStream_t)hip_stream));
}

}  // extern "C"
