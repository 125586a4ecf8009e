// The norm after a block with its gate, scale and residual, and the norm before the next block, in one pass over memory:
//     c = post(b),  x' = x + scale gate * c,  n = pre(x')
// A row lives in the registers of the NT threads that share it, C pieces of eight elements each; its statistics are sums over
// those threads, in fp32, the mean first and then the centred squares.  Bound by memory: forward four rows of d elements read or
// written, backward six; 16384 x 4096, bf16, 98 to 101 us (5.4 TB/s) and 174 to 192, with 8 for the join (4.4).  The backward pass forms the
// statistics again from the rows that it reads anyway, so nothing is kept from the forward pass.
// Wider rows keep their sums in scratch memory too: bf16 8192 x 8192 120 us (4.5 TB/s) and 320 (2.5), 4096 x 16384 243 (2.2) and 1206
// (0.7); fp32 backward 441 (3.7) and 1417 (1.1).
//
// Backward, from dx' and dn (x is x'):  dx = dx' + pre'(dn),  dc = scale gate * dx,  db = post'(dc),  and sums over rows:
// dgate = scale dx * c (rows of its group), dpost_w = dc * b^, dpost_b = dc, dpre_w = dn * x^, dpre_b = dn, where ^ is the
// normalised row and norm'(q) = r (q w - mean(q w) - ^ mean(q w ^)) (the first mean: layer norm only).  A workgroup takes a
// run of rows and keeps its sums in registers; a second launch adds the parts of all workgroups in order.
#include "dn_ffn.h"
#include "dn_wave.h"

namespace dn {
namespace {

typedef float v2f __attribute__((ext_vector_type(2)));

// sums over the NT threads of a row, in all of them
template <int NT>
struct RowSum {
    v2f *slots;   // two times NT / 64
    int turn = 0;
    __device__ __forceinline__ v2f operator()(v2f v)
    {
        v[0] = wave_sum(v[0]);
        v[1] = wave_sum(v[1]);
        if (NT == 64) return v;
        // two sets of slots in turn: whoever writes one again has passed the barrier that its readers came to afterwards
        v2f *s = slots + turn * (NT / 64);
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        // a barrier that leaves the next row's loads under way
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __asm__ volatile("" ::: "memory");
        v = s[0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) v += s[w];
        return v;
    }
};

// A thread's C pieces of a row, as they lie in memory.
template <class T, int NT, int C>
struct Raw {
    typename Eight<T>::type v[C];
    __device__ __forceinline__ void get(const void *p, int64_t at, int t, int d)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int n = (c * NT + t) * 8;
            v[c] = get8<T>(p, at + n, d - n);
        }
    }
    __device__ __forceinline__ float operator()(int c, int j) const { return (float)v[c][j]; }
    // keeps a loop from holding the numbers as fp32, in twice the registers
    __device__ __forceinline__ void stay()
    {
        if constexpr (sizeof(T) == 2)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                v4u w = __builtin_bit_cast(v4u, v[c]);
                __asm__("" : "+v"(w));
                v[c] = __builtin_bit_cast(typename Eight<T>::type, w);
            }
    }
};

// every element of a thread's pieces
#define EACH(c, j)                                                                                                                 \
    _Pragma("unroll") for (int c = 0; c < C; ++c) _Pragma("unroll") for (int j = 0; j < 8; ++j)

// STREAM: rows of results, past the L2 (2048 x 2048, bf16: forward 10.0 -> 9.1 us, backward 17.4 -> 16.8)
template <class T, int NT, int C, bool STREAM>
__device__ __forceinline__ void store_row(void *p, int64_t at, const float (&v)[C][8], int t, int d)
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int n = (c * NT + t) * 8;
        store8<T, false, STREAM>(p, at + n, v[c], d - n);
    }
}

// v and w normalised in place; elements past the row stay 0.  Returns the reciprocals of their deviations.
template <int NT, int C>
__device__ __forceinline__ v2f normalise(float (&v)[C][8], float (&w)[C][8], int how_v, int how_w, int t, int d, float eps,
                                         RowSum<NT> &sum)
{
    if (how_v == DN_NORM_LAYER || how_w == DN_NORM_LAYER) {
        v2f s = {};
        EACH(c, j)
        {
            s[0] += v[c][j];
            s[1] += w[c][j];
        }
        s = sum(s) / (float)d;
        const float mv = how_v == DN_NORM_LAYER ? s[0] : 0.f, mw = how_w == DN_NORM_LAYER ? s[1] : 0.f;
        EACH(c, j)
        if ((c * NT + t) * 8 + j < d) {
            v[c][j] -= mv;
            w[c][j] -= mw;
        }
    }
    v2f q = {};
    EACH(c, j)
    {
        q[0] += v[c][j] * v[c][j];
        q[1] += w[c][j] * w[c][j];
    }
    q = sum(q) / (float)d;
    const v2f r = {how_v ? 1.f / sqrtf(q[0] + eps) : 1.f, how_w ? 1.f / sqrtf(q[1] + eps) : 1.f};
    EACH(c, j)
    {
        v[c][j] *= r[0];
        w[c][j] *= r[1];
    }
    return r;
}

// AHEAD: a row's reads go out before the row before it is worked on.
template <class T, int NT, int C, bool AHEAD>
__global__ __launch_bounds__(NT < 128 ? 256 : NT) void norm_forward_kernel(const NormArgs a)
{
    constexpr int RB = NT < 128 ? 256 / NT : 1;   // rows of a workgroup at a time, a wave each
    __shared__ v2f slots[2 * (NT / 64)];
    RowSum<NT> sum{slots};
    const int t = threadIdx.x % NT;
    Raw<T, NT, C> post_w, post_b, pre_w, pre_b, raw_x, raw_b, raw_gate;
    if (a.post_w) post_w.get(a.post_w, 0, t, a.d);
    if (a.post_b) post_b.get(a.post_b, 0, t, a.d);
    if (a.pre_w) pre_w.get(a.pre_w, 0, t, a.d);
    if (a.pre_b) pre_b.get(a.pre_b, 0, t, a.d);
    auto fetch = [&](int64_t m) {
        raw_x.get(a.x, m * a.d, t, a.d);
        if (a.b) raw_b.get(a.b, m * a.d, t, a.d);
        if (a.gate) raw_gate.get(a.gate, m / a.group * a.d, t, a.d);
    };
    const int64_t step = (int64_t)gridDim.x * RB;
    int64_t m = (int64_t)blockIdx.x * RB + threadIdx.x / NT;
    if (AHEAD && m < a.rows) fetch(m);
    for (; m < a.rows; m += step) {
        if (!AHEAD) fetch(m);
        post_w.stay();
        post_b.stay();
        pre_w.stay();
        pre_b.stay();
        const int64_t at = m * a.d;
        float x[C][8], b[C][8] = {}, gate[C][8], none[C][8] = {};
        EACH(c, j) x[c][j] = raw_x(c, j);
        if (a.b) EACH(c, j) b[c][j] = raw_b(c, j);
        if (a.gate) EACH(c, j) gate[c][j] = raw_gate(c, j);
        if (AHEAD && m + step < a.rows) fetch(m + step);
        if (a.b) {
            if (a.post) {
                normalise<NT, C>(b, none, a.post, 0, t, a.d, a.eps, sum);
                if (a.post_w) EACH(c, j) b[c][j] *= post_w(c, j);
                if (a.post_b) EACH(c, j) b[c][j] += post_b(c, j);
            }
            if (a.gate) EACH(c, j) b[c][j] *= gate[c][j];
            EACH(c, j) x[c][j] += a.scale * b[c][j];
            store_row<T, NT, C, true>(a.x_out, at, x, t, a.d);
        }
        if (a.pre) {   // of x' before it is rounded to T
            normalise<NT, C>(x, none, a.pre, 0, t, a.d, a.eps, sum);
            if (a.pre_w) EACH(c, j) x[c][j] *= pre_w(c, j);
            if (a.pre_b) EACH(c, j) x[c][j] += pre_b(c, j);
            store_row<T, NT, C, true>(a.n_out, at, x, t, a.d);
        }
    }
}

// q becomes r (q - mean(q) - hat mean(q hat))
template <int NT, int C>
__device__ __forceinline__ void norm_back(float (&q)[C][8], const float (&hat)[C][8], int how, float r, int d, RowSum<NT> &sum)
{
    v2f s = {};
    EACH(c, j)
    {
        s[0] += q[c][j] * hat[c][j];
        s[1] += q[c][j];
    }
    s = sum(s) / (float)d;
    const float mean = how == DN_NORM_LAYER ? s[1] : 0.f;
    EACH(c, j) q[c][j] = r * (q[c][j] - hat[c][j] * s[0] - mean);
}

// The sums over rows that a workgroup hands on, in this order, [parts][d] each where they are wanted; the gate's are the last.
enum Sums : int { S_POST_W, S_POST_B, S_PRE_W, S_PRE_B, S_GATE, S_COUNT };

// With a gate that all rows share, scale dx summed alone (s0) and times b^ (s1) give all of the block's sums: dpost_w = gate s1,
// dpost_b = gate s0, dgate = w s1 + shift s0.  GROUPS: the part is whole groups, whose dgate is written as each ends and whose
// dpost are added up.
template <class T, int NT, int C, bool AHEAD, bool GROUPS>
__global__ __launch_bounds__(NT, NT <= 512 && C == 1 && sizeof(T) == 2 && !GROUPS ? 4 : 1) void norm_backward_kernel(const NormArgs a)
{
    __shared__ v2f slots[2 * (NT / 64)];
    RowSum<NT> sum{slots};
    const int t = threadIdx.x, part = blockIdx.x;
    int64_t m, end;
    if (!GROUPS) {
        const int64_t g = part / a.group_parts;
        m = g * a.group + (int64_t)(part % a.group_parts) * a.part_rows;
        end = min(min(m + a.part_rows, (g + 1) * a.group), (int64_t)a.rows);
    } else {
        m = (int64_t)part * a.part_rows;
        end = min(m + a.part_rows, (int64_t)a.rows);
    }
    Raw<T, NT, C> post_w, post_b, pre_w, gate, raw_x, raw_b, raw_dx, raw_dn;
    if (a.post_w) post_w.get(a.post_w, 0, t, a.d);
    if (a.post_b) post_b.get(a.post_b, 0, t, a.d);
    if (a.pre_w) pre_w.get(a.pre_w, 0, t, a.d);
    if (a.gate) gate.get(a.gate, m / a.group * a.d, t, a.d);
    auto fetch = [&](int64_t r) {
        const int64_t at = r * a.d;
        if (a.pre) raw_x.get(a.x, at, t, a.d);
        if (a.b) raw_b.get(a.b, at, t, a.d);
        if (a.pre) raw_dn.get(a.dn, at, t, a.d);
        if (a.dx_out) raw_dx.get(a.dx_out, at, t, a.d);
    };
    float sums[S_GATE][C][8] = {}, s0[C][8] = {}, s1[C][8] = {};
    auto close = [&]() {   // a gate's rows, or this part of them: their dpost, and dgate in s1
        EACH(c, j)
        {
            const float k = a.gate ? gate(c, j) : 1.f;
            sums[S_POST_W][c][j] += k * s1[c][j];
            sums[S_POST_B][c][j] += k * s0[c][j];
            s1[c][j] = (a.post_w ? s1[c][j] * post_w(c, j) : s1[c][j]) + (a.post_b ? s0[c][j] * post_b(c, j) : 0.f);
        }
    };
    if (AHEAD) fetch(m);
    for (; m < end; ++m) {
        if (!AHEAD) fetch(m);
        post_w.stay();
        post_b.stay();
        pre_w.stay();
        gate.stay();
        const int64_t at = m * a.d;
        float x[C][8] = {}, b[C][8] = {}, g[C][8] = {}, q[C][8] = {};
        if (a.pre) EACH(c, j) x[c][j] = raw_x(c, j);
        if (a.b) EACH(c, j) b[c][j] = raw_b(c, j);
        if (a.pre) EACH(c, j) q[c][j] = raw_dn(c, j);
        if (a.dx_out) EACH(c, j) g[c][j] = raw_dx(c, j);
        if (AHEAD && m + 1 < end) fetch(m + 1);
        v2f r = {1.f, 1.f};
        if (a.pre || a.post) r = normalise<NT, C>(x, b, a.pre, a.post, t, a.d, a.eps, sum);
        if (a.pre) {
            EACH(c, j)
            {
                sums[S_PRE_W][c][j] += q[c][j] * x[c][j];
                sums[S_PRE_B][c][j] += q[c][j];
            }
            if (a.pre_w) EACH(c, j) q[c][j] *= pre_w(c, j);
            norm_back<NT, C>(q, x, a.pre, r[0], a.d, sum);
            EACH(c, j) g[c][j] += q[c][j];
        }
        store_row<T, NT, C, true>(a.dx, at, g, t, a.d);
        if (!a.b) continue;
        EACH(c, j)
        {
            g[c][j] *= a.scale;
            s0[c][j] += g[c][j];
            s1[c][j] += g[c][j] * b[c][j];
        }
        if (a.gate) EACH(c, j) g[c][j] *= gate(c, j);
        if (a.post) {
            if (a.post_w) EACH(c, j) g[c][j] *= post_w(c, j);
            norm_back<NT, C>(g, b, a.post, r[1], a.d, sum);
        }
        store_row<T, NT, C, true>(a.db, at, g, t, a.d);
        if (GROUPS && (m + 1 == end || (m + 1) % a.group == 0)) {   // a gate's last row
            close();
            if (a.dgate) {
                const int64_t row = m / a.group * a.d;
                if (a.f32_out) store_row<float, NT, C, false>(a.dgate, row, s1, t, a.d);
                else store_row<T, NT, C, true>(a.dgate, row, s1, t, a.d);
            }
            EACH(c, j) s0[c][j] = s1[c][j] = 0.f;
            if (a.gate && m + 1 < end) gate.get(a.gate, (m + 1) / a.group * a.d, t, a.d);
        }
    }
    if (!GROUPS) close();
    void *const want[S_COUNT] = {a.dpost_w, a.dpost_b, a.dpre_w, a.dpre_b, GROUPS ? nullptr : a.dgate};
    float *ws = a.ws;
#pragma unroll
    for (int k = 0; k < S_COUNT; ++k)
        if (want[k]) {
            store_row<float, NT, C, false>(ws, (int64_t)part * a.d, k < S_GATE ? sums[k < S_GATE ? k : 0] : s1, t, a.d);
            ws += (int64_t)a.parts * a.d;
        }
}
#undef EACH

// Column sums of the workgroups' parts, in order.  A workgroup takes 32 columns of one set of parts, sixteen threads a column;
// blockIdx.y: a parameter, then the gate's groups.
template <class T>
__global__ __launch_bounds__(512) void norm_join_kernel(const NormArgs a)
{
    __shared__ float share[16][32];
    const int n = blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
    void *const want[S_COUNT] = {a.dpost_w, a.dpost_b, a.dpre_w, a.dpre_b, a.group_parts > 1 ? a.dgate : nullptr};
    int which = 0, set = 0, y = blockIdx.y;
    for (; which < S_GATE; ++which)
        if (want[which]) {
            if (y == 0) break;
            --y;
            ++set;
        }
    const int from = which == S_GATE ? y * a.group_parts : 0;
    const int to = which == S_GATE ? min(a.parts, from + a.group_parts) : a.parts;
    float s = 0.f;
    if (n < a.d)
#pragma unroll 8
        for (int p = from + lane; p < to; p += 16) s += a.ws[((int64_t)set * a.parts + p) * a.d + n];
    share[lane][threadIdx.x & 31] = s;
    __syncthreads();
    if (lane || n >= a.d) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) s += share[k][threadIdx.x & 31];
    const int64_t at = which == S_GATE ? (int64_t)y * a.d + n : n;
    if (a.f32_out) static_cast<float *>(want[which])[at] = s;
    else static_cast<T *>(want[which])[at] = (T)s;
}

template <class T, int NT, int C>
hipError_t forward(const NormArgs &a, hipStream_t s)
{
    constexpr int block = NT < 128 ? 256 : NT, rows = NT < 128 ? 256 / NT : 1;
    // as many workgroups as run at once, so that they end together: 20 waves a compute unit, 16 of fp32, by their registers.  (Rows of two
    // pieces a thread take more: of 512 threads one workgroup runs at a time, and twice as many are launched.)
    constexpr int most = 256 * ((sizeof(T) == 2 ? 1280 : 1024) / block > 0 ? (sizeof(T) == 2 ? 1280 : 1024) / block : 1);
    const int64_t need = ((int64_t)a.rows + rows - 1) / rows;
    launch_kernel(norm_forward_kernel<T, NT, C, C == 1>, dim3((unsigned)(need < most ? need : most)), dim3(block), 0, s, a);
    return hipGetLastError();
}

template <class T, int NT, int C>
hipError_t backward(const NormArgs &a, hipStream_t s)
{
    if (a.group_parts > 1) launch_kernel(norm_backward_kernel<T, NT, C, C == 1, false>, dim3((unsigned)a.parts), dim3(NT), 0, s, a);
    else launch_kernel(norm_backward_kernel<T, NT, C, C == 1, true>, dim3((unsigned)a.parts), dim3(NT), 0, s, a);
    const hipError_t e = hipGetLastError();
    const bool gates = a.dgate && a.group_parts > 1;
    const int params = (a.dpost_w != nullptr) + (a.dpost_b != nullptr) + (a.dpre_w != nullptr) + (a.dpre_b != nullptr);
    const int groups = gates ? (int)(((int64_t)a.rows + a.group - 1) / a.group) : 0;
    if (e != hipSuccess || params + groups == 0) return e;
    launch_kernel(norm_join_kernel<T>, dim3((unsigned)((a.d + 31) / 32), (unsigned)(params + groups)), dim3(512), 0, s, a);
    return hipGetLastError();
}

// As many threads as a row needs at eight columns each, by halves of powers of two: those past its end wait with the others.  65536 rows of
// 1024, bf16, on 128 threads 105 us forward and 183 backward (on 256: 170 and 274), of 520 98 and 171 (180 and 293).
template <class T>
hipError_t forward_by_width(const NormArgs &a, hipStream_t s)
{
    if (a.d <= 512) return forward<T, 64, 1>(a, s);
    if (a.d <= 1024) return forward<T, 128, 1>(a, s);
    if (a.d <= 1536) return forward<T, 192, 1>(a, s);
    if (a.d <= 2048) return forward<T, 256, 1>(a, s);
    if (a.d <= 8 * 384) return forward<T, 384, 1>(a, s);
    if (a.d <= 4096) return forward<T, 512, 1>(a, s);
    if (a.d <= 8192) return forward<T, 512, 2>(a, s);
    return forward<T, 1024, 2>(a, s);
}
template <class T>
hipError_t backward_by_width(const NormArgs &a, hipStream_t s)
{
    if (a.d <= 512) return backward<T, 64, 1>(a, s);
    if (a.d <= 1024) return backward<T, 128, 1>(a, s);
    if (a.d <= 1536) return backward<T, 192, 1>(a, s);
    if (a.d <= 2048) return backward<T, 256, 1>(a, s);
    if (a.d <= 8 * 384) return backward<T, 384, 1>(a, s);
    if (a.d <= 4096) return backward<T, 512, 1>(a, s);
    if (a.d <= 8192) return backward<T, 512, 2>(a, s);
    return backward<T, 1024, 2>(a, s);
}

}  // namespace

size_t norm_backward_plan(int type, NormArgs &a)
{
    // parts: as many workgroups as run at once, so that they end together (more parts would write and read more partial sums too).
    // Waves of a compute unit go by the registers: 16, 8 of fp32 and of rows of two pieces a thread.  (That is the kernel for parts of a
    // gate's rows.  The one for whole gates takes 155 to 159 registers in 16 bits, so that 12 waves run, and of 512 threads one workgroup at
    // a time, where two are planned: 16384 x 4096 with a gate a row 278 us, 3.9 TB/s.)
    const int64_t threads = a.d <= 512 ? 64 : a.d <= 1024 ? 128 : a.d <= 1536 ? 192 : a.d <= 2048 ? 256 : a.d <= 8 * 384 ? 384 : a.d <= 8192 ? 512 : 1024;
    auto rows_of = [&](int waves) {
        const int64_t most = 256 * (waves * 64 / threads > 0 ? waves * 64 / threads : 1), part = ((int64_t)a.rows + most - 1) / most;
        return part < 4 ? (int64_t)4 : part;
    };
    const bool few = type == DN_F32 || a.d > 4096;
    int64_t part = rows_of(few ? 8 : 16);
    if (a.group > part) {
        a.group_parts = (int32_t)(((int64_t)a.group + part - 1) / part);   // two at least
    } else {
        a.group_parts = 1;
        part = part / a.group * a.group;
    }
    a.part_rows = (int32_t)part;
    if (a.group_parts > 1) {
        // the last group may be short: only the parts that have rows
        const int64_t whole = a.rows / a.group, rest = a.rows % a.group;
        a.parts = (int32_t)(whole * a.group_parts + (rest + part - 1) / part);
    } else {
        a.parts = (int32_t)(((int64_t)a.rows + part - 1) / part);
    }
    return (size_t)S_COUNT * (size_t)a.parts * (size_t)a.d * sizeof(float);
}

hipError_t launch_norm_forward(int type, const NormArgs &a, hipStream_t s)
{
    return type == DN_F32 ? forward_by_width<float>(a, s) : type == DN_F16 ? forward_by_width<f16>(a, s) : forward_by_width<bf16>(a, s);
}
hipError_t launch_norm_backward(int type, const NormArgs &a, hipStream_t s)
{
    return type == DN_F32 ? backward_by_width<float>(a, s) : type == DN_F16 ? backward_by_width<f16>(a, s) : backward_by_width<bf16>(a, s);
}

}  // namespace dn
