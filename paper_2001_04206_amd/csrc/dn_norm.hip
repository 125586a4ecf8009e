// The norm after a block with its gate, scale and residual, and the norm before the next block, in one pass over memory:
//     c = post(b),  x' = x + scale gate * c,  n = pre(x')
// A row lives in the registers of the NT threads that share it, C pieces of eight elements each; its statistics are sums over
// those threads, in fp32, the mean first and then the centred squares.  Bound by memory: forward four rows of d elements read or
// written, backward six.  The backward pass forms the statistics again from the rows that it reads anyway, so nothing is kept
// from the forward pass.
//
// Backward, from dx' and dn (x is x'):  dx = dx' + pre'(dn),  dc = scale gate * dx,  db = post'(dc),  and sums over rows:
// dgate = scale dx * c (rows of its group), dpost_w = dc * b^, dpost_b = dc, dpre_w = dn * x^, dpre_b = dn, where ^ is the
// normalised row and norm'(q) = r (q w - mean(q w) - ^ mean(q w ^)) (the first mean: layer norm only).  A workgroup takes a
// run of rows and keeps its sums in registers; a second launch adds the parts of all workgroups in order.
#include "dn_ffn.h"

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
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            v[0] += __shfl_xor(v[0], o);
            v[1] += __shfl_xor(v[1], o);
        }
        if (NT == 64) return v;
        // two sets of slots in turn: whoever writes one again has passed the barrier that its readers came to afterwards
        v2f *s = slots + turn * (NT / 64);
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) v += s[w];
        return v;
    }
};

template <class T, int NT, int C>
__device__ __forceinline__ void load_row(float (&v)[C][8], const void *p, int64_t at, int t, int d)
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int n = (c * NT + t) * 8;
        load8<T>(v[c], p, at + n, d - n);
    }
}
template <class T, int NT, int C>
__device__ __forceinline__ void store_row(void *p, int64_t at, const float (&v)[C][8], int t, int d)
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int n = (c * NT + t) * 8;
        store8<T>(p, at + n, v[c], d - n);
    }
}

// v and w normalised in place; elements past the row stay 0.  r: the reciprocals of their deviations.
template <int NT, int C>
__device__ __forceinline__ v2f normalise(float (&v)[C][8], float (&w)[C][8], int how_v, int how_w, int t, int d, float eps,
                                         RowSum<NT> &sum)
{
    if (how_v == DN_NORM_LAYER || how_w == DN_NORM_LAYER) {
        v2f s = {};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[0] += v[c][j];
                s[1] += w[c][j];
            }
        s = sum(s) / (float)d;
        const float mv = how_v == DN_NORM_LAYER ? s[0] : 0.f, mw = how_w == DN_NORM_LAYER ? s[1] : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if ((c * NT + t) * 8 + j < d) {
                    v[c][j] -= mv;
                    w[c][j] -= mw;
                }
    }
    v2f q = {};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            q[0] += v[c][j] * v[c][j];
            q[1] += w[c][j] * w[c][j];
        }
    q = sum(q) / (float)d;
    const v2f r = {how_v ? 1.f / sqrtf(q[0] + eps) : 1.f, how_w ? 1.f / sqrtf(q[1] + eps) : 1.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[c][j] *= r[0];
            w[c][j] *= r[1];
        }
    return r;
}

template <class T, int NT, int C>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_forward_kernel(const NormArgs a)
{
    constexpr int RB = NT < 256 ? 256 / NT : 1;   // rows of a workgroup at a time
    __shared__ v2f slots[2 * (NT / 64)];
    RowSum<NT> sum{slots};
    const int t = threadIdx.x % NT;
    for (int64_t m = (int64_t)blockIdx.x * RB + threadIdx.x / NT; m < a.rows; m += (int64_t)gridDim.x * RB) {
        const int64_t at = m * a.d;
        float x[C][8], none[C][8] = {};
        load_row<T, NT, C>(x, a.x, at, t, a.d);
        if (a.b) {
            float b[C][8], p[C][8];
            load_row<T, NT, C>(b, a.b, at, t, a.d);
            if (a.post) {
                normalise<NT, C>(b, none, a.post, 0, t, a.d, a.eps, sum);
                if (a.post_w) {
                    load_row<T, NT, C>(p, a.post_w, 0, t, a.d);
#pragma unroll
                    for (int c = 0; c < C; ++c)
#pragma unroll
                        for (int j = 0; j < 8; ++j) b[c][j] *= p[c][j];
                }
                if (a.post_b) {
                    load_row<T, NT, C>(p, a.post_b, 0, t, a.d);
#pragma unroll
                    for (int c = 0; c < C; ++c)
#pragma unroll
                        for (int j = 0; j < 8; ++j) b[c][j] += p[c][j];
                }
            }
            if (a.gate) {
                load_row<T, NT, C>(p, a.gate, m / a.group * a.d, t, a.d);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) b[c][j] *= p[c][j];
            }
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] += a.scale * b[c][j];
            store_row<T, NT, C>(a.x_out, at, x, t, a.d);
        }
        if (a.pre) {   // of x' before it is rounded to T
            float p[C][8];
            normalise<NT, C>(x, none, a.pre, 0, t, a.d, a.eps, sum);
            if (a.pre_w) {
                load_row<T, NT, C>(p, a.pre_w, 0, t, a.d);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[c][j] *= p[c][j];
            }
            if (a.pre_b) {
                load_row<T, NT, C>(p, a.pre_b, 0, t, a.d);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[c][j] += p[c][j];
            }
            store_row<T, NT, C>(a.n_out, at, x, t, a.d);
        }
    }
}

// q becomes r (q w - mean(q w) - hat mean(q w hat))
template <class T, int NT, int C>
__device__ __forceinline__ void norm_back(float (&q)[C][8], const float (&hat)[C][8], const void *w, int how, float r, int t, int d,
                                          RowSum<NT> &sum)
{
    if (w) {
        float p[C][8];
        load_row<T, NT, C>(p, w, 0, t, d);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) q[c][j] *= p[c][j];
    }
    v2f s = {};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s[0] += q[c][j] * hat[c][j];
            s[1] += q[c][j];
        }
    s = sum(s) / (float)d;
    const float mean = how == DN_NORM_LAYER ? s[1] : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[c][j] = r * (q[c][j] - hat[c][j] * s[0] - mean);
}

// The sums over rows that a workgroup hands on, in this order, [parts][d] each where they are wanted; the gate's are the last.
enum Sums : int { S_POST_W, S_POST_B, S_PRE_W, S_PRE_B, S_GATE, S_COUNT };

template <class T, int NT, int C>
__global__ __launch_bounds__(NT) void norm_backward_kernel(const NormArgs a)
{
    __shared__ v2f slots[2 * (NT / 64)];
    RowSum<NT> sum{slots};
    const int t = threadIdx.x, part = blockIdx.x;
    // rows of this part: a piece of one group, or whole groups
    int64_t m, end;
    if (a.group_parts > 1) {
        const int64_t g = part / a.group_parts;
        m = g * a.group + (int64_t)(part % a.group_parts) * a.part_rows;
        end = min(min(m + a.part_rows, (g + 1) * a.group), (int64_t)a.rows);
    } else {
        m = (int64_t)part * a.part_rows;
        end = min(m + a.part_rows, (int64_t)a.rows);
    }
    float sums[S_COUNT][C][8] = {};
    for (; m < end; ++m) {
        const int64_t at = m * a.d;
        float x[C][8] = {}, b[C][8] = {}, g[C][8] = {}, q[C][8] = {};
        if (a.pre) load_row<T, NT, C>(x, a.x, at, t, a.d);
        if (a.b) load_row<T, NT, C>(b, a.b, at, t, a.d);
        if (a.pre) load_row<T, NT, C>(q, a.dn, at, t, a.d);
        if (a.dx_out) load_row<T, NT, C>(g, a.dx_out, at, t, a.d);
        v2f r = {1.f, 1.f};
        if (a.pre || a.post) r = normalise<NT, C>(x, b, a.pre, a.post, t, a.d, a.eps, sum);
        if (a.pre) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sums[S_PRE_W][c][j] += q[c][j] * x[c][j];
                    sums[S_PRE_B][c][j] += q[c][j];
                }
            norm_back<T, NT, C>(q, x, a.pre_w, a.pre, r[0], t, a.d, sum);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) g[c][j] += q[c][j];
        }
        store_row<T, NT, C>(a.dx, at, g, t, a.d);
        if (!a.b) continue;
        float p[C][8];
        if (a.dgate) {
            // c = post(b)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) q[c][j] = b[c][j];
            if (a.post && a.post_w) {
                load_row<T, NT, C>(p, a.post_w, 0, t, a.d);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[c][j] *= p[c][j];
            }
            if (a.post && a.post_b) {
                load_row<T, NT, C>(p, a.post_b, 0, t, a.d);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[c][j] += p[c][j];
            }
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[S_GATE][c][j] += a.scale * g[c][j] * q[c][j];
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) g[c][j] *= a.scale;
        if (a.gate) {
            load_row<T, NT, C>(p, a.gate, m / a.group * a.d, t, a.d);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) g[c][j] *= p[c][j];
        }
        if (a.post) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sums[S_POST_W][c][j] += g[c][j] * b[c][j];
                    sums[S_POST_B][c][j] += g[c][j];
                }
            norm_back<T, NT, C>(g, b, a.post_w, a.post, r[1], t, a.d, sum);
        }
        store_row<T, NT, C>(a.db, at, g, t, a.d);
        if (a.dgate && a.group_parts == 1 && (m + 1 == end || (m + 1) % a.group == 0)) {   // a whole group's
            const int64_t row = m / a.group * a.d;
            if (a.f32_out) store_row<float, NT, C>(a.dgate, row, sums[S_GATE], t, a.d);
            else store_row<T, NT, C>(a.dgate, row, sums[S_GATE], t, a.d);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[S_GATE][c][j] = 0.f;
        }
    }
    void *const want[S_COUNT] = {a.dpost_w, a.dpost_b, a.dpre_w, a.dpre_b, a.group_parts > 1 ? a.dgate : nullptr};
    float *ws = a.ws;
#pragma unroll
    for (int k = 0; k < S_COUNT; ++k)
        if (want[k]) {
            store_row<float, NT, C>(ws, (int64_t)part * a.d, sums[k], t, a.d);
            ws += (int64_t)a.parts * a.d;
        }
}

// Column sums of the workgroups' parts, in order.  A workgroup takes 32 columns of one set of parts, eight threads a column;
// blockIdx.y: a parameter, then the gate's groups.
template <class T>
__global__ __launch_bounds__(256) void norm_join_kernel(const NormArgs a)
{
    __shared__ float share[8][32];
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
        for (int p = from + lane; p < to; p += 8) s += a.ws[((int64_t)set * a.parts + p) * a.d + n];
    share[lane][threadIdx.x & 31] = s;
    __syncthreads();
    if (lane || n >= a.d) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) s += share[k][threadIdx.x & 31];
    const int64_t at = which == S_GATE ? (int64_t)y * a.d + n : n;
    if (a.f32_out) static_cast<float *>(want[which])[at] = s;
    else static_cast<T *>(want[which])[at] = (T)s;
}

template <class T, int NT, int C>
hipError_t forward(const NormArgs &a, hipStream_t s)
{
    constexpr int block = NT < 256 ? 256 : NT, rows = NT < 256 ? 256 / NT : 1;
    const int64_t need = ((int64_t)a.rows + rows - 1) / rows, most = 256 * (2048 / block);
    launch_kernel(norm_forward_kernel<T, NT, C>, dim3((unsigned)(need < most ? need : most)), dim3(block), 0, s, a);
    return hipGetLastError();
}

template <class T, int NT, int C>
hipError_t backward(const NormArgs &a, hipStream_t s)
{
    launch_kernel(norm_backward_kernel<T, NT, C>, dim3((unsigned)a.parts), dim3(NT), 0, s, a);
    const hipError_t e = hipGetLastError();
    const bool gates = a.dgate && a.group_parts > 1;
    const int params = (a.dpost_w != nullptr) + (a.dpost_b != nullptr) + (a.dpre_w != nullptr) + (a.dpre_b != nullptr);
    const int groups = gates ? (int)(((int64_t)a.rows + a.group - 1) / a.group) : 0;
    if (e != hipSuccess || params + groups == 0) return e;
    launch_kernel(norm_join_kernel<T>, dim3((unsigned)((a.d + 31) / 32), (unsigned)(params + groups)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <class T>
hipError_t forward_by_width(const NormArgs &a, hipStream_t s)
{
    if (a.d <= 512) return forward<T, 64, 1>(a, s);
    if (a.d <= 2048) return forward<T, 256, 1>(a, s);
    if (a.d <= 4096) return forward<T, 512, 1>(a, s);
    if (a.d <= 8192) return forward<T, 512, 2>(a, s);
    return forward<T, 1024, 2>(a, s);
}
template <class T>
hipError_t backward_by_width(const NormArgs &a, hipStream_t s)
{
    if (a.d <= 512) return backward<T, 64, 1>(a, s);
    if (a.d <= 2048) return backward<T, 256, 1>(a, s);
    if (a.d <= 4096) return backward<T, 512, 1>(a, s);
    if (a.d <= 8192) return backward<T, 512, 2>(a, s);
    return backward<T, 1024, 2>(a, s);
}

}  // namespace

size_t norm_backward_plan(NormArgs &a)
{
    // parts: as many as keep the chip full, so many threads a row being taken; more would write and read more partial sums
    const int64_t threads = a.d <= 512 ? 64 : a.d <= 2048 ? 256 : 512, most = 256 * 1024 / threads;
    int64_t part = ((int64_t)a.rows + most - 1) / most;
    if (part < 1) part = 1;
    if (a.group > part) {
        a.group_parts = (int32_t)(((int64_t)a.group + part - 1) / part);
        if (a.group_parts == 1) part = a.group;
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
