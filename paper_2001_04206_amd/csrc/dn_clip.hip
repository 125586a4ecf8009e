// Clipping by the norm of many tensors together.
//
// Two passes over memory: squares, and (where there is something to write) products.  Pieces of all tensors of a launch are numbered on
// end; workgroup b takes pieces b, b + grid, .., so that what is added to what depends on the tensors' sizes alone.  The squares are added
// in 64 bits, which neither overflow nor lose small tensors beside large ones, at two instructions an element.  Bound by memory: 336 tensors of
// 805 million bf16 elements into fp32 ones, 1.35 ms (4.8 TB/s); 14 small ones by the two launches, 3.8 and 3.4 us, and the call, 18.
#include <stdlib.h>

#include <algorithm>

#include "dn_ffn_host.h"

namespace dn {
namespace {

constexpr int kSpans = 80;            // of a launch: its arguments stay within 4 KB
constexpr int kPiece = 256 * 8 * 4;   // elements
constexpr int kGroups = 1024;         // workgroups of a launch, four a compute unit

struct ClipArgs {
    struct Span { const void *g; void *y; int64_t n; int32_t first; int16_t type, out_type; } s[kSpans];   // first: its first piece
    double *parts;         // this launch's (squares); all of them, or their sum (products)
    float *norm;           // written by one workgroup, NULL: not by this launch
    int32_t n, pieces, all_parts;
    float max_norm;
};
static_assert(sizeof(ClipArgs) <= 4096, "a launch's arguments");

__device__ __forceinline__ double sum_of_block(double v, double *share)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) share[threadIdx.x >> 6] = v;
    __syncthreads();
    return (share[0] + share[1]) + (share[2] + share[3]);
}

__device__ __forceinline__ int span_of(const ClipArgs &a, int piece)
{
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.s[mid].first <= piece) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <class T>
__device__ __forceinline__ double squares(const void *g, int64_t at, int64_t n)
{
    double s[4] = {};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int64_t i = at + q * 2048 + threadIdx.x * 8;
        float v[8];
        load8<T>(v, g, i, (int)(n - i < 8 ? n - i : 8));
#pragma unroll
        for (int j = 0; j < 8; ++j) s[q] = fma((double)v[j], (double)v[j], s[q]);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

__global__ __launch_bounds__(256) void squares_kernel(const ClipArgs a)
{
    __shared__ double share[4];
    double sum = 0.;
    for (int p = blockIdx.x; p < a.pieces; p += gridDim.x) {
        const ClipArgs::Span &s = a.s[span_of(a, p)];
        const int64_t at = (int64_t)(p - s.first) * kPiece;
        sum += s.type == DN_F32 ? squares<float>(s.g, at, s.n) : s.type == DN_F16 ? squares<f16>(s.g, at, s.n) : squares<bf16>(s.g, at, s.n);
    }
    sum = sum_of_block(sum, share);
    if (threadIdx.x == 0) a.parts[blockIdx.x] = sum;
}

// The sum of many launches' parts, formed once, in the order in which the workgroups of a single launch form it.  Where every workgroup of every
// launch does, that grows with the square of the number of tensors: 8000 of 100 000 bf16 elements into fp32 take 12.6 ms so, 6.0 with this (the call, 0.75 us
// a tensor), 336 of 2.4 million 1.39 and 1.36.
__global__ __launch_bounds__(256) void total_kernel(const double *parts, int n, double *total, float *norm)
{
    __shared__ double share[4];
    double sum = 0.;
    for (int i = threadIdx.x; i < n; i += 256 * 16) {
        double v[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) v[q] = i + q * 256 < n ? parts[i + q * 256] : 0.;
#pragma unroll
        for (int q = 0; q < 16; ++q) sum += v[q];
    }
    sum = sum_of_block(sum, share);
    if (threadIdx.x) return;
    *total = sum;
    *norm = (float)sqrt(sum);
}

template <class T, class U>
__device__ __forceinline__ void times(const ClipArgs::Span &s, int64_t at, float by, double small)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int64_t i = at + q * 2048 + threadIdx.x * 8;
        const int left = (int)(s.n - i < 8 ? s.n - i : 8);
        float v[8];
        load8<T>(v, s.g, i, left);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = small != 0. ? (float)((double)v[j] * small) : v[j] * by;
        store8<U>(s.y, i, v, left);
    }
}

__global__ __launch_bounds__(256) void times_kernel(const ClipArgs a)
{
    __shared__ double share[4];
    double sum = 0.;
    for (int i = threadIdx.x; i < a.all_parts; i += 256) sum += a.parts[i];
    const double norm = sqrt(sum_of_block(sum, share));
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    const bool clip = norm > (double)a.max_norm && norm < (double)INFINITY;
    // Below the normal numbers of fp32 a factor would have few bits or none where results do not (gradients near 1e38, max_norm 1e-3): there
    // products are formed in 64 bits.
    const double ratio = clip ? (double)a.max_norm / norm : 1., small = ratio < 0x1p-126 ? ratio : 0.;
    const float by = (float)ratio;
    for (int p = a.pieces - 1 - (int)blockIdx.x; p >= 0; p -= gridDim.x) {   // what was read last may still be near
        const ClipArgs::Span &s = a.s[span_of(a, p)];
        if (!s.y || (!clip && s.y == s.g)) continue;
        const int64_t at = (int64_t)(p - s.first) * kPiece;
        if (s.type == DN_F32) times<float, float>(s, at, by, small);
        else if (s.type == DN_F16) s.out_type == DN_F32 ? times<f16, float>(s, at, by, small) : times<f16, f16>(s, at, by, small);
        else s.out_type == DN_F32 ? times<bf16, float>(s, at, by, small) : times<bf16, bf16>(s, at, by, small);
    }
}

int groups_of(int64_t pieces) { return pieces < 1 ? 1 : pieces < kGroups ? (int)pieces : kGroups; }

// Spans in runs of a launch each: at most kSpans, and pieces that 31 bits can number.  f(args, pieces, run): false ends it.
template <class F>
bool runs(const dn_span *spans, int32_t n, F f)
{
    ClipArgs a{};
    int64_t pieces = 0;
    int run = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (!spans[i].count) continue;
        const int64_t more = (spans[i].count + kPiece - 1) / kPiece;
        if (a.n == kSpans || (a.n && pieces + more > 0x7fffffff)) {
            a.pieces = (int32_t)pieces;
            if (!f(a, run++)) return false;
            a.n = 0;
            pieces = 0;
        }
        a.s[a.n++] = {spans[i].grad_dev, spans[i].out_dev, spans[i].count, (int32_t)pieces, (int16_t)spans[i].type, (int16_t)spans[i].out_type};
        pieces += more;
    }
    a.pieces = (int32_t)pieces;
    return f(a, run);   // the last one, if only to write the norm
}

dn_status check(const dn_span *spans, int32_t n)
{
    if (n < 0 || (n && !spans)) return DN_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n; ++i) {
        const dn_span &s = spans[i];
        if (!type_ok(s.type) || (s.out_type != s.type && s.out_type != DN_F32)) return DN_ERR_INVALID_ARG;
        if (s.count < 0 || s.count > (int64_t)1 << 43) return DN_ERR_SHAPE;   // 2^31 pieces and fewer
        if (!s.count) continue;
        if (!s.grad_dev || !multiples(s.type, s.grad_dev) || !multiples(s.out_type, s.out_dev)) return DN_ERR_INVALID_ARG;
    }
    return DN_OK;
}

// No result (nor the norm) may lie where another tensor's gradient or result does: two workgroups would write there, or one read what the
// other wrote.
dn_status apart(const dn_span *spans, int32_t n, const float *norm)
{
    struct Range { uintptr_t from, to; bool written; };
    Range *r = static_cast<Range *>(malloc(sizeof(Range) * (2 * (size_t)n + 1)));
    if (!r) return DN_ERR_OOM;
    int64_t m = 0;
    bool sorted = true;
    auto add = [&](const void *p, int64_t bytes, bool written) {
        r[m] = {(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written};
        sorted = sorted && (!m || r[m - 1].from <= r[m].from);
        ++m;
    };
    for (int32_t i = 0; i < n; ++i)
        if (spans[i].count) {
            const bool same = spans[i].out_dev == spans[i].grad_dev && spans[i].out_type == spans[i].type;
            add(spans[i].grad_dev, spans[i].count * size_of(spans[i].type), same);
            if (spans[i].out_dev && !same) add(spans[i].out_dev, spans[i].count * size_of(spans[i].out_type), true);
        }
    add(norm, sizeof(float), true);
    if (!sorted) std::sort(r, r + m, [](const Range &x, const Range &y) { return x.from < y.from; });
    // the furthest end so far of what is read, and of what is written
    uintptr_t read = 0, written = 0;
    dn_status s = DN_OK;
    for (int64_t i = 0; i < m; ++i) {
        if (r[i].from < written || (r[i].written && r[i].from < read)) s = DN_ERR_INVALID_ARG;
        uintptr_t &end = r[i].written ? written : read;
        end = end > r[i].to ? end : r[i].to;
    }
    free(r);
    return s;
}

struct Parts {
    size_t n = 0;       // of all launches
    bool many = false;  // launches
    size_t bytes() const { return up256((n + many) * sizeof(double)); }   // their sum behind them
};
Parts parts_of(const dn_span *spans, int32_t n)
{
    Parts p;
    runs(spans, n, [&](const ClipArgs &a, int run) {
        p.n += (size_t)groups_of(a.pieces);
        p.many = run > 0;
        return true;
    });
    return p;
}

}  // namespace
}  // namespace dn

using namespace dn;

extern "C" {

size_t dn_clip_workspace_bytes(const dn_span *spans, int32_t n_spans)
{
    return check(spans, n_spans) == DN_OK ? parts_of(spans, n_spans).bytes() : kBad;
}

dn_status dn_clip(const dn_span *spans, int32_t n_spans, float max_norm, float *norm_dev, void *workspace_dev,
                  size_t workspace_bytes, void *hip_stream)
{
    dn_status st = check(spans, n_spans);
    if (st != DN_OK) return st;
    if (!(max_norm >= 0.f) || !norm_dev || !multiples(DN_F32, norm_dev)) return DN_ERR_INVALID_ARG;
    if ((st = apart(spans, n_spans, norm_dev)) != DN_OK) return st;
    const Parts parts = parts_of(spans, n_spans);
    if ((st = workspace(parts.bytes(), workspace_dev, workspace_bytes)) != DN_OK) return st;
    const hipStream_t s = (hipStream_t)hip_stream;
    double *ws = static_cast<double *>(workspace_dev), *at = ws;
    const bool summed = runs(spans, n_spans, [&](ClipArgs &a, int) {
        a.parts = at;
        at += groups_of(a.pieces);
        launch_kernel(squares_kernel, dim3(groups_of(a.pieces)), dim3(256), 0, s, a);
        return hipGetLastError() == hipSuccess;
    });
    if (!summed) return DN_ERR_DEVICE;
    if (parts.many) {
        launch_kernel(total_kernel, dim3(1), dim3(256), 0, s, (const double *)ws, (int)parts.n, at, norm_dev);
        if (hipGetLastError() != hipSuccess) return DN_ERR_DEVICE;
    }
    const bool done = runs(spans, n_spans, [&](ClipArgs &a, int) {
        bool any = !parts.many;   // to write the norm
        for (int i = 0; i < a.n; ++i) any = any || a.s[i].y;
        if (!any) return true;
        a.parts = parts.many ? at : ws;
        a.all_parts = parts.many ? 1 : (int32_t)parts.n;
        a.norm = parts.many ? nullptr : norm_dev;
        a.max_norm = max_norm;
        launch_kernel(times_kernel, dim3(groups_of(a.pieces)), dim3(256), 0, s, a);
        return hipGetLastError() == hipSuccess;
    });
    return done ? DN_OK : DN_ERR_DEVICE;
}

}  // extern "C"
