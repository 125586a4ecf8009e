// A block of experts: checks, plans, workspaces and launches, and what follows its products: the pairs' results back together.
#include "dn_experts.h"
#include "dn_ffn_host.h"

namespace dn {
namespace {

// Up to so many tokens the last product forms the sums itself.  Forward pass so, and with a launch for the sums, in us, one token: 22.2 and 27.5 (8 of
// 64 experts, 2048 wide, 1024 hidden, bf16), 13.8 and 17.0 (2 of 8, 512, 1024), 13.7 and 16.9 (2 of 16, 1021, 555, f16), 13.7 and 17.9 (4 of
// 128, 1024, 512, fp32), 25.7 and 28.2 (2 of 8, 2048, 4096); four tokens: 68.3 and 73.8, 13.8 and 17.1, 13.7 and 18.1, 24.4 and 29.2, 65.0 and 63.5; eight:
// 107.9 and 104.4, 13.8 and 17.1, 19.3 and 21.5, 40.8 and 46.2, 87.3 and 75.1, as an expert that several rows share is read by each.
constexpr int kFewTokens = 4, kMostExperts = 1024, kMostChoices = 32;
constexpr int64_t kMostRows = (int64_t)1 << 25, kMostPairs = (int64_t)1 << 24, kMostBytes = ((int64_t)1 << 31) - 1;

// ---- rows ------------------------------------------------------------------------------------------------------------

// Y_t = R_t + the sum over its pairs of (weight) z, in the order of the choices.  A thread: eight columns of a row.  z is fp32, or for results of
// 16 bits (and k in one part) in 24, so that what is rounded is the sum: with z in 16 bits each would be rounded by itself, and results
// without a residual be off by 0.0029 where they are by 0.0024 (bf16; of which H has a rounding, and the result).  Bound by memory: 65536 pairs'
// rows of 2048 into 8192, 92 us (5.1 TB/s; of fp32 118).
struct JoinArgs {
    const void *z, *low;       // low: the low bytes of 24 bits, NULL: fp32
    const void *r;
    void *y;
    int64_t ldz, ldr, ldy;
    const float *weight;       // NULL: ones
    const int32_t *place;
    int32_t rows, cols, k, pairs, parts;
    int64_t plane;             // elements between two parts of z
};
// The weights' derivatives from the parts that the tiles of dh left, one for 64 columns, in order.  In one launch with
// the sums of dX: a backward pass of 64 rows, 2 of 8 experts, 512 wide with 1024 hidden, bf16, took 50 us in two, 45 so.
struct DotArgs {
    const float *dots;
    int32_t parts;
    Group group;
    const int32_t *place;
    float *dweight;
};
__device__ __forceinline__ void join_dots(const DotArgs &a, int i)
{
    if (i < a.group.starts[a.group.experts]) {
        float v = 0.f;
#pragma unroll 4
        for (int s = 0; s < a.parts; ++s) v += a.dots[(int64_t)s * a.group.pairs + i];
        const int q = a.group.order[i];
        if ((uint32_t)q < (uint32_t)a.group.pairs) a.dweight[q] = v;
    }
    if (a.place[i] < 0) a.dweight[i] = 0.f;
}
__global__ __launch_bounds__(256) void dots_kernel(const DotArgs a)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < a.group.pairs) join_dots(a, i);
}

// DOTS: the first threads, one a pair, join the weights' derivatives too
template <class T, bool SHORT, bool DOTS>
__global__ __launch_bounds__(256) void join_pairs_kernel(const JoinArgs a, const DotArgs dots)
{
    if (DOTS) {
        const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
        if (i < dots.group.pairs) join_dots(dots, (int)i);
    }
    const uint32_t eights = ((uint32_t)a.cols + 7) / 8;
    const uint64_t first = (uint64_t)blockIdx.x * 256;
    const uint32_t row0 = (uint32_t)(first / eights), c0 = (uint32_t)(first % eights) + threadIdx.x, more = c0 / eights;
    const int64_t t = (int64_t)row0 + more;
    if (t >= a.rows) return;
    const int n = (int)(c0 - more * eights) * 8, left = a.cols - n;
    float v[8] = {};
    if (a.r) load8<T>(v, a.r, t * a.ldr + n, left);
    for (int j0 = 0; j0 < a.k; j0 += 4) {
        float z[4][8], w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int j = min(j0 + q, a.k - 1), p = a.place[t * a.k + j];
            const bool has = j0 + q < a.k && (uint32_t)p < (uint32_t)a.pairs;
            w[q] = !has ? 0.f : a.weight ? a.weight[t * a.k + j] : 1.f;
            if constexpr (SHORT) {
                load24(z[q], a.z, a.low, has ? p * a.ldz + n : n);   // (any pair's row: its weight is 0)
                if (!has)
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[q][i] = 0.f;
                continue;
            }
            load8<float>(z[q], a.z, has ? p * a.ldz + n : 0, has ? left : 0);
            for (int s = 1; s < a.parts; ++s) {
                float more[8];
                load8<float>(more, a.z, has ? s * a.plane + p * a.ldz + n : 0, has ? left : 0);
#pragma unroll
                for (int i = 0; i < 8; ++i) z[q][i] += more[i];
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = fmaf(w[q], z[q][j], v[j]);
    }
    store8<T>(a.y, t * a.ldy + n, v, left);
}

template <class T, bool SHORT>
hipError_t join_as(const JoinArgs &a, const DotArgs &dots, hipStream_t s)
{
    uint64_t threads = (uint64_t)a.rows * (((uint32_t)a.cols + 7) / 8);
    if (dots.dweight && threads < (uint64_t)a.pairs) threads = (uint64_t)a.pairs;
    const dim3 grid((unsigned)((threads + 255) / 256)), block(256);
    if (dots.dweight) launch_kernel(join_pairs_kernel<T, SHORT, true>, grid, block, 0, s, a, dots);
    else launch_kernel(join_pairs_kernel<T, SHORT, false>, grid, block, 0, s, a, dots);
    return hipGetLastError();
}
hipError_t launch_join(int type, const JoinArgs &a, hipStream_t s, const DotArgs &dots = {})
{
    if (type == DN_F32) return join_as<float, false>(a, dots, s);
    if (type == DN_F16) return a.low ? join_as<f16, true>(a, dots, s) : join_as<f16, false>(a, dots, s);
    return a.low ? join_as<bf16, true>(a, dots, s) : join_as<bf16, false>(a, dots, s);
}
hipError_t launch_experts(int type, Product p, Epilogue e, ProductKernel kernel, const ProductArgs &a, int64_t tiles, hipStream_t s, int gathered = 0)
{
    return type == DN_F32   ? launch_experts_f32(p, e, kernel, gathered, a, tiles, s)
           : type == DN_F16 ? launch_experts_f16(p, e, kernel, gathered, a, tiles, s)
                            : launch_experts_bf16(p, e, kernel, gathered, a, tiles, s);
}

// ---- plans -----------------------------------------------------------------------------------------------------------

// Tiles of rows: at most, whatever the lists hold.
int64_t most_tiles(int64_t pairs, int experts, int rows) { return pairs / rows + (pairs < experts ? pairs : experts); }

// Which kernel a product of the experts takes, and its k in how many parts: what is expected to take least, by the times that plan_product
// goes by.  How the pairs are spread is not known here: each expert's last tile is taken to be half full.  Weights come at 4.6 TB/s (large
// tiles: 3.8; the kernel for few rows: 5): 64 tokens through 8 of 64 experts, 2048 wide with 1024 hidden, take 108 us for the gated product
// on the kernel for few rows (large tiles 141); a whole forward pass of 1024 tokens 234 on medium tiles (large ones 281, small ones 243), of 128
// 190 (all on the kernel for few rows 242).  The product with the activation's derivative moves ten bytes an element beside it, and large
// tiles have no registers for that: 409 us on medium ones at 8192 tokens, 442 on large ones.  Parts are for the products whose results the pairs' sums read: these add them too.
struct Plan { ProductKernel kernel = K_SMALL; int parts = 1; };
Plan plan_experts(int type, Product p, Epilogue e, int64_t pairs, int experts, int N, int K, int segments, bool few_tokens = false)
{
    const int planes = e == E_GATED ? 2 : 1, bk = type == DN_F32 ? 32 : 64;
    const double es = (double)size_of(type), met = (double)(pairs < experts ? pairs : experts);
    const bool packed = p == P_FWD && (N * size_of(type) % 16 || K * size_of(type) % 16);   // tiles copy the matrices first
    const double weights = p == P_GRAD ? 0 : es * met * planes * N * K * segments / 4.6e6;
    double best = 1e300;
    Plan plan;
    auto tiles_of = [&](int rows) {
        const double t = (double)pairs / rows + met / 2;
        return t > met ? t : met;
    };
    if (p == P_FWD && (int64_t)K * size_of(type) >= 32 && most_tiles(pairs, experts, 16) * ((N + 15) / 16) < 1 << 23) {   // 2^32 threads
        best = 6 + es * tiles_of(16) * planes * N * K / 5e6;
        plan.kernel = K_FEW;
        if (few_tokens) return plan;
    }
    struct Way { ProductKernel kernel; int rows, cols, together; double stage, least, round, behind; };
    const Way tiny{K_TINY, 64, 128, 3, 0.9, 0.9, 3, 1}, large{K_LARGE, 256, 256, 1, 1.5, 1.5, 8, 4.6 / 3.8}, medium{K_MEDIUM, 128, 256, 1, 0.8, 0.8, 6, 1};
    const Way small = type == DN_F32 ? Way{K_SMALL, 128, 128, 2, 1.8, 1.8, 6, 1} : Way{K_SMALL, 128, 128, 2, 0.5, 0.9, 4, 1};
    for (const Way &w : {large, medium, small, tiny}) {
        if (type == DN_F32 ? w.kernel > K_SMALL : w.kernel == K_TINY) continue;
        if (w.kernel == K_LARGE && e == E_DEXPERT) continue;
        const int64_t cols = w.cols / planes;
        double tiles = (double)((N + cols - 1) / cols), steps;
        if (p == P_GRAD) {   // K: the result's rows; its terms are the pairs
            tiles *= (double)experts * ((K + w.rows - 1) / w.rows);
            steps = (double)pairs / met / bk + 0.5;
        } else {
            tiles *= tiles_of(w.rows);
            steps = (double)((K + bk - 1) / bk * segments);
        }
        for (int parts = 1; parts <= (e == E_STORE && p != P_GRAD ? 4 : 1) && parts * 4 <= steps; ++parts) {
            const double deep = ceil(tiles * parts / 256), rounds = ceil(deep / w.together);
            const double stage = deep * w.stage > rounds * w.least ? deep * w.stage : rounds * w.least;
            double us = ceil(steps / parts) * stage + rounds * w.round;
            if (us < weights * w.behind + 6) us = weights * w.behind + 6;
            us += (parts > 1 ? 3 : 0) + (parts - 1) * 8. * pairs * N / 4.5e6 + (packed ? 4 + 2 * es * experts * planes * N * K / 4.6e6 : 0);
            if (us < best) {
                best = us;
                plan = {w.kernel, parts};
            }
        }
    }
    return plan;
}

struct Block {
    dn_experts_desc d;
    int64_t pairs, ldh, ldz;     // between rows of H, of z
    Plan up, down, dh, dx, dwgu, dwd;
    bool short_z, short_dx;      // pairs' results in 24 bits
    bool few;                    // the last product forms the sums over choices itself
    bool pack_w;                 // the matrices are copied to 16-byte rows
    int parts;                   // of the weights' derivatives
    size_t h, z, x, w1, w2, fwd_bytes;                        // bytes of H, z, X, Wg (and Wu), Wd; workspace
    size_t dots, dgu, dx_parts, bwd_bytes;            // the pairs' dX
};

dn_status block_of(const dn_experts_desc *d, Block &b)
{
    if (!d) return DN_ERR_INVALID_ARG;
    b.d = *d;
    dn_status s = common(d->type, d->grad_type, d->act, d->rows, d->d, d->f, d->grad_scale);
    if (s != DN_OK) return s;
    if (d->experts < 1 || d->experts > kMostExperts || d->k < 1 || d->k > kMostChoices || d->rows >= kMostRows) return DN_ERR_SHAPE;
    if ((s = row_length(d->type, b.d.ldx, d->d)) != DN_OK || (s = row_length(d->type, b.d.ldr, d->d)) != DN_OK ||
        (s = row_length(d->type, b.d.ldy, d->d)) != DN_OK)
        return s;
    const int64_t e = size_of(d->type), n = d->experts;
    b.pairs = (int64_t)d->rows * d->k;
    b.ldh = up8(d->f);
    b.ldz = up8(d->d);
    if (b.pairs >= kMostPairs || 2 * b.ldh * e > kRowBytes || n * b.ldh >= kMostBytes || n * b.ldz >= kMostBytes) return DN_ERR_SHAPE;
    if (most_tiles(b.pairs, d->experts, 64) * (((b.ldh > b.ldz ? b.ldh : b.ldz) + 63) / 64) >= 1 << 23) return DN_ERR_SHAPE;   // a launch's threads
    if (too_many(b.pairs, d->d) || too_many(b.pairs, 2 * b.ldh) || too_many(n * d->f, d->d) || too_many(n * d->d, d->f)) return DN_ERR_SHAPE;
    const int64_t wide = b.d.ldx > b.ldz ? b.d.ldx : b.ldz, wider = b.d.ldy > wide ? b.d.ldy : wide;
    if (d->rows * wider * e > kMostBytes) return DN_ERR_SHAPE;
    b.up = plan_experts(d->type, P_FWD, E_GATED, b.pairs, d->experts, d->f, d->d, 1, d->rows <= kFewTokens);
    b.down = plan_experts(d->type, P_FWD, E_STORE, b.pairs, d->experts, d->d, d->f, 1, d->rows <= kFewTokens);
    b.dh = plan_experts(d->type, P_DELTA, E_DEXPERT, b.pairs, d->experts, d->f, d->d, 1);
    b.dx = plan_experts(d->type, P_DELTA, E_STORE, b.pairs, d->experts, d->d, d->f, 2);
    b.dwgu = plan_experts(d->type, P_GRAD, E_STORE, b.pairs, d->experts, d->d, (int)(2 * b.ldh), 1);
    b.dwd = plan_experts(d->type, P_GRAD, E_STORE, b.pairs, d->experts, d->f, d->d, 1);
    b.short_z = e == 2 && b.down.parts == 1 && b.down.kernel != K_FEW;
    b.short_dx = e == 2 && b.dx.parts == 1;
    b.few = b.down.kernel == K_FEW && d->rows <= kFewTokens;
    b.pack_w = d->d * e % 16 || d->f * e % 16;
    const size_t wgu = b.pack_w ? packed_bytes(d->type, n * d->f, d->d) : 0, wd = b.pack_w ? packed_bytes(d->type, n * d->d, d->f) : 0;
    b.h = up256((size_t)(b.pairs * b.ldh * e));
    b.z = up256((size_t)(b.pairs * b.ldz * b.down.parts) * sizeof(float));
    b.dx_parts = up256((size_t)(b.pairs * b.ldz * b.dx.parts) * sizeof(float));
    b.x = packed_bytes(d->type, d->rows, d->d);
    b.w1 = wgu;
    b.w2 = wd;
    b.fwd_bytes = b.h + b.z + (b.up.kernel == K_FEW ? 0 : b.x + 2 * wgu) + (b.down.kernel == K_FEW ? 0 : wd);
    b.parts = (int)((d->f + 255) / 256 * 4);   // of 64 columns, whole tiles
    b.dots = up256((size_t)b.pairs * b.parts * sizeof(float));
    b.dgu = up256((size_t)(b.pairs * 2 * b.ldh * e));
    b.bwd_bytes = b.dots + b.h + b.dgu + b.dx_parts + 2 * b.x + 2 * wgu + wd;
    return DN_OK;
}

ProductArgs product(const Group &g, int M, int N, int K, int segments, int64_t b_stride)
{
    ProductArgs a{};
    a.M = M;
    a.N = N;
    a.K = K;
    a.segments = segments;
    a.split = 1;
    a.group = g;
    a.group.b_stride = b_stride;
    return a;
}

}  // namespace

int rows_of_tile(ProductKernel kernel) { return kernel == K_FEW ? 16 : kernel == K_TINY ? 64 : kernel == K_LARGE ? 256 : 128; }

}  // namespace dn

using namespace dn;

extern "C" {

size_t dn_experts_forward_workspace_bytes(const dn_experts_desc *d)
{
    Block b;
    return block_of(d, b) == DN_OK ? b.fwd_bytes : kBad;
}

size_t dn_experts_backward_workspace_bytes(const dn_experts_desc *d)
{
    Block b;
    return block_of(d, b) == DN_OK ? b.bwd_bytes : kBad;
}

dn_status dn_experts_forward(const dn_experts_desc *d, const void *X_dev, const void *Wg_dev, const void *Wu_dev, const void *Wd_dev,
                             const float *weight_dev, const int32_t *starts_dev, const int32_t *order_dev, const int32_t *place_dev,
                             const void *R_dev, void *Y_dev, void *GU_dev, void *workspace_dev, size_t workspace_bytes,
                             void *hip_stream)
{
    Block b;
    dn_status s = block_of(d, b);
    if (s != DN_OK) return s;
    if (!X_dev || !Wg_dev || !Wu_dev || !Wd_dev || !weight_dev || !starts_dev || !order_dev || !place_dev || !Y_dev) return DN_ERR_INVALID_ARG;
    if (!multiples(d->type, X_dev, Wg_dev, Wu_dev, Wd_dev, R_dev, Y_dev, GU_dev) || !multiples(DN_F32, weight_dev, starts_dev, order_dev, place_dev))
        return DN_ERR_INVALID_ARG;
    if (!b.pack_w && ((uintptr_t)Wg_dev | (uintptr_t)Wu_dev | (uintptr_t)Wd_dev) % 16) return DN_ERR_INVALID_ARG;
    if ((s = workspace(b.fwd_bytes, workspace_dev, workspace_bytes)) != DN_OK) return s;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t e = size_of(d->type), n = d->experts, f = d->f;
    char *H = static_cast<char *>(workspace_dev), *z = H + b.h;
    const Group g{starts_dev, order_dev, d->experts, d->k, (int32_t)b.pairs, d->rows, 0, 0};
    ProductArgs a = product(g, 0, d->f, d->d, 1, 0), c = product(g, 0, d->d, d->f, 1, 0);
    Packer pack{d->type, z + b.z};
    if (b.up.kernel == K_FEW) {
        operand_a(a, {X_dev, b.d.ldx * e, d->d});
        operand_b(a, {Wg_dev, d->d * e, d->d});
        a.b[1] = Wu_dev;
    } else {
        operand_a(a, pack.take(X_dev, b.d.ldx, d->rows, d->d));
        operand_b(a, pack.take(Wg_dev, d->d, n * d->f, d->d, b.pack_w));
        a.b[1] = pack.take(Wu_dev, d->d, n * d->f, d->d, b.pack_w).p;
    }
    if (b.down.kernel == K_FEW) operand_b(c, {Wd_dev, d->f * e, d->f});
    else operand_b(c, pack.take(Wd_dev, d->f, n * d->d, d->f, b.pack_w));
    if (pack.run(stream) != hipSuccess) return DN_ERR_DEVICE;
    a.group.b_stride = a.ldb * d->f;
    a.f.y = H;
    a.f.ldy = b.ldh;
    a.f.zeros = (int)(b.ldh - d->f);
    a.f.y2 = GU_dev;
    a.f.ldy2 = 2 * (int64_t)d->f;
    a.f.half = d->f;
    a.f.act = d->act;
    auto tiles = [&](const Plan &p) { return most_tiles(b.pairs, d->experts, rows_of_tile(p.kernel)); };
    if (launch_experts(d->type, P_FWD, E_GATED, b.up.kernel, a, tiles(b.up), stream) != hipSuccess) return DN_ERR_DEVICE;
    operand_a(c, {H, b.ldh * e, (int32_t)b.ldh});
    c.group.b_stride = c.ldb * d->d;
    if (b.few) {
        const FewDown few{H, Wd_dev, R_dev, Y_dev, weight_dev, starts_dev, place_dev, b.ldh * e, f * e, f * e * d->d, b.d.ldr, b.d.ldy,
                          d->d, d->f, d->k, d->experts, (int32_t)b.pairs};
        return device(d->type == DN_F32   ? launch_few_down_f32(few, d->rows, stream)
                      : d->type == DN_F16 ? launch_few_down_f16(few, d->rows, stream)
                                          : launch_few_down_bf16(few, d->rows, stream));
    }
    c.f.y = z;
    c.f.ldy = b.ldz;
    c.f.f32_out = 1;
    char *low = b.short_z ? z + (size_t)(b.pairs * b.ldz) * 2 : nullptr;
    c.f.y2 = low;
    c.split = b.down.parts;
    c.group.c_stride = b.pairs * b.ldz * (int64_t)sizeof(float);
    if (launch_experts(d->type, P_FWD, low ? E_PAIR : E_STORE, b.down.kernel, c, tiles(b.down), stream) != hipSuccess) return DN_ERR_DEVICE;
    return device(launch_join(d->type, {z, low, R_dev, Y_dev, b.ldz, b.d.ldr, b.d.ldy, weight_dev, place_dev, d->rows, d->d, d->k, (int32_t)b.pairs, b.down.parts, b.pairs * b.ldz}, stream));
}

dn_status dn_experts_backward(const dn_experts_desc *d, const void *X_dev, const void *Wg_dev, const void *Wu_dev, const void *Wd_dev,
                              const float *weight_dev, const int32_t *starts_dev, const int32_t *order_dev, const int32_t *place_dev,
                              const void *GU_dev, const void *dY_dev, void *dX_dev, void *dWg_dev, void *dWu_dev, void *dWd_dev,
                              float *dweight_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    Block b;
    dn_status s = block_of(d, b);
    if (s != DN_OK) return s;
    if (!X_dev || !Wg_dev || !Wu_dev || !Wd_dev || !weight_dev || !starts_dev || !order_dev || !place_dev || !GU_dev || !dY_dev || !dWg_dev ||
        !dWu_dev || !dWd_dev)
        return DN_ERR_INVALID_ARG;
    if (!multiples(d->type, X_dev, Wg_dev, Wu_dev, Wd_dev, GU_dev, dY_dev, dX_dev) || !multiples(d->grad_type, dWg_dev, dWu_dev, dWd_dev) ||
        !multiples(DN_F32, weight_dev, starts_dev, order_dev, place_dev, dweight_dev))
        return DN_ERR_INVALID_ARG;
    if (!b.pack_w && ((uintptr_t)Wg_dev | (uintptr_t)Wu_dev | (uintptr_t)Wd_dev) % 16) return DN_ERR_INVALID_ARG;
    if ((s = workspace(b.bwd_bytes, workspace_dev, workspace_bytes)) != DN_OK) return s;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t e = size_of(d->type), n = d->experts, f = d->f;
    char *dots = static_cast<char *>(workspace_dev), *H = dots + b.dots;
    char *dG = H + b.h, *dU = dG + b.ldh * e, *dx = dG + b.dgu;
    const Group g{starts_dev, order_dev, d->experts, d->k, (int32_t)b.pairs, d->rows, 0, 0};
    Packer pack{d->type, dx + b.dx_parts};
    const Packer::Rows X = pack.take(X_dev, b.d.ldx, d->rows, d->d), dY = pack.take(dY_dev, b.d.ldy, d->rows, d->d);
    const Packer::Rows Wd = pack.take(Wd_dev, f, n * d->d, f, b.pack_w);
    const Packer::Rows Wg = dX_dev ? pack.take(Wg_dev, d->d, n * f, d->d, b.pack_w) : Packer::Rows{};
    const Packer::Rows Wu = dX_dev ? pack.take(Wu_dev, d->d, n * f, d->d, b.pack_w) : Packer::Rows{};
    if (pack.run(stream) != hipSuccess) return DN_ERR_DEVICE;
    auto tiles = [&](const Plan &p) { return most_tiles(b.pairs, d->experts, rows_of_tile(p.kernel)); };
    {   // dh, and from it dG, dU, w H and the weights' derivatives
        ProductArgs a = product(g, 0, d->f, d->d, 1, Wd.ld * d->d);
        operand_a(a, dY);
        operand_b(a, Wd);
        a.f.y = dG;
        a.f.ldy = 2 * b.ldh;
        a.f.half_y = b.ldh;
        a.f.zeros = (int)(b.ldh - f);
        a.f.y2 = H;
        a.f.ldy2 = b.ldh;
        a.f.r = GU_dev;
        a.f.ldr = 2 * f;
        a.f.half = f;
        a.f.act = d->act;
        a.f.weight = weight_dev;
        a.f.order = order_dev;
        a.f.pairs = (uint32_t)b.pairs;
        a.f.dots = reinterpret_cast<float *>(dots);
        a.f.dots_ld = b.pairs;
        if (launch_experts(d->type, P_DELTA, E_DEXPERT, b.dh.kernel, a, tiles(b.dh), stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    DotArgs joined{};
    if (dweight_dev) {
        const int cols = b.dh.kernel == K_SMALL || b.dh.kernel == K_TINY ? 128 : 256, parts = (int)((f + cols - 1) / cols * (cols / 64));
        joined = {reinterpret_cast<const float *>(dots), parts, g, place_dev, dweight_dev};
        if (!dX_dev) {
            launch_kernel(dots_kernel, dim3((unsigned)((b.pairs + 255) / 256)), dim3(256), 0, stream, joined);
            if (hipGetLastError() != hipSuccess) return DN_ERR_DEVICE;
        }
    }
    if (dX_dev) {
        ProductArgs a = product(g, 0, d->d, d->f, 2, Wg.ld * f);
        operand_a(a, {dG, 2 * b.ldh * e, (int32_t)b.ldh});
        a.a[1] = dU;
        operand_b(a, Wg);
        a.b[1] = Wu.p;
        a.f.y = dx;
        a.f.ldy = b.ldz;
        a.f.f32_out = 1;
        char *low = b.short_dx ? dx + (size_t)(b.pairs * b.ldz) * 2 : nullptr;
        a.f.y2 = low;
        a.split = b.dx.parts;
        a.group.c_stride = b.pairs * b.ldz * (int64_t)sizeof(float);
        if (launch_experts(d->type, P_DELTA, low ? E_PAIR : E_STORE, b.dx.kernel, a, tiles(b.dx), stream) != hipSuccess) return DN_ERR_DEVICE;
        if (launch_join(d->type, {dx, low, nullptr, dX_dev, b.ldz, 0, d->d, nullptr, place_dev, d->rows, d->d, d->k, (int32_t)b.pairs, b.dx.parts,
                                  b.pairs * b.ldz},
                        stream, joined) != hipSuccess)
            return DN_ERR_DEVICE;
    }
    const bool f32_out = d->grad_type == DN_F32;
    const int64_t matrix = (int64_t)d->d * f * size_of(d->grad_type);
    {   // dWg and dWu: the columns of dG (and of the zeros up to ldh), then those of dU
        ProductArgs a = product(g, (int)(2 * b.ldh), d->d, 0, 1, 0);
        operand_a(a, {dG, 2 * b.ldh * e, (int32_t)(2 * b.ldh)});
        operand_b(a, X);
        a.group.c_stride = matrix;
        a.f.y = dWg_dev;
        a.f.ldy = d->d;
        a.f.y2 = dWu_dev;
        a.f.ldy2 = d->d;
        a.f.m_split = (int)b.ldh;
        a.f.m_valid = d->f;
        a.f.f32_out = f32_out;
        a.f.alpha = d->grad_scale;
        if (launch_experts(d->type, P_GRAD, E_STORE, b.dwgu.kernel, a, 0, stream, 1) != hipSuccess) return DN_ERR_DEVICE;
    }
    ProductArgs a = product(g, d->d, d->f, 0, 1, 0);
    operand_a(a, dY);
    operand_b(a, {H, b.ldh * e, (int32_t)b.ldh});
    a.group.c_stride = matrix;
    a.f.y = dWd_dev;
    a.f.ldy = f;
    a.f.f32_out = f32_out;
    a.f.alpha = d->grad_scale;
    return device(launch_experts(d->type, P_GRAD, E_STORE, b.dwd.kernel, a, 0, stream));
}

}  // extern "C"
