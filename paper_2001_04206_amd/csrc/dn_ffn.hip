// Host side of the residual feed-forward block's operators: checks, plans, workspaces and launches.
#include "dn_ffn.h"

#include <math.h>

namespace dn {
namespace {

constexpr int64_t kRowBytes = (int64_t)8 << 20;   // a tile's 32-bit offsets hold 255 rows of this
constexpr size_t kBad = (size_t)-1;

int64_t size_of(int type) { return type == DN_F32 ? 4 : 2; }
bool type_ok(int type) { return type == DN_F32 || type == DN_F16 || type == DN_BF16; }
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

hipError_t launch_product(int type, Product p, Epilogue e, const ProductPlan &plan, const ProductArgs &a, hipStream_t s)
{
    return type == DN_F32 ? launch_product_f32(p, e, plan, a, s)
           : type == DN_F16 ? launch_product_f16(p, e, plan, a, s) : launch_product_bf16(p, e, plan, a, s);
}

// sixteen-byte pieces: rows of `n` elements `ld` apart from p on
bool pieces(int type, const void *p, int64_t ld, int64_t n)
{
    const int64_t e = size_of(type);
    return ((uintptr_t)p | (uintptr_t)(ld * e) | (uintptr_t)(n * e)) % 16 == 0;
}

dn_status drop_of(float p, uint64_t seed, uint64_t offset, Dropout &d)
{
    if (!(p >= 0.f && p < 1.f)) return DN_ERR_INVALID_ARG;
    const int t = (int)floorf(p * 65536.f + 0.5f);
    d.t = (uint32_t)(t > 65535 ? 65535 : t);
    d.scale = 65536.f / (float)(65536 - (int)d.t);
    d.k0 = (uint32_t)seed;
    d.k1 = (uint32_t)(seed >> 32);
    d.o0 = (uint32_t)offset;
    d.o1 = (uint32_t)(offset >> 32);
    return DN_OK;
}

// a leading dimension: 0 means contiguous
dn_status row_length(int type, int64_t &ld, int64_t n)
{
    if (ld == 0) ld = n;
    return ld < n || ld * size_of(type) > kRowBytes ? DN_ERR_SHAPE : DN_OK;
}
// more threads than a launch can have: one for eight columns, or 512 for a tile, 64 x 64 the smallest one
bool too_many(int64_t rows, int64_t cols)
{
    constexpr int64_t kThreads = (int64_t)1 << 32;
    return rows * ((cols + 7) / 8) >= kThreads || (rows + 63) / 64 * ((cols + 63) / 64) >= kThreads / 512;
}
dn_status common(int type, int grad_type, int act, int32_t rows, int32_t n, int32_t m, float grad_scale)
{
    if (!type_ok(type) || (grad_type != type && grad_type != DN_F32)) return DN_ERR_INVALID_ARG;
    if (act == DN_ACT_SOFTMAX) return DN_ERR_UNSUPPORTED;
    if (act < DN_ACT_LINEAR || act > DN_ACT_GELU || !isfinite(grad_scale)) return DN_ERR_INVALID_ARG;
    if (rows < 1 || n < 1 || m < 1) return DN_ERR_SHAPE;
    if ((int64_t)n * size_of(type) > kRowBytes || (int64_t)m * size_of(type) > kRowBytes) return DN_ERR_SHAPE;
    return too_many(rows, n) || too_many(rows, m) || too_many(n, m) ? DN_ERR_SHAPE : DN_OK;
}
template <class... P>
bool multiples(int type, const P *...p)
{
    uintptr_t all = 0;
    ((all |= (uintptr_t)p), ...);
    return all % (uintptr_t)size_of(type) == 0;
}

dn_status workspace(size_t need, const void *ws, size_t bytes)
{
    if (need == 0) return DN_OK;
    if (!ws || (uintptr_t)ws % 256) return DN_ERR_INVALID_ARG;
    return bytes < need ? DN_ERR_SHAPE : DN_OK;
}
// Operands of tiles: those whose rows are not in sixteen-byte pieces are copied to the workspace, from `at` on.
int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
size_t packed_bytes(int type, int64_t rows, int64_t cols) { return up256((size_t)rows * (size_t)(up8(cols) * size_of(type))); }
struct Packer {
    int type;
    char *at;
    PackArgs a{};
    struct Rows {
        const void *p;
        int64_t ld;     // bytes
        int32_t ext;    // elements of a row that may be read
    };
    Rows take(const void *p, int64_t ld, int64_t rows, int64_t cols, bool must = false)
    {
        if (!must && pieces(type, p, ld, cols)) return {p, ld * size_of(type), (int32_t)cols};
        auto &m = a.m[a.n++];
        m.x = p;
        m.y = at;
        m.ldx = ld;
        m.rows = (int32_t)rows;
        m.cols = (int32_t)cols;
        m.first = a.groups;
        a.groups += rows * (up8(cols) / 8);
        at += packed_bytes(type, rows, cols);
        return {m.y, up8(cols) * size_of(type), (int32_t)up8(cols)};
    }
    hipError_t run(hipStream_t s, const MaskArgs *mask = nullptr) const { return launch_mask_pack(type, mask, a, s); }
};
void operand_a(ProductArgs &a, const Packer::Rows &r)
{
    a.a[0] = a.a[1] = r.p;
    a.lda = r.ld;
    a.a_ext = r.ext;
}
void operand_b(ProductArgs &a, const Packer::Rows &r)
{
    a.b[0] = a.b[1] = r.p;
    a.ldb = r.ld;
    a.b_ext = r.ext;
}

dn_status device(hipError_t e) { return e == hipSuccess ? DN_OK : DN_ERR_DEVICE; }

// ---- dense layer -------------------------------------------------------------------------------------------------
struct Linear {
    dn_linear_desc d;
    Dropout drop;
    ProductPlan fwd, dx, dw;
    size_t fwd_part = 0, fwd_bytes = 0;                  // workspace: parts of a product, packed operands
    size_t delta = 0, bwd_part = 0, bwd_bytes = 0;       // delta, parts, packed operands
};

dn_status linear_of(const dn_linear_desc *d, Linear &l)
{
    if (!d) return DN_ERR_INVALID_ARG;
    l.d = *d;
    dn_status s = common(d->type, d->grad_type, d->act, d->rows, d->n_in, d->n_out, d->grad_scale);
    if (s != DN_OK) return s;
    if ((s = drop_of(d->drop, d->seed, d->offset, l.drop)) != DN_OK) return s;
    if ((s = row_length(d->type, l.d.ldx, d->n_in)) != DN_OK || (s = row_length(d->type, l.d.ldw, d->n_in)) != DN_OK ||
        (s = row_length(d->type, l.d.ldr, d->n_out)) != DN_OK || (s = row_length(d->type, l.d.ldy, d->n_out)) != DN_OK)
        return s;
    const size_t packed = packed_bytes(d->type, d->rows, d->n_in) + packed_bytes(d->type, d->n_out, d->n_in);
    l.fwd = plan_product(d->type, P_FWD, E_LINEAR, d->rows, d->n_out, d->n_in, 1, false);
    l.fwd_part = up256(l.fwd.ws_bytes);
    l.fwd_bytes = l.fwd.kernel == K_FEW ? 0 : l.fwd_part + packed;
    l.dx = plan_product(d->type, P_DELTA, E_STORE, d->rows, d->n_in, d->n_out, 1, false);
    l.dw = plan_product(d->type, P_GRAD, E_STORE, d->n_out, d->n_in, d->rows, 1, true);
    l.delta = packed_bytes(d->type, d->rows, d->n_out);
    l.bwd_part = up256(l.dx.ws_bytes > l.dw.ws_bytes ? l.dx.ws_bytes : l.dw.ws_bytes);
    l.bwd_bytes = l.delta + l.bwd_part + packed;
    return DN_OK;
}

// ---- gated block ---------------------------------------------------------------------------------------------------
struct Gated {
    dn_ffn_desc d;
    Dropout drop;
    int64_t ldh;         // between rows of H; dU starts so many columns after dG
    ProductPlan up, down, dh, dx, dwgu, dwd;
    size_t h = 0, fwd_part = 0, fwd_bytes = 0;                       // workspace: H, parts of a product, packed operands
    size_t dgu = 0, dz = 0, bwd_part = 0, bwd_bytes = 0;             // H, dG and dU, dZ, parts, packed operands
};

dn_status gated_of(const dn_ffn_desc *d, Gated &g)
{
    if (!d) return DN_ERR_INVALID_ARG;
    g.d = *d;
    dn_status s = common(d->type, d->grad_type, d->act, d->rows, d->d, d->f, d->grad_scale);
    if (s != DN_OK) return s;
    if ((s = drop_of(d->drop, d->seed, d->offset, g.drop)) != DN_OK) return s;
    if ((s = row_length(d->type, g.d.ldx, d->d)) != DN_OK || (s = row_length(d->type, g.d.ldr, d->d)) != DN_OK ||
        (s = row_length(d->type, g.d.ldy, d->d)) != DN_OK)
        return s;
    const int64_t e = size_of(d->type);
    g.ldh = up8(d->f);
    if (2 * g.ldh * e > kRowBytes) return DN_ERR_SHAPE;
    g.h = up256((size_t)d->rows * (size_t)(g.ldh * e));
    const size_t ups = packed_bytes(d->type, d->rows, d->d) + 2 * packed_bytes(d->type, d->f, d->d), packed = ups + packed_bytes(d->type, d->d, d->f);
    g.up = plan_product(d->type, P_FWD, E_GATED, d->rows, d->f, d->d, 1, false);
    g.down = plan_product(d->type, P_FWD, E_LINEAR, d->rows, d->d, d->f, 1, false);
    g.fwd_part = up256(g.up.ws_bytes > g.down.ws_bytes ? g.up.ws_bytes : g.down.ws_bytes);
    g.fwd_bytes = g.h + g.fwd_part + (g.up.kernel == K_FEW ? 0 : ups) + (g.down.kernel == K_FEW ? 0 : packed - ups);
    g.dh = plan_product(d->type, P_DELTA, E_DGATED, d->rows, d->f, d->d, 1, false);
    g.dx = plan_product(d->type, P_DELTA, E_STORE, d->rows, d->d, d->f, 2, false);
    g.dwgu = plan_product(d->type, P_GRAD, E_STORE, (int)(2 * g.ldh), d->d, d->rows, 1, true);
    g.dwd = plan_product(d->type, P_GRAD, E_STORE, d->d, d->f, d->rows, 1, true);
    for (const ProductPlan *p : {&g.dh, &g.dx, &g.dwgu, &g.dwd}) g.bwd_part = g.bwd_part > p->ws_bytes ? g.bwd_part : p->ws_bytes;
    g.bwd_part = up256(g.bwd_part);
    g.dgu = 2 * g.h;
    g.dz = packed_bytes(d->type, d->rows, d->d);
    g.bwd_bytes = g.h + g.dgu + g.dz + g.bwd_part + packed;
    return DN_OK;
}

// ---- norms ---------------------------------------------------------------------------------------------------------
dn_status norm_of(const dn_norm_desc *d, NormArgs &a)
{
    a = NormArgs{};
    if (!d || !type_ok(d->type) || (d->grad_type != d->type && d->grad_type != DN_F32)) return DN_ERR_INVALID_ARG;
    if (d->post < DN_NORM_NONE || d->post > DN_NORM_LAYER || d->pre < DN_NORM_NONE || d->pre > DN_NORM_LAYER) return DN_ERR_INVALID_ARG;
    if (!isfinite(d->scale) || !isfinite(d->eps) || d->eps < 0.f) return DN_ERR_INVALID_ARG;
    if (d->rows < 1 || d->d < 1 || d->d > kNormWidth || d->rows_per_gate < 1) return DN_ERR_SHAPE;
    a.rows = d->rows;
    a.d = d->d;
    a.group = d->rows_per_gate < d->rows ? d->rows_per_gate : d->rows;
    a.post = d->post;
    a.pre = d->pre;
    a.f32_out = d->grad_type == DN_F32;
    a.scale = d->scale;
    a.eps = d->eps;
    return DN_OK;
}

}  // namespace

constexpr int kUnits = 256;   // compute units

ProductPlan plan_product(int type, Product p, Epilogue e, int M, int N, int K, int segments, bool sums)
{
    ProductPlan plan;
    const int bk = type == DN_F32 ? 32 : 64, steps = (K + bk - 1) / bk * segments;
    plan.steps = steps;
    const bool few = p == P_FWD && M <= kFewRows && (int64_t)K * size_of(type) >= 32;
    if (few && M <= 16) {
        plan.kernel = K_FEW;
        return plan;
    }
    // Which kernel, and k in how many parts: whichever is expected to take least.  Microseconds a stage, a round of workgroups and
    // bytes, as measured.  A stage of a 256 x 256 tile takes 1.5 us whether the chip is full or not, one of 128 x 256 0.8; fp32 is
    // bound by its matrix instruction at any size, 1.8 us for a tile of 128 x 128 and 0.95 for one of 64 x 128.  2048 x 4096 x 1024
    // so takes 20 us on 256 medium tiles (128 large ones: 32), 8192 x 4096 x 4096 260 on 512 large ones (medium: 330); few short tiles
    // are better small, more waves sharing their epilogue: 700 x 1024 x 512 11.8 us (medium: 16.2), but 1024 x 2048 x 8192 61 for
    // the medium ones' 43, as a stage of any tile takes what memory does.  In fp32
    // 1301 x 1021 x 777 32 us on 168 tiny tiles (small ones in parts: 33 and 5 to join them), 8192 x 4096 x 4096 1941 on 2048 small
    // ones (tiny: 1988).  Weights come at 4.6 TB/s, and up to 64 rows the kernel that stages nothing competes, whose workgroups of 16
    // columns each read all rows, at 11 TB/s: through a gated product of 4096 x 8192 x 2, 8 rows take 29 us there (tiles: 35), 32 rows
    // 42 (tiles: 35), 64 rows 58 (tiles: 37).  Up to 16 rows it is taken without asking.  Tiles at widths that are no multiple of
    // 16 bytes need a copy first.
    const int planes = e == E_GATED ? 2 : 1;
    const double es = (double)size_of(type), weights = es * planes * N * K * segments / 4.6e6;
    double best = 1e300;
    const double copies = (int64_t)K * size_of(type) % 16 == 0 ? 0 : 4 + 2 * (weights + es * M * K / 4.6e6);
    if (few) {
        best = 6 + weights + (N + 15) / 16 * ((M + 15) / 16 * 16.) * K * es / 11e6 - copies;
        plan.kernel = K_FEW;
    }
    struct Way { ProductKernel kernel; int rows, cols, together; double stage, least, round; };   // least: of a stage, when alone
    const Way tiny{K_TINY, 64, 128, 3, 0.95, 0.95, 6}, large{K_LARGE, 256, 256, 1, 1.5, 1.5, 8}, medium{K_MEDIUM, 128, 256, 1, 0.8, 0.8, 6};
    const Way small = type == DN_F32 ? Way{K_SMALL, 128, 128, 2, 1.8, 1.8, 6} : Way{K_SMALL, 128, 128, 2, 0.5, 0.9, 4};
    for (const Way &w : {large, medium, small, tiny}) {
        if (type == DN_F32 ? w.kernel > K_SMALL : w.kernel == K_TINY) continue;
        const int64_t cols = w.cols / planes, t = (M + w.rows - 1) / w.rows * ((N + cols - 1) / cols);
        for (int split = 1; split <= 32 && split * 4 <= steps + 3; ++split) {
            int each = (steps + split - 1) / split;
            if (w.kernel == K_LARGE) each = (each + 1) / 2 * 2;
            const int parts = (steps + each - 1) / each;
            const int64_t deep = (t * parts + kUnits - 1) / kUnits, rounds = (deep + w.together - 1) / w.together;   // on a compute unit
            const double stage = deep * w.stage > rounds * w.least ? deep * w.stage : rounds * w.least;
            double us = each * stage + rounds * w.round;
            if (p == P_FWD && us < weights) us = weights;
            if (parts > 1) us += 3 + 8e-6 * parts * planes * M * N / 4.5;
            if (us < best) {
                best = us;
                plan.kernel = w.kernel;
                plan.split = parts;
                plan.steps = each;
            }
        }
    }
    if (plan.split > 1) plan.ws_bytes = (size_t)plan.split * (size_t)M * (size_t)N * planes * sizeof(float);
    if (sums && plan.kernel == K_LARGE) plan.ws_bytes += (size_t)kSumParts * (size_t)M * sizeof(float);
    else if (sums && plan.split > 1) plan.ws_bytes += (size_t)plan.split * (size_t)M * sizeof(float);
    return plan;
}

}  // namespace dn

using namespace dn;

extern "C" {

size_t dn_linear_forward_workspace_bytes(const dn_linear_desc *d)
{
    Linear l;
    return linear_of(d, l) == DN_OK ? l.fwd_bytes : kBad;
}

size_t dn_linear_backward_workspace_bytes(const dn_linear_desc *d)
{
    Linear l;
    return linear_of(d, l) == DN_OK ? l.bwd_bytes : kBad;
}

dn_status dn_linear_forward(const dn_linear_desc *d, const void *X_dev, const void *W_dev, const void *bias_dev,
                            const void *R_dev, void *Y_dev, void *Z_dev, void *workspace_dev, size_t workspace_bytes,
                            void *hip_stream)
{
    Linear l;
    dn_status s = linear_of(d, l);
    if (s != DN_OK) return s;
    if (!X_dev || !W_dev || !Y_dev || !multiples(d->type, X_dev, W_dev, bias_dev, R_dev, Y_dev, Z_dev)) return DN_ERR_INVALID_ARG;
    if ((s = workspace(l.fwd_bytes, workspace_dev, workspace_bytes)) != DN_OK) return s;
    const hipStream_t stream = (hipStream_t)hip_stream;
    ProductArgs a{};
    a.M = d->rows;
    a.N = d->n_out;
    a.K = d->n_in;
    a.segments = 1;
    a.ws = static_cast<float *>(workspace_dev);
    if (l.fwd.kernel == K_FEW) {
        operand_a(a, {X_dev, l.d.ldx * size_of(d->type), d->n_in});
        operand_b(a, {W_dev, l.d.ldw * size_of(d->type), d->n_in});
    } else {
        Packer pack{d->type, static_cast<char *>(workspace_dev) + l.fwd_part};
        operand_a(a, pack.take(X_dev, l.d.ldx, d->rows, d->n_in));
        operand_b(a, pack.take(W_dev, l.d.ldw, d->n_out, d->n_in));
        if (pack.run(stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    a.f.y = Y_dev;
    a.f.ldy = l.d.ldy;
    a.f.y2 = Z_dev;
    a.f.ldy2 = d->n_out;
    a.f.r = R_dev;
    a.f.ldr = l.d.ldr;
    a.f.bias = bias_dev;
    a.f.act = d->act;
    a.f.drop = l.drop;
    return device(launch_product(d->type, P_FWD, E_LINEAR, l.fwd, a, stream));
}

dn_status dn_linear_backward(const dn_linear_desc *d, const void *X_dev, const void *W_dev, const void *Z_dev,
                             const void *dY_dev, void *dX_dev, void *dW_dev, void *dbias_dev, void *workspace_dev,
                             size_t workspace_bytes, void *hip_stream)
{
    Linear l;
    dn_status s = linear_of(d, l);
    if (s != DN_OK) return s;
    if (!X_dev || !W_dev || !dY_dev || (!Z_dev && d->act != DN_ACT_LINEAR) || (dbias_dev && !dW_dev)) return DN_ERR_INVALID_ARG;
    if (!multiples(d->type, X_dev, W_dev, Z_dev, dY_dev, dX_dev) || !multiples(d->grad_type, dW_dev, dbias_dev)) return DN_ERR_INVALID_ARG;
    if ((s = workspace(l.bwd_bytes, workspace_dev, workspace_bytes)) != DN_OK) return s;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t e = size_of(d->type);
    char *ws = static_cast<char *>(workspace_dev);
    // delta, without dropout's scale, by which the products' sums are multiplied; dY itself where it is that and lies well
    Packer::Rows delta{dY_dev, l.d.ldy * e, d->n_out};
    const bool mask = d->act != DN_ACT_LINEAR || l.drop.t || !pieces(d->type, dY_dev, l.d.ldy, d->n_out);
    MaskArgs m{};
    if (mask) {
        const int64_t ld = up8(d->n_out);
        m.x = dY_dev;
        m.z = Z_dev;
        m.y = ws;
        m.ldx = l.d.ldy;
        m.ldz = d->n_out;
        m.ldy = ld;
        m.rows = d->rows;
        m.cols = d->n_out;
        m.zeros = (int)(ld - d->n_out);
        m.act = d->act;
        m.drop = l.drop;
        m.drop.scale = 1.f;
        delta = {ws, ld * e, (int32_t)ld};
    }
    Packer pack{d->type, ws + l.delta + l.bwd_part};
    const Packer::Rows X = dW_dev ? pack.take(X_dev, l.d.ldx, d->rows, d->n_in) : Packer::Rows{};
    const Packer::Rows W = dX_dev ? pack.take(W_dev, l.d.ldw, d->n_out, d->n_in) : Packer::Rows{};
    if (pack.run(stream, mask ? &m : nullptr) != hipSuccess) return DN_ERR_DEVICE;
    ProductArgs a{};
    a.segments = 1;
    a.ws = reinterpret_cast<float *>(ws + l.delta);
    operand_a(a, delta);
    a.N = d->n_in;
    a.f.ldy = d->n_in;
    if (dX_dev) {
        operand_b(a, W);
        a.M = d->rows;
        a.K = d->n_out;
        a.f.y = dX_dev;
        a.f.alpha = l.drop.scale;
        if (launch_product(d->type, P_DELTA, E_STORE, l.dx, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    if (dW_dev) {
        operand_b(a, X);
        a.M = d->n_out;
        a.K = d->rows;
        a.f.y = dW_dev;
        a.f.sums = dbias_dev;
        a.f.f32_out = d->grad_type == DN_F32;
        a.f.alpha = l.drop.scale * d->grad_scale;
        if (launch_product(d->type, P_GRAD, E_STORE, l.dw, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    return DN_OK;
}

size_t dn_ffn_forward_workspace_bytes(const dn_ffn_desc *d)
{
    Gated g;
    return gated_of(d, g) == DN_OK ? g.fwd_bytes : kBad;
}

size_t dn_ffn_backward_workspace_bytes(const dn_ffn_desc *d)
{
    Gated g;
    return gated_of(d, g) == DN_OK ? g.bwd_bytes : kBad;
}

dn_status dn_ffn_forward(const dn_ffn_desc *d, const void *X_dev, const void *Wg_dev, const void *bg_dev, const void *Wu_dev,
                         const void *bu_dev, const void *Wd_dev, const void *bd_dev, const void *R_dev, void *Y_dev,
                         void *GU_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    Gated g;
    dn_status s = gated_of(d, g);
    if (s != DN_OK) return s;
    if (!X_dev || !Wg_dev || !Wu_dev || !Wd_dev || !Y_dev) return DN_ERR_INVALID_ARG;
    if (!multiples(d->type, X_dev, Wg_dev, bg_dev, Wu_dev, bu_dev, Wd_dev, bd_dev, R_dev, Y_dev, GU_dev)) return DN_ERR_INVALID_ARG;
    if ((s = workspace(g.fwd_bytes, workspace_dev, workspace_bytes)) != DN_OK) return s;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t e = size_of(d->type);
    char *H = static_cast<char *>(workspace_dev);
    ProductArgs a{}, b{};
    Packer pack{d->type, H + g.h + g.fwd_part};
    if (g.up.kernel == K_FEW) {
        operand_a(a, {X_dev, g.d.ldx * e, d->d});
        operand_b(a, {Wg_dev, d->d * e, d->d});
        a.b[1] = Wu_dev;
    } else {
        operand_a(a, pack.take(X_dev, g.d.ldx, d->rows, d->d));
        const bool both = !pieces(d->type, Wg_dev, d->d, d->d) || !pieces(d->type, Wu_dev, d->d, d->d);   // they share a stride
        operand_b(a, pack.take(Wg_dev, d->d, d->f, d->d, both));
        a.b[1] = pack.take(Wu_dev, d->d, d->f, d->d, both).p;
    }
    if (g.down.kernel == K_FEW) operand_b(b, {Wd_dev, d->f * e, d->f});
    else operand_b(b, pack.take(Wd_dev, d->f, d->d, d->f));
    if (pack.run(stream) != hipSuccess) return DN_ERR_DEVICE;
    a.M = d->rows;
    a.N = d->f;
    a.K = d->d;
    a.segments = 1;
    a.ws = reinterpret_cast<float *>(H + g.h);
    a.f.y = H;
    a.f.ldy = g.ldh;
    a.f.zeros = (int)(g.ldh - d->f);
    a.f.y2 = GU_dev;
    a.f.ldy2 = 2 * (int64_t)d->f;
    a.f.half = d->f;
    a.f.bias = bg_dev;
    a.f.bias2 = bu_dev;
    a.f.act = d->act;
    if (launch_product(d->type, P_FWD, E_GATED, g.up, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    operand_a(b, {H, g.ldh * e, (int32_t)g.ldh});
    b.M = d->rows;
    b.N = d->d;
    b.K = d->f;
    b.segments = 1;
    b.ws = a.ws;
    b.f.y = Y_dev;
    b.f.ldy = g.d.ldy;
    b.f.r = R_dev;
    b.f.ldr = g.d.ldr;
    b.f.bias = bd_dev;
    b.f.drop = g.drop;
    return device(launch_product(d->type, P_FWD, E_LINEAR, g.down, b, stream));
}

dn_status dn_ffn_backward(const dn_ffn_desc *d, const void *X_dev, const void *Wg_dev, const void *Wu_dev, const void *Wd_dev,
                          const void *GU_dev, const void *dY_dev, void *dX_dev, void *dWg_dev, void *dbg_dev, void *dWu_dev,
                          void *dbu_dev, void *dWd_dev, void *dbd_dev, void *workspace_dev, size_t workspace_bytes,
                          void *hip_stream)
{
    Gated g;
    dn_status s = gated_of(d, g);
    if (s != DN_OK) return s;
    if (!X_dev || !Wg_dev || !Wu_dev || !Wd_dev || !GU_dev || !dY_dev || !dWg_dev || !dWu_dev || !dWd_dev) return DN_ERR_INVALID_ARG;
    if (!multiples(d->type, X_dev, Wg_dev, Wu_dev, Wd_dev, GU_dev, dY_dev, dX_dev) ||
        !multiples(d->grad_type, dWg_dev, dbg_dev, dWu_dev, dbu_dev, dWd_dev, dbd_dev))
        return DN_ERR_INVALID_ARG;
    if ((s = workspace(g.bwd_bytes, workspace_dev, workspace_bytes)) != DN_OK) return s;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t e = size_of(d->type), f = d->f;
    char *ws = static_cast<char *>(workspace_dev);
    char *H = ws, *dG = H + g.h, *dU = dG + g.ldh * e;
    // dZ without dropout's scale, by which the sums of the two products that read it are multiplied; dY itself where it is that
    // and lies well
    Packer::Rows dZ{dY_dev, g.d.ldy * e, d->d};
    const bool mask = g.drop.t || !pieces(d->type, dY_dev, g.d.ldy, d->d);
    MaskArgs m{};
    if (mask) {
        const int64_t ld = up8(d->d);
        m.x = dY_dev;
        m.y = ws + g.h + g.dgu;
        m.ldx = g.d.ldy;
        m.ldy = ld;
        m.rows = d->rows;
        m.cols = d->d;
        m.zeros = (int)(ld - d->d);
        m.act = -1;
        m.drop = g.drop;
        m.drop.scale = 1.f;
        dZ = {m.y, ld * e, (int32_t)ld};
    }
    Packer pack{d->type, ws + g.h + g.dgu + g.dz + g.bwd_part};
    const Packer::Rows X = pack.take(X_dev, g.d.ldx, d->rows, d->d), Wd = pack.take(Wd_dev, f, d->d, f);
    const bool both = !pieces(d->type, Wg_dev, d->d, d->d) || !pieces(d->type, Wu_dev, d->d, d->d);   // they share a stride
    const Packer::Rows Wg = dX_dev ? pack.take(Wg_dev, d->d, f, d->d, both) : Packer::Rows{};
    const Packer::Rows Wu = dX_dev ? pack.take(Wu_dev, d->d, f, d->d, both) : Packer::Rows{};
    if (pack.run(stream, mask ? &m : nullptr) != hipSuccess) return DN_ERR_DEVICE;
    float *part = reinterpret_cast<float *>(ws + g.h + g.dgu + g.dz);
    const bool f32_out = d->grad_type == DN_F32;
    {   // dH, and from it dG, dU and H
        ProductArgs a{};
        operand_a(a, dZ);
        operand_b(a, Wd);
        a.M = d->rows;
        a.N = d->f;
        a.K = d->d;
        a.segments = 1;
        a.ws = part;
        a.f.y = dG;
        a.f.ldy = 2 * g.ldh;
        a.f.half_y = g.ldh;
        a.f.zeros = (int)(g.ldh - f);
        a.f.y2 = H;
        a.f.ldy2 = g.ldh;
        a.f.r = GU_dev;
        a.f.ldr = 2 * f;
        a.f.half = f;
        a.f.act = d->act;
        a.f.alpha = g.drop.scale;
        if (launch_product(d->type, P_DELTA, E_DGATED, g.dh, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    if (dX_dev) {
        ProductArgs a{};
        operand_a(a, {dG, 2 * g.ldh * e, (int32_t)g.ldh});
        a.a[1] = dU;
        operand_b(a, Wg);
        a.b[1] = Wu.p;
        a.M = d->rows;
        a.N = d->d;
        a.K = d->f;
        a.segments = 2;
        a.ws = part;
        a.f.y = dX_dev;
        a.f.ldy = d->d;
        if (launch_product(d->type, P_DELTA, E_STORE, g.dx, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    {   // dWg and dWu: the columns of dG (and of the zeros up to ldh), then those of dU
        ProductArgs a{};
        operand_a(a, {dG, 2 * g.ldh * e, (int32_t)(2 * g.ldh)});
        operand_b(a, X);
        a.M = (int)(2 * g.ldh);
        a.N = d->d;
        a.K = d->rows;
        a.segments = 1;
        a.ws = part;
        a.f.y = dWg_dev;
        a.f.ldy = d->d;
        a.f.y2 = dWu_dev;
        a.f.ldy2 = d->d;
        a.f.sums = dbg_dev;
        a.f.sums2 = dbu_dev;
        a.f.m_split = (int)g.ldh;
        a.f.m_valid = d->f;
        a.f.f32_out = f32_out;
        a.f.alpha = d->grad_scale;
        if (launch_product(d->type, P_GRAD, E_STORE, g.dwgu, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    ProductArgs a{};
    operand_a(a, dZ);
    operand_b(a, {H, g.ldh * e, (int32_t)g.ldh});
    a.M = d->d;
    a.N = d->f;
    a.K = d->rows;
    a.segments = 1;
    a.ws = part;
    a.f.y = dWd_dev;
    a.f.ldy = f;
    a.f.sums = dbd_dev;
    a.f.f32_out = f32_out;
    a.f.alpha = g.drop.scale * d->grad_scale;
    return device(launch_product(d->type, P_GRAD, E_STORE, g.dwd, a, stream));
}

size_t dn_norm_backward_workspace_bytes(const dn_norm_desc *d)
{
    NormArgs a;
    return norm_of(d, a) == DN_OK ? up256(norm_backward_plan(d->type, a)) : kBad;
}

dn_status dn_norm_forward(const dn_norm_desc *d, const void *x_dev, const void *b_dev, const void *gate_dev,
                          const void *post_w_dev, const void *post_b_dev, const void *pre_w_dev, const void *pre_b_dev,
                          void *x_out_dev, void *n_out_dev, void *hip_stream)
{
    NormArgs a;
    const dn_status s = norm_of(d, a);
    if (s != DN_OK) return s;
    if (!x_dev || (b_dev && !x_out_dev) || (d->pre && !n_out_dev) || (!b_dev && !d->pre)) return DN_ERR_INVALID_ARG;
    if ((post_b_dev && d->post != DN_NORM_LAYER) || (pre_b_dev && d->pre != DN_NORM_LAYER)) return DN_ERR_INVALID_ARG;
    if (!multiples(d->type, x_dev, b_dev, gate_dev, post_w_dev, post_b_dev, pre_w_dev, pre_b_dev, x_out_dev, n_out_dev)) return DN_ERR_INVALID_ARG;
    a.x = x_dev;
    a.b = b_dev;
    a.gate = gate_dev;
    a.post_w = d->post ? post_w_dev : nullptr;   // a weight without its norm takes no part
    a.post_b = post_b_dev;
    a.pre_w = d->pre ? pre_w_dev : nullptr;
    a.pre_b = pre_b_dev;
    a.x_out = x_out_dev;
    a.n_out = n_out_dev;
    return device(launch_norm_forward(d->type, a, (hipStream_t)hip_stream));
}

dn_status dn_norm_backward(const dn_norm_desc *d, const void *x_dev, const void *b_dev, const void *gate_dev,
                           const void *post_w_dev, const void *post_b_dev, const void *pre_w_dev, const void *dx_out_dev,
                           const void *dn_dev, void *dx_dev, void *db_dev, void *dgate_dev, void *dpost_w_dev,
                           void *dpost_b_dev, void *dpre_w_dev, void *dpre_b_dev, void *workspace_dev,
                           size_t workspace_bytes, void *hip_stream)
{
    NormArgs a;
    dn_status s = norm_of(d, a);
    if (s != DN_OK) return s;
    if (!dx_dev || (d->pre && (!x_dev || !dn_dev)) || (b_dev && !db_dev) || (!b_dev && !d->pre)) return DN_ERR_INVALID_ARG;
    if ((dgate_dev && (!b_dev || !gate_dev)) || (dpost_w_dev && (!b_dev || !d->post)) || (dpre_w_dev && !d->pre) ||
        (dpost_b_dev && (!b_dev || d->post != DN_NORM_LAYER)) || (dpre_b_dev && d->pre != DN_NORM_LAYER) ||
        (post_b_dev && d->post != DN_NORM_LAYER))
        return DN_ERR_INVALID_ARG;
    if (!multiples(d->type, x_dev, b_dev, gate_dev, post_w_dev, post_b_dev, pre_w_dev, dx_out_dev, dn_dev, dx_dev, db_dev) ||
        !multiples(d->grad_type, dgate_dev, dpost_w_dev, dpost_b_dev, dpre_w_dev, dpre_b_dev))
        return DN_ERR_INVALID_ARG;
    if ((s = workspace(up256(norm_backward_plan(d->type, a)), workspace_dev, workspace_bytes)) != DN_OK) return s;
    a.x = x_dev;
    a.b = b_dev;
    a.gate = gate_dev;
    a.post_w = d->post ? post_w_dev : nullptr;   // a weight without its norm takes no part
    a.post_b = post_b_dev;
    a.pre_w = d->pre ? pre_w_dev : nullptr;
    a.dx_out = dx_out_dev;
    a.dn = dn_dev;
    a.dx = dx_dev;
    a.db = db_dev;
    a.dgate = dgate_dev;
    a.dpost_w = dpost_w_dev;
    a.dpost_b = dpost_b_dev;
    a.dpre_w = dpre_w_dev;
    a.dpre_b = dpre_b_dev;
    a.ws = static_cast<float *>(workspace_dev);
    return device(launch_norm_backward(d->type, a, (hipStream_t)hip_stream));
}

dn_status dn_dropout(int32_t type, const void *X_dev, void *Y_dev, int32_t rows, int32_t cols, int64_t ldx, int64_t ldy,
                     float drop, uint64_t seed, uint64_t offset, void *hip_stream)
{
    if (!X_dev || !Y_dev || !type_ok(type) || !multiples(type, X_dev, Y_dev)) return DN_ERR_INVALID_ARG;
    MaskArgs m{};
    dn_status s = drop_of(drop, seed, offset, m.drop);
    if (s != DN_OK) return s;
    if (rows < 1 || cols < 1 || too_many(rows, cols)) return DN_ERR_SHAPE;
    if ((s = row_length(type, ldx, cols)) != DN_OK || (s = row_length(type, ldy, cols)) != DN_OK) return s;
    m.x = X_dev;
    m.y = Y_dev;
    m.ldx = ldx;
    m.ldy = ldy;
    m.rows = rows;
    m.cols = cols;
    m.act = -1;
    return device(launch_mask_pack(type, &m, {}, (hipStream_t)hip_stream));
}

}  // extern "C"
