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
dn_status common(int type, int grad_type, int act, int32_t rows, int32_t n, int32_t m, float grad_scale)
{
    if (!type_ok(type) || (grad_type != type && grad_type != DN_F32)) return DN_ERR_INVALID_ARG;
    if (act == DN_ACT_SOFTMAX) return DN_ERR_UNSUPPORTED;
    if (act < DN_ACT_LINEAR || act > DN_ACT_GELU || !isfinite(grad_scale)) return DN_ERR_INVALID_ARG;
    if (rows < 1 || n < 1 || m < 1) return DN_ERR_SHAPE;
    if ((int64_t)n * size_of(type) > kRowBytes || (int64_t)m * size_of(type) > kRowBytes) return DN_ERR_SHAPE;
    // tiles of a launch, at 128 x 64 columns the smallest ones
    if (((int64_t)rows + 127) / 128 * (((int64_t)(n > m ? n : m) + 63) / 64) > 0x7fffffff) return DN_ERR_SHAPE;
    return DN_OK;
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
dn_status device(hipError_t e) { return e == hipSuccess ? DN_OK : DN_ERR_DEVICE; }

// ---- dense layer -------------------------------------------------------------------------------------------------
struct Linear {
    dn_linear_desc d;
    Dropout drop;
    bool plain;          // delta is dY
    int64_t ldd;         // between rows of delta
    size_t delta = 0, part = 0, bytes = 0;   // backward workspace: delta, parts of a product
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
    l.plain = d->act == DN_ACT_LINEAR && l.drop.t == 0;
    l.ldd = l.plain ? l.d.ldy : ((int64_t)d->n_out + 7) / 8 * 8;
    if (!l.plain) l.delta = up256((size_t)d->rows * (size_t)l.ldd * (size_t)size_of(d->type));
    // parts: of whichever operands, at whichever alignment
    for (int direct = 0; direct < 2; ++direct) {
        const size_t x = plan_product(d->type, P_DELTA, E_STORE, d->rows, d->n_in, d->n_out, 1, direct, false).ws_bytes;
        const size_t w = plan_product(d->type, P_GRAD, E_STORE, d->n_out, d->n_in, d->rows, 1, direct, true).ws_bytes;
        l.part = l.part > x ? l.part : x;
        l.part = l.part > w ? l.part : w;
    }
    l.bytes = l.delta + up256(l.part);
    return DN_OK;
}
size_t linear_forward_bytes(const Linear &l)
{
    const dn_linear_desc &d = l.d;
    const size_t a = plan_product(d.type, P_FWD, E_LINEAR, d.rows, d.n_out, d.n_in, 1, false, false).ws_bytes;
    const size_t b = plan_product(d.type, P_FWD, E_LINEAR, d.rows, d.n_out, d.n_in, 1, true, false).ws_bytes;
    return up256(a > b ? a : b);
}

// ---- gated block ---------------------------------------------------------------------------------------------------
struct Gated {
    dn_ffn_desc d;
    Dropout drop;
    int64_t ldh;         // between rows of H; dU starts so many columns after dG
    size_t h = 0, fwd_bytes = 0;
    size_t dgu = 0, dz = 0, part = 0, bwd_bytes = 0;
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
    g.ldh = ((int64_t)d->f + 15) / 16 * 16;
    if (2 * g.ldh * e > kRowBytes) return DN_ERR_SHAPE;
    g.h = up256((size_t)d->rows * (size_t)(g.ldh * e));
    size_t part = 0;
    auto take = [&](Product p, Epilogue ep, int M, int N, int K, int segments, bool sums) {
        for (int direct = 0; direct < 2; ++direct) {
            const size_t n = plan_product(d->type, p, ep, M, N, K, segments, direct, sums).ws_bytes;
            part = part > n ? part : n;
        }
    };
    take(P_FWD, E_GATED, d->rows, d->f, d->d, 1, false);
    take(P_FWD, E_LINEAR, d->rows, d->d, d->f, 1, false);
    g.fwd_bytes = g.h + up256(part);
    part = 0;
    take(P_DELTA, E_DGATED, d->rows, d->f, d->d, 1, false);
    take(P_DELTA, E_STORE, d->rows, d->d, d->f, 2, false);
    take(P_GRAD, E_STORE, (int)(2 * g.ldh), d->d, d->rows, 1, true);
    take(P_GRAD, E_STORE, d->d, d->f, d->rows, 1, true);
    g.part = up256(part);
    g.dgu = 2 * g.h;
    g.dz = g.drop.t ? up256((size_t)d->rows * (size_t)(((int64_t)d->d + 7) / 8 * 8 * e)) : 0;
    g.bwd_bytes = g.h + g.dgu + g.dz + g.part;
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

ProductPlan plan_product(int type, Product p, Epilogue e, int M, int N, int K, int segments, bool direct, bool sums)
{
    ProductPlan plan;
    plan.direct = direct;
    const int bk = type == DN_F32 ? 32 : 64, steps = (K + bk - 1) / bk * segments;
    plan.steps = steps;
    if (p == P_FWD && M <= 64) {
        plan.kernel = K_FEW;
        return plan;
    }
    auto tiles = [&](int64_t edge) { return (M + edge - 1) / edge * ((N + (e == E_GATED ? edge / 2 : edge) - 1) / (e == E_GATED ? edge / 2 : edge)); };
    if (type != DN_F32 && direct && tiles(256) >= 192) {
        plan.kernel = K_LARGE;
        if (sums) plan.ws_bytes = (size_t)kSumParts * (size_t)M * sizeof(float);
        return plan;
    }
    plan.kernel = direct ? K_SMALL : K_SMALL_ANY;
    // two workgroups of 128 x 128 fit a compute unit: split k until there are that many, at four steps at least
    const int64_t t = tiles(128);
    int64_t split = (512 + t / 2) / t;
    if (split > steps / 4) split = steps / 4;
    if (split > 1) {
        plan.steps = (int)((steps + split - 1) / split);
        plan.split = (steps + plan.steps - 1) / plan.steps;
    }
    if (plan.split > 1) plan.ws_bytes = (size_t)plan.split * ((size_t)M * (size_t)N * (e == E_GATED ? 2 : 1) + (sums ? (size_t)M : 0)) * sizeof(float);
    return plan;
}

}  // namespace dn

using namespace dn;

extern "C" {

size_t dn_linear_forward_workspace_bytes(const dn_linear_desc *d)
{
    Linear l;
    return linear_of(d, l) == DN_OK ? linear_forward_bytes(l) : kBad;
}

size_t dn_linear_backward_workspace_bytes(const dn_linear_desc *d)
{
    Linear l;
    return linear_of(d, l) == DN_OK ? l.bytes : kBad;
}

dn_status dn_linear_forward(const dn_linear_desc *d, const void *X_dev, const void *W_dev, const void *bias_dev,
                            const void *R_dev, void *Y_dev, void *Z_dev, void *workspace_dev, size_t workspace_bytes,
                            void *hip_stream)
{
    Linear l;
    dn_status s = linear_of(d, l);
    if (s != DN_OK) return s;
    if (!X_dev || !W_dev || !Y_dev || !multiples(d->type, X_dev, W_dev, bias_dev, R_dev, Y_dev, Z_dev)) return DN_ERR_INVALID_ARG;
    const int64_t e = size_of(d->type);
    ProductArgs a{};
    a.a[0] = a.a[1] = X_dev;
    a.b[0] = a.b[1] = W_dev;
    a.lda = l.d.ldx * e;
    a.ldb = l.d.ldw * e;
    a.M = d->rows;
    a.N = d->n_out;
    a.K = d->n_in;
    a.segments = 1;
    a.f.y = Y_dev;
    a.f.ldy = l.d.ldy;
    a.f.y2 = Z_dev;
    a.f.ldy2 = d->n_out;
    a.f.r = R_dev;
    a.f.ldr = l.d.ldr;
    a.f.bias = bias_dev;
    a.f.act = d->act;
    a.f.drop = l.drop;
    const bool direct = pieces(d->type, X_dev, l.d.ldx, d->n_in) && pieces(d->type, W_dev, l.d.ldw, d->n_in);
    const ProductPlan plan = plan_product(d->type, P_FWD, E_LINEAR, a.M, a.N, a.K, 1, direct, false);
    if ((s = workspace(plan.ws_bytes, workspace_dev, workspace_bytes)) != DN_OK) return s;
    a.ws = static_cast<float *>(workspace_dev);
    return device(launch_product(d->type, P_FWD, E_LINEAR, plan, a, (hipStream_t)hip_stream));
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
    if ((s = workspace(l.bytes, workspace_dev, workspace_bytes)) != DN_OK) return s;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t e = size_of(d->type);
    const void *delta = dY_dev;
    if (!l.plain) {
        MaskArgs m{};
        m.x = dY_dev;
        m.z = Z_dev;
        m.y = workspace_dev;
        m.ldx = l.d.ldy;
        m.ldz = d->n_out;
        m.ldy = l.ldd;
        m.rows = d->rows;
        m.cols = d->n_out;
        m.act = d->act;
        m.drop = l.drop;
        m.drop.scale = 1.f;   // the products' sums are multiplied by it
        if (launch_mask(d->type, m, stream) != hipSuccess) return DN_ERR_DEVICE;
        delta = workspace_dev;
    }
    float *part = reinterpret_cast<float *>(static_cast<char *>(workspace_dev) + l.delta);
    const bool direct_x = pieces(d->type, X_dev, l.d.ldx, d->n_in), direct_d = pieces(d->type, delta, l.ldd, d->n_out);
    if (dX_dev) {
        ProductArgs a{};
        a.a[0] = a.a[1] = delta;
        a.b[0] = a.b[1] = W_dev;
        a.lda = l.ldd * e;
        a.ldb = l.d.ldw * e;
        a.M = d->rows;
        a.N = d->n_in;
        a.K = d->n_out;
        a.segments = 1;
        a.ws = part;
        a.f.y = dX_dev;
        a.f.ldy = d->n_in;
        a.f.alpha = l.drop.scale;
        const ProductPlan plan = plan_product(d->type, P_DELTA, E_STORE, a.M, a.N, a.K, 1, direct_d && pieces(d->type, W_dev, l.d.ldw, d->n_in), false);
        if (launch_product(d->type, P_DELTA, E_STORE, plan, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    if (dW_dev) {
        ProductArgs a{};
        a.a[0] = a.a[1] = delta;
        a.b[0] = a.b[1] = X_dev;
        a.lda = l.ldd * e;
        a.ldb = l.d.ldx * e;
        a.M = d->n_out;
        a.N = d->n_in;
        a.K = d->rows;
        a.segments = 1;
        a.ws = part;
        a.f.y = dW_dev;
        a.f.ldy = d->n_in;
        a.f.sums = dbias_dev;
        a.f.f32_out = d->grad_type == DN_F32;
        a.f.alpha = l.drop.scale * d->grad_scale;
        const ProductPlan plan = plan_product(d->type, P_GRAD, E_STORE, a.M, a.N, a.K, 1, direct_d && direct_x, dbias_dev != nullptr);
        if (launch_product(d->type, P_GRAD, E_STORE, plan, a, stream) != hipSuccess) return DN_ERR_DEVICE;
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
    float *part = reinterpret_cast<float *>(static_cast<char *>(workspace_dev) + g.h);
    ProductArgs a{};
    a.a[0] = a.a[1] = X_dev;
    a.b[0] = Wg_dev;
    a.b[1] = Wu_dev;
    a.lda = g.d.ldx * e;
    a.ldb = d->d * e;
    a.M = d->rows;
    a.N = d->f;
    a.K = d->d;
    a.segments = 1;
    a.ws = part;
    a.f.y = workspace_dev;
    a.f.ldy = g.ldh;
    a.f.y2 = GU_dev;
    a.f.ldy2 = 2 * (int64_t)d->f;
    a.f.half = d->f;
    a.f.bias = bg_dev;
    a.f.bias2 = bu_dev;
    a.f.act = d->act;
    const bool direct = pieces(d->type, X_dev, g.d.ldx, d->d) && pieces(d->type, Wg_dev, d->d, d->d) && pieces(d->type, Wu_dev, d->d, d->d);
    ProductPlan plan = plan_product(d->type, P_FWD, E_GATED, a.M, a.N, a.K, 1, direct, false);
    if (launch_product(d->type, P_FWD, E_GATED, plan, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    ProductArgs b{};
    b.a[0] = b.a[1] = workspace_dev;
    b.b[0] = b.b[1] = Wd_dev;
    b.lda = g.ldh * e;
    b.ldb = d->f * e;
    b.M = d->rows;
    b.N = d->d;
    b.K = d->f;
    b.segments = 1;
    b.ws = part;
    b.f.y = Y_dev;
    b.f.ldy = g.d.ldy;
    b.f.r = R_dev;
    b.f.ldr = g.d.ldr;
    b.f.bias = bd_dev;
    b.f.drop = g.drop;
    plan = plan_product(d->type, P_FWD, E_LINEAR, b.M, b.N, b.K, 1, pieces(d->type, Wd_dev, d->f, d->f), false);
    return device(launch_product(d->type, P_FWD, E_LINEAR, plan, b, stream));
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
    float *part = reinterpret_cast<float *>(ws + g.h + g.dgu + g.dz);
    const bool f32_out = d->grad_type == DN_F32;

    // dZ without dropout's scale, by which the sums of the two products that read it are multiplied
    const void *dZ = dY_dev;
    int64_t ldz = g.d.ldy;
    if (g.drop.t) {
        MaskArgs m{};
        m.x = dY_dev;
        m.y = ws + g.h + g.dgu;
        m.ldx = g.d.ldy;
        m.ldy = ((int64_t)d->d + 7) / 8 * 8;
        m.rows = d->rows;
        m.cols = d->d;
        m.act = -1;
        m.drop = g.drop;
        m.drop.scale = 1.f;
        if (launch_mask(d->type, m, stream) != hipSuccess) return DN_ERR_DEVICE;
        dZ = m.y;
        ldz = m.ldy;
    }
    const bool direct_z = pieces(d->type, dZ, ldz, d->d), direct_f = f * e % 16 == 0;
    {   // dH, and from it dG, dU and H
        ProductArgs a{};
        a.a[0] = a.a[1] = dZ;
        a.b[0] = a.b[1] = Wd_dev;
        a.lda = ldz * e;
        a.ldb = f * e;
        a.M = d->rows;
        a.N = d->f;
        a.K = d->d;
        a.segments = 1;
        a.ws = part;
        a.f.y = dG;
        a.f.ldy = 2 * g.ldh;
        a.f.half_y = g.ldh;
        a.f.y2 = H;
        a.f.ldy2 = g.ldh;
        a.f.r = GU_dev;
        a.f.ldr = 2 * f;
        a.f.half = f;
        a.f.act = d->act;
        a.f.alpha = g.drop.scale;
        const ProductPlan plan = plan_product(d->type, P_DELTA, E_DGATED, a.M, a.N, a.K, 1, direct_z && pieces(d->type, Wd_dev, f, f), false);
        if (launch_product(d->type, P_DELTA, E_DGATED, plan, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    if (dX_dev) {
        ProductArgs a{};
        a.a[0] = dG;
        a.a[1] = dU;
        a.b[0] = Wg_dev;
        a.b[1] = Wu_dev;
        a.lda = 2 * g.ldh * e;
        a.ldb = d->d * e;
        a.M = d->rows;
        a.N = d->d;
        a.K = d->f;
        a.segments = 2;
        a.ws = part;
        a.f.y = dX_dev;
        a.f.ldy = d->d;
        const bool direct = direct_f && pieces(d->type, Wg_dev, d->d, d->d) && pieces(d->type, Wu_dev, d->d, d->d);
        const ProductPlan plan = plan_product(d->type, P_DELTA, E_STORE, a.M, a.N, a.K, 2, direct, false);
        if (launch_product(d->type, P_DELTA, E_STORE, plan, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    {   // dWg and dWu: the columns of dG, those up to ldh that no column of G has, and the columns of dU
        ProductArgs a{};
        a.a[0] = a.a[1] = dG;
        a.b[0] = a.b[1] = X_dev;
        a.lda = 2 * g.ldh * e;
        a.ldb = g.d.ldx * e;
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
        const ProductPlan plan = plan_product(d->type, P_GRAD, E_STORE, a.M, a.N, a.K, 1, pieces(d->type, X_dev, g.d.ldx, d->d), dbg_dev || dbu_dev);
        if (launch_product(d->type, P_GRAD, E_STORE, plan, a, stream) != hipSuccess) return DN_ERR_DEVICE;
    }
    ProductArgs a{};
    a.a[0] = a.a[1] = dZ;
    a.b[0] = a.b[1] = H;
    a.lda = ldz * e;
    a.ldb = g.ldh * e;
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
    const ProductPlan plan = plan_product(d->type, P_GRAD, E_STORE, a.M, a.N, a.K, 1, direct_z && direct_f, dbd_dev != nullptr);
    return device(launch_product(d->type, P_GRAD, E_STORE, plan, a, stream));
}

size_t dn_norm_backward_workspace_bytes(const dn_norm_desc *d)
{
    NormArgs a;
    return norm_of(d, a) == DN_OK ? up256(norm_backward_plan(a)) : kBad;
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
    a.post_w = post_w_dev;
    a.post_b = post_b_dev;
    a.pre_w = pre_w_dev;
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
    if ((s = workspace(up256(norm_backward_plan(a)), workspace_dev, workspace_bytes)) != DN_OK) return s;
    a.x = x_dev;
    a.b = b_dev;
    a.gate = gate_dev;
    a.post_w = post_w_dev;
    a.post_b = post_b_dev;
    a.pre_w = pre_w_dev;
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
    if (rows < 1 || cols < 1) return DN_ERR_SHAPE;
    if ((s = row_length(type, ldx, cols)) != DN_OK || (s = row_length(type, ldy, cols)) != DN_OK) return s;
    m.x = X_dev;
    m.y = Y_dev;
    m.ldx = ldx;
    m.ldy = ldy;
    m.rows = rows;
    m.cols = cols;
    m.act = -1;
    return device(launch_mask(type, m, (hipStream_t)hip_stream));
}

}  // extern "C"
