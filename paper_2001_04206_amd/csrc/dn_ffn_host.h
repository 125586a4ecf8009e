// What the host sides of the block's operators and of the experts' share: checks of arguments, and copies of operands.
#pragma once

#include <math.h>

#include "dn_ffn.h"

namespace dn {

constexpr int64_t kRowBytes = (int64_t)8 << 20;   // a tile's 32-bit offsets hold 255 rows of this
constexpr size_t kBad = (size_t)-1;

inline int64_t size_of(int type) { return type == DN_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == DN_F32 || type == DN_F16 || type == DN_BF16; }
inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

inline hipError_t launch_product(int type, Product p, Epilogue e, const ProductPlan &plan, const ProductArgs &a, hipStream_t s)
{
    return type == DN_F32 ? launch_product_f32(p, e, plan, a, s)
           : type == DN_F16 ? launch_product_f16(p, e, plan, a, s) : launch_product_bf16(p, e, plan, a, s);
}

// sixteen-byte pieces: rows of `n` elements `ld` apart from p on
inline bool pieces(int type, const void *p, int64_t ld, int64_t n)
{
    const int64_t e = size_of(type);
    return ((uintptr_t)p | (uintptr_t)(ld * e) | (uintptr_t)(n * e)) % 16 == 0;
}

inline dn_status drop_of(float p, uint64_t seed, uint64_t offset, Dropout &d)
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
inline dn_status row_length(int type, int64_t &ld, int64_t n)
{
    if (ld == 0) ld = n;
    return ld < n || ld * size_of(type) > kRowBytes ? DN_ERR_SHAPE : DN_OK;
}
// more threads than a launch can have: one for eight columns, or 512 for a tile, 64 x 64 the smallest one
inline bool too_many(int64_t rows, int64_t cols)
{
    constexpr int64_t kThreads = (int64_t)1 << 32;
    return rows * ((cols + 7) / 8) >= kThreads || (rows + 63) / 64 * ((cols + 63) / 64) >= kThreads / 512;
}
inline dn_status common(int type, int grad_type, int act, int32_t rows, int32_t n, int32_t m, float grad_scale)
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

inline dn_status workspace(size_t need, const void *ws, size_t bytes)
{
    if (need == 0) return DN_OK;
    if (!ws || (uintptr_t)ws % 256) return DN_ERR_INVALID_ARG;
    return bytes < need ? DN_ERR_SHAPE : DN_OK;
}
// Operands of tiles: those whose rows are not in sixteen-byte pieces are copied to the workspace, from `at` on.
inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
inline size_t packed_bytes(int type, int64_t rows, int64_t cols) { return up256((size_t)rows * (size_t)(up8(cols) * size_of(type))); }
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
inline void operand_a(ProductArgs &a, const Packer::Rows &r)
{
    a.a[0] = a.a[1] = r.p;
    a.lda = r.ld;
    a.a_ext = r.ext;
}
inline void operand_b(ProductArgs &a, const Packer::Rows &r)
{
    a.b[0] = a.b[1] = r.p;
    a.ldb = r.ld;
    a.b_ext = r.ext;
}

inline dn_status device(hipError_t e) { return e == hipSuccess ? DN_OK : DN_ERR_DEVICE; }

}  // namespace dn
