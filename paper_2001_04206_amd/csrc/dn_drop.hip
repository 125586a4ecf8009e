// Dropout by itself, the first step of a layer's backward pass, and copies to 16-byte rows: one pass over memory, eight columns
// a thread.
//
// The mask is never stored: its numbers are computed again wherever it is needed.  A call of the generator is twenty 32 x 32
// bit products for eight elements.  Bound by memory: 16384 x 4096, bf16, 46 us (5.8 TB/s).
#include "dn_ffn.h"

namespace dn {
namespace {

template <class T>
__device__ __forceinline__ void mask8(const MaskArgs &a, uint32_t eights)
{
    // the workgroup's first eight elements by one uniform division, the thread's by a short one
    const uint64_t first = (uint64_t)blockIdx.x * 256;
    const uint32_t row0 = (uint32_t)(first / eights), c0 = (uint32_t)(first % eights) + threadIdx.x, more = c0 / eights;
    const int64_t m = (int64_t)row0 + more;
    const int n = (int)(c0 - more * eights) * 8, left = a.cols - n;
    if (m >= a.rows) return;
    float v[8];
    load8<T>(v, a.x, m * a.ldx + n, left);
    if (a.act > DN_ACT_LINEAR) {
        float z[8], f[8], df[8];
        load8<T>(z, a.z, m * a.ldz + n, left);
        act8<sizeof(T) == 2>(a.act, z, f, df);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= df[j];
    }
    if (a.drop.t) drop8(a.drop, (int)m, n, v);
    store8<T>(a.y, m * a.ldy + n, v, left + a.zeros);
}

template <class T>
__device__ __forceinline__ void pack8(const PackArgs &a, uint32_t block)
{
    const int64_t at = (int64_t)block * 256 + threadIdx.x;
    if (at >= a.groups) return;
    int k = 0;
    while (k + 1 < a.n && at >= a.m[k + 1].first) ++k;
    const auto &m = a.m[k];
    const uint32_t eights = ((uint32_t)m.cols + 7) / 8;
    const int64_t in = at - m.first;
    const int64_t row = (uint32_t)in / eights, n = (in - row * eights) * 8;   // one matrix has fewer than 2^32
    const auto v = get8<T>(m.x, row * m.ldx + n, (int)(m.cols - n));
    *reinterpret_cast<typename Eight<T>::type *>(static_cast<T *>(m.y) + (row * eights * 8 + n)) = v;
}

template <class T>
__global__ __launch_bounds__(256) void mask_kernel(const MaskArgs a, uint32_t eights)
{
    mask8<T>(a, eights);
}

template <class T>
__global__ __launch_bounds__(256) void pack_kernel(const PackArgs a, uint32_t first)
{
    pack8<T>(a, first + blockIdx.x);
}

// Both at once, on workgroups of their own: neither fills the chip for long.  1301 x 777 and 1301 x 1021 with 777 x 1021, fp32: 8 us,
// one after the other 5.4 and 5.7.
template <class T>
__global__ __launch_bounds__(256) void mask_pack_kernel(const MaskArgs a, uint32_t eights, const PackArgs p, uint32_t masks)
{
    if (blockIdx.x < masks) mask8<T>(a, eights);
    else pack8<T>(p, blockIdx.x - masks);
}

template <class T>
hipError_t run(const MaskArgs *a, const PackArgs &p, hipStream_t s)
{
    const uint32_t eights = a ? ((uint32_t)a->cols + 7) / 8 : 0;
    const unsigned masks = a ? (unsigned)(((uint64_t)a->rows * eights + 255) / 256) : 0, packs = (unsigned)((p.groups + 255) / 256);
    if (masks && packs && (uint64_t)masks + packs < 1u << 24) {   // fewer than 2^32 threads
        launch_kernel(mask_pack_kernel<T>, dim3(masks + packs), dim3(256), 0, s, *a, eights, p, masks);
        return hipGetLastError();
    }
    if (masks) launch_kernel(mask_kernel<T>, dim3(masks), dim3(256), 0, s, *a, eights);
    // the matrices together may take more threads than a launch can have
    constexpr unsigned most = 1u << 23;
    for (unsigned first = 0; first < packs; first += most)
        launch_kernel(pack_kernel<T>, dim3(packs - first < most ? packs - first : most), dim3(256), 0, s, p, first);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mask_pack(int type, const MaskArgs *a, const PackArgs &p, hipStream_t s)
{
    return type == DN_F32 ? run<float>(a, p, s) : type == DN_F16 ? run<f16>(a, p, s) : run<bf16>(a, p, s);
}

}  // namespace dn
