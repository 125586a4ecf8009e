// Dropout by itself, and the first step of a layer's backward pass: one pass over memory, eight columns a thread.
//
// The mask is never stored: its numbers are computed again wherever it is needed.  A call of the generator is twenty 32 x 32
// bit products for eight elements.
#include "dn_ffn.h"

namespace dn {
namespace {

template <class T>
__global__ __launch_bounds__(256) void mask_kernel(const MaskArgs a, uint32_t eights)
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
        float z[8];
        load8<T>(z, a.z, m * a.ldz + n, left);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float f, df;
            act_both<sizeof(T) == 2>(a.act, z[j], f, df);
            v[j] *= df;
        }
    }
    if (a.drop.t) drop8(a.drop, (int)m, n, v);
    store8<T>(a.y, m * a.ldy + n, v, left);
}

template <class T>
hipError_t run(const MaskArgs &a, hipStream_t s)
{
    const uint32_t eights = ((uint32_t)a.cols + 7) / 8;
    const uint64_t blocks = ((uint64_t)a.rows * eights + 255) / 256;
    launch_kernel(mask_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, s, a, eights);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mask(int type, const MaskArgs &a, hipStream_t s)
{
    return type == DN_F32 ? run<float>(a, s) : type == DN_F16 ? run<f16>(a, s) : run<bf16>(a, s);
}

}  // namespace dn
