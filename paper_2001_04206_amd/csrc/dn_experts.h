// A block of experts: what its kernels and its host side share.  Internal; the entry points are in include/dn.h.
#pragma once

#include "dn_ffn.h"

namespace dn {

// The experts' products, one source per type: E_GATED of gathered rows, E_STORE or E_PAIR
// forward (Wd), E_DEXPERT, E_STORE or E_PAIR backward (dX; two
// segments) and E_STORE of an expert's terms (P_GRAD; operand `gathered`, 0 or 1, has rows of X or dY).  `tiles`: most tiles of rows that the lists can give (K_FEW: of sixteen).
hipError_t launch_experts_f32(Product p, Epilogue e, ProductKernel kernel, int gathered, ProductArgs a, int64_t tiles, hipStream_t s);
hipError_t launch_experts_f16(Product p, Epilogue e, ProductKernel kernel, int gathered, ProductArgs a, int64_t tiles, hipStream_t s);
hipError_t launch_experts_bf16(Product p, Epilogue e, ProductKernel kernel, int gathered, ProductArgs a, int64_t tiles, hipStream_t s);
int rows_of_tile(ProductKernel kernel);

// Few tokens: the last product and the sum over a row's choices in one launch
struct FewDown {
    const void *h, *w, *r;
    void *y;
    const float *weight;
    const int32_t *starts, *place;
    int64_t ldh, ldw, w_stride;   // bytes
    int64_t ldr, ldy;             // elements
    int32_t N, K, k, experts, pairs;
};
hipError_t launch_few_down_f32(const FewDown &a, int rows, hipStream_t s);
hipError_t launch_few_down_f16(const FewDown &a, int rows, hipStream_t s);
hipError_t launch_few_down_bf16(const FewDown &a, int rows, hipStream_t s);

}  // namespace dn
