// The experts' matrix products on fp32 operands.
#include "dn_experts_launch.h"

namespace dn {

hipError_t launch_experts_f32(Product p, Epilogue e, ProductKernel kernel, int gathered, ProductArgs a, int64_t tiles, hipStream_t s)
{
    return launch_experts<float>(p, e, kernel, gathered, a, tiles, s);
}

hipError_t launch_few_down_f32(const FewDown &a, int rows, hipStream_t s) { return few_down<float>(a, rows, s); }

}  // namespace dn
