// The experts' matrix products on bf16 operands.
#include "dn_experts_launch.h"

namespace dn {

hipError_t launch_experts_bf16(Product p, Epilogue e, ProductKernel kernel, int gathered, ProductArgs a, int64_t tiles, hipStream_t s)
{
    return launch_experts<bf16>(p, e, kernel, gathered, a, tiles, s);
}

hipError_t launch_few_down_bf16(const FewDown &a, int rows, hipStream_t s) { return few_down<bf16>(a, rows, s); }

}  // namespace dn
