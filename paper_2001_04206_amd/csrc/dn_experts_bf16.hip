// The experts' matrix products on bf16 operands.
#include "dn_experts_launch.h"

namespace dn {

hipError_t launch_experts_bf16(Product p, Epilogue e, ProductKernel kernel, int gathered, ProductArgs a, int64_t tiles, hipStream_t s)
{
    return launch_experts<bf16>(p, e, kernel, gathered, a, tiles, s);
}

}  // namespace dn
