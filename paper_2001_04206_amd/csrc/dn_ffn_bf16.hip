// Matrix products of the residual feed-forward block on bf16 operands.
#include "dn_ffn_launch.h"

namespace dn {

hipError_t launch_product_bf16(Product p, Epilogue e, const ProductPlan &plan, ProductArgs a, hipStream_t s)
{
    return launch_product<bf16>(p, e, plan, a, s);
}

}  // namespace dn
