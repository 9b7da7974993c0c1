// Tiled products of bf16 operands.
#include "layers.h"
#include "product_dev.h"

namespace oz {
hipError_t launch_product_bf16(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    return launch_product_type<bf16>(a, plan, partial, st);
}
}  // namespace oz
