// Tiled products of operands in 8 bits, results in bf16.
#include "layers.h"
#include "product_dev.h"

namespace oz {
hipError_t launch_product8_bf16(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    return launch_product_type<int8_t, bf16>(a, plan, partial, st);
}
}  // namespace oz
