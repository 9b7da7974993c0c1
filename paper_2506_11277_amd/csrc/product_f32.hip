// Tiled products of binary32 operands.
#include "layers.h"
#include "product_dev.h"

namespace oz {
hipError_t launch_product_f32(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    return launch_product_type<float>(a, plan, partial, st);
}
}  // namespace oz
