// Tiled products of operands in 8 bits, results in f32.
#include "layers.h"
#include "product_dev.h"

namespace oz {
hipError_t launch_product8_f32(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    return launch_product_type<int8_t, float>(a, plan, partial, st);
}
}  // namespace oz
