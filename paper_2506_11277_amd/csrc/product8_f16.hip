// Tiled products of operands in 8 bits, results in f16.
#include "layers.h"
#include "product_dev.h"

namespace oz {
hipError_t launch_product8_f16(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    return launch_product_type<int8_t, f16>(a, plan, partial, st);
}
}  // namespace oz
