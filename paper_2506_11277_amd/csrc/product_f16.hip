// Tiled products of f16 operands.
#include "layers.h"
#include "product_dev.h"

namespace oz {
hipError_t launch_product_f16(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    return launch_product_type<f16>(a, plan, partial, st);
}
hipError_t launch_pair_f16(const Product &dx, const Product &dw, const BiasGrad &db, int tile, hipStream_t st)
{
    return launch_pair_type<f16>(dx, dw, db, tile, st);
}
}  // namespace oz
