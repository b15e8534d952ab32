// The gated block's backward products with an fp32 dX.
#include "gated_products.h"

namespace sbpi {
hipError_t launch_products_f32(const ProductsLaunch &l, hipStream_t s) {
    return launch_products<true>(l, s);
}
}  // namespace sbpi
