// The gated block's backward products with a bf16 dX.
#include "gated_products.h"

namespace sbpi {
hipError_t launch_products_bf16(const ProductsLaunch &l, hipStream_t s) {
    return launch_products<false>(l, s);
}
}  // namespace sbpi
