// Grouped and 4-bit products in 64x64 tiles, 4 waves, one stage buffer (see q8_grouped_kernel.h).
#include "q8_grouped_kernel.h"

namespace q8 {

int launch_product_64x64(bool mx4, const Product& p, hipStream_t st)
{
    return mx4 ? launch_product_tile<OpMx4, 64, 64, 2, 2, 1, 4, 5>(p, st) : launch_product_tile<OpI8, 64, 64, 2, 2, 1, 4, 5>(p, st);
}

}  // namespace q8
