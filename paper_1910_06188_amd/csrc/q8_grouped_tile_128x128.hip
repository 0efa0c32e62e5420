// Grouped and 4-bit products in 128x128 tiles, 4 waves, one stage buffer (see q8_grouped_kernel.h).
#include "q8_grouped_kernel.h"

namespace q8 {

int launch_product_128x128(bool mx4, const Product& p, hipStream_t st)
{
    return mx4 ? launch_product_tile<OpMx4, 128, 128, 2, 2, 1, 2, 4>(p, st) : launch_product_tile<OpI8, 128, 128, 2, 2, 1, 2, 4>(p, st);
}

}  // namespace q8
