// Grouped and 4-bit products in 256x128 tiles, 8 waves, one stage buffer (see q8_grouped_kernel.h).
#include "q8_grouped_kernel.h"

namespace q8 {

int launch_product_256x128_w8(bool mx4, const Product& p, hipStream_t st)
{
    return mx4 ? launch_product_tile<OpMx4, 256, 128, 4, 2, 1, 2, 2>(p, st) : launch_product_tile<OpI8, 256, 128, 4, 2, 1, 2, 2>(p, st);
}

}  // namespace q8
