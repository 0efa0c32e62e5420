// Grouped and 4-bit products in 256x256 tiles, 8 waves, two stage buffers (see q8_grouped_kernel.h).
#include "q8_grouped_kernel.h"

namespace q8 {

int launch_product_256x256(bool mx4, const Product& p, hipStream_t st)
{
    return mx4 ? launch_product_tile<OpMx4, 256, 256, 2, 4, 2, 2, 1>(p, st) : launch_product_tile<OpI8, 256, 256, 2, 4, 2, 2, 1>(p, st);
}

}  // namespace q8
