// FC products on 4-bit microscaled codes, and FC products whose rows belong to groups (experts) with weights of their own, on 4-bit
// or int8 codes:
//
//   y[r,n] = act( sum_k x[rows[r],k] w[g(r),n,k] + bias[g(r),n] )        g(r) the group of row r
//
// This file holds the choice of the kernel.
#include "q8_launch.h"

namespace q8 {

int launch_product(bool mx4, const Product& p, hipStream_t st) { return launch_product_direct(mx4, p, st); }

}  // namespace q8
