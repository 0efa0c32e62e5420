// FC products on 4-bit microscaled codes, and FC products whose rows belong to groups (experts) with weights of their own, on 4-bit
// or int8 codes:
//
//   y[r,n] = act( sum_k x[rows[r],k] w[g(r),n,k] + bias[g(r),n] )        g(r) the group of row r
//
// This file holds the choice of the kernel.
#include "q8_launch.h"

namespace q8 {

int launch_product_64x64(bool, const Product&, hipStream_t);
int launch_product_64x128(bool, const Product&, hipStream_t);
int launch_product_128x128(bool, const Product&, hipStream_t);
int launch_product_256x256(bool, const Product&, hipStream_t);

static const struct {
    int (*launch)(bool, const Product&, hipStream_t);
    int rows;
} kTiles[] = {
    {launch_product_64x64, 64},
    {launch_product_64x128, 64},
    {launch_product_128x128, 128},
    {launch_product_256x256, 256}};

static int g_variant = 0;
void set_product_variant(int v) { g_variant = v; }

// Whether the tiled kernels take the sizes and addresses: whole 16-byte vectors, and 32-bit offsets into a tile's rows and, where rows of x are
// picked by index, into the whole of x.
static bool tile_eligible(const Product& p, int64_t rows)
{
    const int64_t most = (int64_t)1 << 31;
    return p.pitch % 16 == 0 && reinterpret_cast<uintptr_t>(p.x) % 16 == 0 && reinterpret_cast<uintptr_t>(p.w) % 16 == 0 && rows * p.N * 4 < most &&
           256 * p.pitch < most && (!p.x_rows || (p.x_count * p.pitch < most && p.x_count * 4 < most));
}

int launch_product(bool mx4, const Product& p, hipStream_t st)
{
    int v = g_variant;
    if (v < 0 || v > 1 + (int)(sizeof(kTiles) / sizeof(kTiles[0]))) return 1;
    if (v == 0) v = p.M / p.n_groups >= 64 ? 4 : 1;
    if (v > 1 && tile_eligible(p, kTiles[v - 2].rows)) return kTiles[v - 2].launch(mx4, p, st);
    return launch_product_direct(mx4, p, st);
}

}  // namespace q8
