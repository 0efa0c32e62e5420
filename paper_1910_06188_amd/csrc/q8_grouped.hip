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

// The kernel of a launch, by sizes alone: sums of a tiled kernel do not depend on its tile, so that outputs of every type are the same sums.
//   1 (32x32, the reduction dealt out over the waves) while tiles are few: up to 256 for short rows (1 x 1024 -> 4096 on 4-bit codes 3.8 us, 64x64 tiles 4.6;
//     300 x 520 -> 1000, 320 tiles, 6.0 and 4.5), up to 1024 for rows of 2 KiB and more, whose serial walk a larger tile cannot hide (64 x 4096 -> 1024 5.3 and
//     8.4; int8, 200 rows of 8 experts, 4096 -> 1024 12.8 and 20.0).
//   2 (64x64) for groups of few rows each, which leave most of a larger tile empty (64 rows of 64 experts, 1024 -> 4096 15.9 us, 64x128 17.7, 128x128 20.6).
//   5 (256x256) for long rows once every unit has a tile: it asks LDS for the least (4096^3 to bf16 41.5 us, 128x128 47.0; but 12288 x 4096 -> 1024, 192 tiles,
//     37.9 and 32.0).
//   4 (128x128) from three tiles a unit on, two for long rows (12288 x 1024 -> 4096 to bf16 49 us, 64x128 60; 2048 x 1024 -> 4096, two tiles a unit, 13.2
//     and 11.1), unless groups are so small that the rows left over count for more (128 rows a group, 1024 -> 2048: 37.0 and 29.6).
//   3 (64x128) in between, and 2 again where those are fewer than two a unit (2048 x 1024 -> 1024 6.5 us, 64x128 7.1).
static int choose(const Product& p)
{
    const int64_t groups = p.group_rows ? (p.n_groups < p.M ? p.n_groups : p.M) : 0;  // of which half a tile each is left over
    const auto tiles = [&](int64_t rows, int64_t cols) { return ((p.M + rows - 1) / rows + groups / 2) * ((p.N + cols - 1) / cols); };
    const bool is_long = p.pitch >= 2048;
    if (tiles(32, 32) <= 256 || (is_long && tiles(32, 32) <= 1024)) return 1;
    if (p.M < 96 * groups) return 2;
    if (is_long && tiles(256, 256) >= 256) return 5;
    if (p.M > 160 * groups && tiles(128, 128) >= (is_long ? 512 : 768)) return 4;
    return tiles(64, 128) >= 512 ? 3 : 2;
}

int launch_product(bool mx4, const Product& p, hipStream_t st)
{
    int v = g_variant;
    if (v < 0 || v > 1 + (int)(sizeof(kTiles) / sizeof(kTiles[0]))) return 1;
    if (v == 0) v = choose(p);
    if (v > 1 && tile_eligible(p, kTiles[v - 2].rows)) return kTiles[v - 2].launch(mx4, p, st);
    return launch_product_direct(mx4, p, st);
}

}  // namespace q8
