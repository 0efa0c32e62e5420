// FC products on 4-bit microscaled codes, and FC products whose rows belong to groups (experts) with weights of their own, on 4-bit
// or int8 codes:
//
//   y[r,n] = act( sum_k x[rows[r],k] w[g(r),n,k] + bias[g(r),n] )        g(r) the group of row r
//
// This file holds the choice of the kernel.
#include "q8.h"
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
// Long rows are those of 2 KiB of codes and more; times in us, the alternatives taken in turn.  Over 720 shapes the choice takes 1.5 % longer than the best.
//   1 (32x32, the reduction dealt out over the waves) up to 256 tiles (300 x 520 -> 1000, 320 of them, 5.5, 64x64 4.2), and up to 512 of long rows, whose serial
//     walk a larger tile cannot hide (64 x 4096 -> 1024 4.7 and 7.6; int8, 275 rows of 16 experts, 4096 -> 512 9.5 and 19.7; but 754 rows of 8 experts, 2048 ->
//     1024, about 900, 14.6 and 9.1).
//   5 (256x256) for long rows whose tiles leave less than a quarter of a round of the 256 units idle: it moves the fewest operand bytes, but a unit holds one at
//     a time and waits for the last round (4096 -> 1024 to bf16: 14336 rows, 224 tiles, 36.8 and 128x128 38.2; 24576 rows, 384, 66.9 and 56.4, of 16 experts 68.2 and
//     63.3; codes of normal numbers, on those of a layer behind a GELU within 2 % of that).  Rows have to be 4 KiB for several rounds (8192 x 8192 -> 4096 133 and 139;
//     8192 x 4096 -> 4096 78 and 73), 8 KiB for int8 (4096 x 16384 -> 4096 223 and 255; 14336 x 4096 -> 1024 64.0 and 64.3) and for fp32 outputs, whose stores
//     nothing covers (4096 x 16384 -> 4096 135 and 141; 4096 x 4096 -> 4096 45 and 40).
//   4 (128x128) from two tiles a unit on (8192 x 2048 -> 4096 to bf16 40.8, 64x128 51.9; 12288 x 1024 -> 4096 37 and 44.5), three where groups are smaller than a
//     tile (57 rows each of 128, int8, 768 -> 1024 23.3 and 25.4; but 29 rows each 17.9 and 16.9), of long rows from one and a half.
//   3 (64x128) against 2 (64x64): from two tiles a unit on (8192 rows of 16 experts, 512 -> 4096 24.5 and 32.4), unless rows are short and groups small (4809 rows
//     of 64, 768 -> 2048 17.8 and 17.2); and for short rows to 4-bit codes, of which its waves store 16 bytes a lane and the other's 8 (5330 rows of 64 experts,
//     1024 -> 512 6.4 and 7.5).
static int choose(bool mx4, const Product& p)
{
    const int64_t groups = p.group_rows ? (p.n_groups < p.M ? p.n_groups : p.M) : 0;  // of which half a tile each is left over
    const auto tiles = [&](int64_t rows, int64_t cols) { return ((p.M + rows - 1) / rows + groups / 2) * ((p.N + cols - 1) / cols); };
    const bool is_long = p.pitch >= 2048, small = p.M < 96 * groups;
    if (tiles(32, 32) <= (is_long ? 512 : 256)) return 1;
    const int64_t largest = tiles(256, 256), idle = -largest & 255;
    const int64_t least = !mx4 || p.y_type == Q8_TYPE_F32 ? 8192 : largest <= 256 ? 2048 : 4096;  // bytes of a row
    if (!small && idle < 64 && p.pitch >= least) return 5;
    if (p.M >= 48 * groups && tiles(128, 128) >= (is_long ? 384 : small ? 768 : 512)) return 4;
    if (!is_long && p.y_type == Q8_TYPE_MX4) return 3;
    return tiles(64, 128) >= 512 && (is_long || !small) ? 3 : 2;
}

int launch_product(bool mx4, const Product& p, hipStream_t st)
{
    int v = g_variant;
    if (v < 0 || v > 1 + (int)(sizeof(kTiles) / sizeof(kTiles[0]))) return 1;
    const bool automatic = v == 0;
    if (automatic) v = choose(mx4, p);
    // Rows of y too long for a tile's offsets may fit the ones of fewer rows.  So whether a launch is tiled does not hang on the tile, which depends on y's type.
    for (; v > 1; v = automatic ? v - 1 : 1)
        if (tile_eligible(p, kTiles[v - 2].rows)) return kTiles[v - 2].launch(mx4, p, st);
    return launch_product_direct(mx4, p, st);
}

}  // namespace q8
