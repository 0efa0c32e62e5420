// What the kernels of the grouped products share: the two kinds of operands, where a workgroup's rows are, and the epilogue.
#pragma once
#include "q8.h"
#include "q8_device.h"
#include "q8_epilogue.h"
#include "q8_launch.h"
#include "q8_mx4_device.h"

namespace q8 {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

// One MFMA takes 32 bytes of 32 rows of either operand, 16 bytes a lane: 32 int8 codes, or 64 4-bit codes of which a lane holds
// one block with its scale.  So both kinds move through memory, LDS and registers alike, in units of 128 bytes of a row, and only
// the instruction, the accumulator's type and the scales differ.
//
// A lane's 16 bytes of step s of a unit are chunk 4 (lane / 32) + s, not 2 s + lane / 32 as the instruction numbers them: a sum does
// not mind the order of its terms as long as both operands have the same one, and this way the four scales that a lane needs for a unit
// are the four bytes of one group's word, one for each step, which the instruction picks by a constant.
struct OpI8 {
    static constexpr bool kMx4 = false;
    using Acc = v16i;
    using Sum = int;
    template <int kStep>
    static __device__ __forceinline__ Acc mfma(v4i a, v4i b, Acc c, int, int)
    {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
    }
};
struct OpMx4 {
    static constexpr bool kMx4 = true;
    using Acc = v16f;
    using Sum = float;
    template <int kStep>
    static __device__ __forceinline__ Acc mfma(v4i a, v4i b, Acc c, int sa, int sb)
    {
        const v8i a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a8, b8, c, 4, 4, kStep, sa, kStep, sb);  // format 4: E2M1
    }
};

// Inclusive scan over the 64 lanes of a + b, at most `most` (< 2^31) and so never above 32 bits; truncated addition is associative.
template <int kCtrl, int kRowMask>
__device__ __forceinline__ unsigned dpp_add_most(unsigned v, unsigned most)
{
    return min(v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, kRowMask, 0xf, true), most);
}
__device__ __forceinline__ unsigned wave_scan_most(unsigned v, unsigned most)
{
    v = dpp_add_most<0x111, 0xf>(v, most);  // row_shr:1
    v = dpp_add_most<0x112, 0xf>(v, most);
    v = dpp_add_most<0x114, 0xf>(v, most);
    v = dpp_add_most<0x118, 0xf>(v, most);
    v = dpp_add_most<0x142, 0xa>(v, most);  // row_bcast:15
    v = dpp_add_most<0x143, 0xc>(v, most);  // row_bcast:31
    return v;
}

// Rows are dealt out to groups in order and only as far as y goes, and a negative number of rows counts as none, so that whatever
// group_rows holds no two groups share a row and none leaves y.  Every wave works this out by itself: the counts of 64 groups a pass, one
// a lane, and two scans in the vector ALU.
struct GroupPass {
    unsigned start, upto;   // this lane's group: first row, first row behind it
    unsigned tiles, ends;   // its tiles of kRows rows, and those of this pass up to its last
};
template <int kRows>
__device__ __forceinline__ GroupPass group_pass(const int32_t* __restrict__ group_rows, int n_groups, unsigned M, int g0, unsigned before)
{
    const int lane = threadIdx.x & 63;
    const unsigned n = g0 + lane < n_groups ? min((unsigned)max(group_rows[g0 + lane], 0), M) : 0u;
    GroupPass q;
    q.upto = min(before + wave_scan_most(n, M), M);
    const unsigned prev = (unsigned)__shfl_up((int)q.upto, 1);
    q.start = lane ? prev : before;
    q.tiles = (q.upto - q.start + kRows - 1) / kRows;
    q.ends = wave_scan_most(q.tiles, 0x7fffffffu);
    return q;
}

// The tiles of kRows rows that stay inside a group: how many there are, and of the t-th its group, its first row of y and its rows (0: there is no
// such tile).  The first 64 groups are looked at once for both.
struct RowTile {
    int group, row, rows;
};
template <int kRows>
struct RowTiles {
    const int32_t* group_rows;
    int n_groups;
    unsigned M, count;
    GroupPass first;
    __device__ __forceinline__ explicit RowTiles(const Product& p) : group_rows(p.group_rows), n_groups(p.n_groups), M((unsigned)p.M)
    {
        if (!group_rows) {
            count = (M + kRows - 1) / kRows;
            return;
        }
        first = group_pass<kRows>(group_rows, n_groups, M, 0, 0);
        count = (unsigned)__builtin_amdgcn_readlane((int)first.ends, 63);
        unsigned before = (unsigned)__builtin_amdgcn_readlane((int)first.upto, 63);  // rows of the groups already passed
        for (int g0 = 64; g0 < n_groups; g0 += 64) {
            const GroupPass q = group_pass<kRows>(group_rows, n_groups, M, g0, before);
            count += (unsigned)__builtin_amdgcn_readlane((int)q.ends, 63);
            before = (unsigned)__builtin_amdgcn_readlane((int)q.upto, 63);
        }
    }
    __device__ __forceinline__ RowTile find(unsigned t) const
    {
        if (!group_rows) {
            const int row = (int)(t * kRows);
            return RowTile{0, row, min(kRows, (int)M - row)};
        }
        GroupPass q = first;
        for (int g0 = 0;;) {
            const unsigned long long behind = __ballot(t < q.ends);
            if (behind) {
                const int l = __builtin_ctzll(behind);
                const unsigned before = (unsigned)__builtin_amdgcn_readlane((int)(q.ends - q.tiles), l);
                const int row = __builtin_amdgcn_readlane((int)q.start, l) + (int)((t - before) * kRows);
                return RowTile{g0 + l, row, min(kRows, __builtin_amdgcn_readlane((int)q.upto, l) - row)};
            }
            g0 += 64;
            if (g0 >= n_groups) return RowTile{0, 0, 0};
            t -= (unsigned)__builtin_amdgcn_readlane((int)q.ends, 63);
            q = group_pass<kRows>(group_rows, n_groups, M, g0, (unsigned)__builtin_amdgcn_readlane((int)q.upto, 63));
        }
    }
};

// Per-column constants and the value of an output.
struct ProductColumn {
    int bq;       // int8: quantized bias
    float r, b;   // int8: 1 / (S_x S_W); 4-bit: the bias
};
template <class Op>
__device__ __forceinline__ ProductColumn product_column(const Product& p, int group, int64_t n, float sx)
{
    const float b = p.bias ? p.bias[(int64_t)group * p.N + n] : 0.0f;
    if constexpr (Op::kMx4) return ProductColumn{0, 1.0f, b};
    const float sw = p.sw[group];
    return ProductColumn{p.bias ? quantize_bias(b, sx, sw) : 0, dequant_factor(sx, sw), 0.0f};
}
template <class Op>
__device__ __forceinline__ float product_value(typename Op::Sum sum, const ProductColumn& c)
{
    if constexpr (Op::kMx4)
        return __fadd_rn(sum, c.b);
    else
        return (float)(sum + c.bq) * c.r;
}

template <class Op>
__device__ __forceinline__ float product_gelu(float v)
{
    return gelu_erf<Op::kMx4>(v);
}

// Maximum over each half of 32 lanes.
__device__ __forceinline__ unsigned half_wave_max_u32(unsigned v)
{
    v = quad_max_u32(v);
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));  // row_half_mirror
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));  // row_mirror
    return max(v, (unsigned)__shfl_xor((int)v, 16));
}

// The epilogue of a 32x32 tile whose KW partial sums, one of each wave, lie in LDS at part[(w * 32 + row) * pitch + column].  They are added in the order
// of the waves.  A thread keeps its column, and a row's 32 lanes stay together.  Returns the bits of the largest |y| of this thread.
template <class Op, int KW>
__device__ __forceinline__ unsigned finish_tile(const Product& p, const RowTile& tile, int64_t n0, const typename Op::Sum* part, int pitch)
{
    const int l32 = threadIdx.x & 31;
    const int64_t n = n0 + l32;
    const bool gelu = p.flags & Q8_EPI_GELU, requant = p.flags & Q8_EPI_REQUANT;
    unsigned amax = 0;
    if (n >= p.N) return amax;
    const float sx = Op::kMx4 ? 0.0f : p.sx[0], next_scale = requant ? p.next_scale[0] : 0.0f;
    const ProductColumn c = product_column<Op>(p, tile.group, n, sx);
    for (int r = threadIdx.x / 32; r < tile.rows; r += KW * 2) {
        typename Op::Sum sum = part[r * pitch + l32];
#pragma unroll
        for (int w = 1; w < KW; ++w) sum += part[(w * 32 + r) * pitch + l32];
        float y = product_value<Op>(sum, c);
        if (gelu) y = product_gelu<Op>(y);
        const int64_t m = tile.row + r, at = m * p.N + n;
        if (p.y_type == Q8_TYPE_MX4) {
            const unsigned byte = mx4_scale_byte(half_wave_max_u32(f32_abs_bits(y)));
            const float next = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), 0xB1, 0xf, 0xf, true));
            const unsigned code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, y, next, mx4_scale(byte), 0);
            if (l32 % 2 == 0) static_cast<uint8_t*>(p.y)[at / 2] = byte == kMxNan ? 0 : (uint8_t)code;
            if (l32 == 0) p.y_scales[((n / kMxGroup) * p.M + m) * 4 + (n % kMxGroup) / 32] = (uint8_t)byte;
        } else if (p.y_type == Q8_TYPE_BF16) {
            static_cast<unsigned short*>(p.y)[at] = f32_to_bf16(y);
        } else if (requant) {
            static_cast<int8_t*>(p.y)[at] = (int8_t)quantize_code(y, next_scale);
        } else {
            static_cast<float*>(p.y)[at] = y;
        }
        amax = max(amax, f32_abs_bits(y));
    }
    return amax;
}

}  // namespace q8
