// Grouped and 4-bit FC products in tiles of 32x32 outputs, for any size and alignment: the shape of the direct int8 kernel.
//
//   workgroup = KW waves, one tile of 32 rows of a group and 32 columns of its weights
//   wave w    = the 128-byte units w, w + KW, ... of the reduction: eight 1 KiB loads of whole 128-byte lines into registers, through
//               LDS of its own into MFMA operands, the next unit's loads in flight meanwhile; no barrier until the partial sums meet
//
// Rows outside a group re-read its last one and their sums are not stored; a row of x whose index is out of range counts as zeros.
// The partial sums of a tile are added in the order of the waves.
#include "q8_grouped_device.h"
#include "q8_load16.h"

namespace q8 {

constexpr int kPdUnit = 128, kPdSteps = kPdUnit / 32, kPdTile = 32;

__device__ __forceinline__ int pd_swizzle(int r) { return (r ^ (r >> 3)) & 7; }

__device__ __forceinline__ void pd_wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <class Op, int KW>
__global__ __launch_bounds__(KW * 64, 4) void product_direct_kernel(Product p, unsigned tiles_m)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kLoads = 2 * kPdTile / 8, kStage = 2 * kPdTile * kPdUnit;
    constexpr int kRow = kPdTile + 8;
    static_assert(kPdTile * kRow * 4 <= kStage, "the partial sums take the place of the staged operands");
    using Sum = typename Op::Sum;
    __shared__ __attribute__((aligned(16))) char lds[KW * kStage];
    __shared__ unsigned wave_amax[KW];
    Sum* part = reinterpret_cast<Sum*>(lds);

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, hi = lane >> 5, chunk = lane & 7, row8 = lane >> 3;
    const RowTile tile = RowTiles<kPdTile>(p).find(blockIdx.x % tiles_m);
    if (tile.rows <= 0) return;
    const int64_t n0 = (int64_t)(blockIdx.x / tiles_m) * kPdTile;
    const int pitch = (int)p.pitch;
    const int last_a = tile.rows - 1, last_b = (int)min((int64_t)kPdTile, p.N - n0) - 1;

    // x row of the tile's row r, or -1
    const auto x_row = [&](int r) -> int64_t {
        const int m = tile.row + min(r, last_a);
        if (!p.x_rows) return m;
        const int id = p.x_rows[m];
        return id >= 0 && id < p.x_count ? id : -1;
    };
    const uint8_t* row[kLoads];
    unsigned present = 0;  // bit i: load i of this lane is of a row that exists
#pragma unroll
    for (int i = 0; i < kLoads / 2; ++i) {
        const int64_t id = x_row(8 * i + row8);
        present |= (id >= 0 ? 1u : 0u) << i;
        row[i] = p.x + max(id, (int64_t)0) * pitch;
        row[kLoads / 2 + i] = p.w + ((int64_t)tile.group * p.N + n0 + min(8 * i + row8, last_b)) * pitch;
    }
    const int64_t groups = pitch / 64;  // 4-bit: groups of 128 elements in a row
    const int64_t xs_row = Op::kMx4 ? x_row(l32) : 0, ws_row = n0 + min(l32, last_b);

    char* stage = lds + wave * kStage;
    int put[kLoads], get_a[kPdSteps], get_b[kPdSteps];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) put[i] = (8 * i + row8) * kPdUnit + ((chunk ^ pd_swizzle(8 * i + row8)) << 4);
#pragma unroll
    for (int s = 0; s < kPdSteps; ++s) {
        get_a[s] = l32 * kPdUnit + (((4 * hi + s) ^ pd_swizzle(l32)) << 4);
        get_b[s] = (kPdTile + l32) * kPdUnit + (((4 * hi + s) ^ pd_swizzle(kPdTile + l32)) << 4);
    }

    typename Op::Acc acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0;

    const int full = pitch / kPdUnit, units = (pitch + kPdUnit - 1) / kPdUnit;
    v4i in[kLoads];
    int sa = 0, sb = 0;
    auto load_unit = [&](int u) {
        const int at = u * kPdUnit + 16 * chunk;
        if (u < full) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) in[i] = load16_any(reinterpret_cast<const int8_t*>(row[i]) + at);
        } else {  // the unit that the row's end cuts short
#pragma unroll
            for (int i = 0; i < kLoads; ++i) in[i] = load16_bounded(reinterpret_cast<const int8_t*>(row[i]) + at, pitch - at, pitch);
        }
        if constexpr (Op::kMx4) {
            const int64_t g = 2 * u + hi;
            sa = sb = 0;
            if (g < groups) {
                if (xs_row >= 0) sa = *reinterpret_cast<const int*>(p.xs + (g * p.x_count + xs_row) * 4);
                sb = *reinterpret_cast<const int*>(p.ws + (((int64_t)tile.group * groups + g) * p.N + ws_row) * 4);
            }
        }
    };
    if (wave < units) load_unit(wave);
    for (int u = wave; u < units; u += KW) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if (i < kLoads / 2 && !(present >> i & 1)) in[i] = v4i{0, 0, 0, 0};
            *reinterpret_cast<v4i*>(stage + put[i]) = in[i];
        }
        const int ua = sa, ub = sb;
        if (u + KW < units) load_unit(u + KW);
        pd_wave_order();
        v4i fa[kPdSteps], fb[kPdSteps];
#pragma unroll
        for (int s = 0; s < kPdSteps; ++s) {
            fa[s] = *reinterpret_cast<const v4i*>(stage + get_a[s]);
            fb[s] = *reinterpret_cast<const v4i*>(stage + get_b[s]);
        }
        acc = Op::template mfma<0>(fa[0], fb[0], acc, ua, ub);
        acc = Op::template mfma<1>(fa[1], fb[1], acc, ua, ub);
        acc = Op::template mfma<2>(fa[2], fb[2], acc, ua, ub);
        acc = Op::template mfma<3>(fa[3], fb[3], acc, ua, ub);
        pd_wave_order();
    }
    __syncthreads();  // the partial sums lie where other waves staged

    // Accumulator register e of lane (l32, hi) is row 8 (e / 4) + 4 hi + e % 4, column l32.
#pragma unroll
    for (int e = 0; e < 16; ++e) part[(wave * kPdTile + 8 * (e >> 2) + 4 * hi + (e & 3)) * kRow + l32] = acc[e];
    __syncthreads();

    unsigned amax = finish_tile<Op, KW>(p, tile, n0, part, kRow);
    if (p.flags & Q8_EPI_ABSMAX) {
        amax = wave_max_u32(amax);
        if (lane == 0) wave_amax[wave] = amax;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 1; w < KW; ++w) amax = max(amax, wave_amax[w]);
            unsigned* slot = reinterpret_cast<unsigned*>(p.out_amax);
            if (amax > __hip_atomic_load(slot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(slot, amax);
        }
    }
#endif
}

template <class Op>
static int launch(const Product& p, hipStream_t st)
{
    const int64_t tm = row_tiles(p.M, p.n_groups, kPdTile), tiles = tm * ((p.N + kPdTile - 1) / kPdTile);
    if (tiles >= (int64_t)1 << 26) return 1;  // a launch is limited to 2^32 threads
    const dim3 grid((unsigned)tiles);
#define Q8_PD_LAUNCH(KW) hipLaunchKernelGGL((product_direct_kernel<Op, KW>), grid, dim3(KW * 64), 0, st, p, (unsigned)tm)
    if (tiles <= 512)
        Q8_PD_LAUNCH(8);
    else if (tiles <= 1024)
        Q8_PD_LAUNCH(4);
    else if (tiles <= 2048)
        Q8_PD_LAUNCH(2);
    else
        Q8_PD_LAUNCH(1);
#undef Q8_PD_LAUNCH
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

int launch_product_direct(bool mx4, const Product& p, hipStream_t st) { return mx4 ? launch<OpMx4>(p, st) : launch<OpI8>(p, st); }

}  // namespace q8
