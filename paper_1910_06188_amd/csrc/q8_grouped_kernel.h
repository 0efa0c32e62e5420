// Tiled kernel of the grouped and 4-bit FC products, gfx950.  Included by one translation unit per tile shape (q8_grouped_tile_*.hip).
//
// A workgroup owns BM rows of one group and BN columns of the group's weights.  It walks the reduction in stages of 128 bytes a row
// (128 int8 codes, 256 4-bit ones), loaded straight into LDS by 16 bytes a lane, swizzled so that the fragment reads of the MFMAs
// are free of bank conflicts.  The scales of a stage (4-bit: two words a row) come into LDS with it, four bytes a lane.  kSlots stage
// buffers: one (load, wait, multiply; other workgroups of the unit fill the gaps) or two (the next stage loads under this one's MFMAs).
//
// Loads and stores go through buffer descriptors whose bounds checks take the place of branches: a lane whose row of x does not exist, or whose
// 16 bytes lie behind the end of a row, is given an offset out of range and reads zeros; outputs outside the tile's rows and columns are dropped.
#pragma once
#include "q8_gemm_kernel.h"
#include "q8_grouped_device.h"

namespace q8 {

constexpr unsigned kOutOfRange = 0x80000000u;  // above the extent of every descriptor here

// 4 bytes per lane from a buffer straight into LDS: lane l lands at lds_addr + 4 l.
__device__ __forceinline__ void lds_dma4(v4i rsrc, unsigned voff, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(lds_addr), "v"(voff), "s"(rsrc) : "memory");
}

// kOut: the type of y.  For 4-bit outputs the MFMA's operands change places, so that a lane holds one row and 16 columns of a 32x32
// block, and a block of the format -- 32 neighbours of a row -- is two lanes'.
template <class Op, int BM, int BN, int WGM, int WGN, int kSlots, int kWgs, int kOut>
__global__ __launch_bounds__(WGM* WGN * 64, kWgs* WGM* WGN / 4) void product_tile_kernel(Product p, unsigned tiles_n, unsigned group_m)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool kSwap = kOut == Q8_TYPE_MX4;
    constexpr int NW = WGM * WGN;
    constexpr int TM = BM / WGM, TN = BN / WGN, FM = TM / 32, FN = TN / 32;
    constexpr int A_BYTES = BM * kBK, B_BYTES = BN * kBK, OPERANDS = A_BYTES + B_BYTES;
    constexpr int SCALES = Op::kMx4 ? (BM + BN) * 8 : 0, SLOT = OPERANDS + SCALES;  // scales: [A | B][group of the stage][row]
    constexpr int A_LOADS = BM / 8 / NW, B_LOADS = BN / 8 / NW;
    constexpr int S_UNITS = Op::kMx4 ? (BM + BN) / 32 : 0, S_LOADS = (S_UNITS + NW - 1) / NW;  // 64 rows of one group each
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "tile rows must split over the waves");
    static_assert(TM % 32 == 0 && TN % 32 == 0 && BM % 64 == 0 && BN % 64 == 0, "whole MFMA blocks and whole scale loads");
    static_assert(kSlots == 1 || kSlots == 2, "the waits below are for all loads");
    static_assert(kWgs * kSlots * SLOT <= 160 * 1024, "LDS is 160 KiB per compute unit");
    __shared__ __attribute__((aligned(1024))) char lds[kSlots * SLOT];

    const int lane = threadIdx.x & 63, l32 = lane & 31, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned lds_base = (unsigned)(size_t)(lds_ptr_t)lds;

    // The launch has room for every group ending inside a tile; the tiles that there are go to the XCDs in equal, contiguous shares.
    const unsigned tiles_m = count_row_tiles<BM>(p.group_rows, p.n_groups, (int)p.M), tiles = tiles_m * tiles_n;
    if (blockIdx.x >= tiles) return;
    const int pid = tile_of_workgroup(xcd_remap((int)blockIdx.x, (int)tiles), (int)tiles_m, (int)tiles_n, (int)group_m);
    const RowTile tile = find_row_tile<BM>(p.group_rows, p.n_groups, (int)p.M, (unsigned)pid / tiles_n);
    const int n0 = (int)((unsigned)pid % tiles_n) * BN;
    const int N = (int)p.N, pitch = (int)p.pitch;
    const int last_a = tile.rows - 1, last_b = min(BN, N - n0) - 1;

    // Row of the x descriptor for the tile's row r: its place among the tile's rows, or in the whole of x.
    const auto x_row = [&](int r) -> int {
        const int m = min(r, last_a);
        if (!p.x_rows) return m;
        const int id = p.x_rows[tile.row + m];
        return id >= 0 && id < (int)p.x_count ? id : -1;
    };
    const int64_t x_first = p.x_rows ? 0 : tile.row;
    const unsigned x_extent = p.x_rows ? (unsigned)p.x_count : (unsigned)tile.rows;
    const uint8_t* Xt = p.x + x_first * pitch;
    const uint8_t* Wt = p.w + ((int64_t)tile.group * N + n0) * pitch;
    unsigned a_off[A_LOADS], b_off[B_LOADS];
    const int chunk = lane & 7, row8 = lane >> 3;
#pragma unroll
    for (int i = 0; i < A_LOADS; ++i) {
        const int r = (wave * A_LOADS + i) * 8 + row8, id = x_row(r);
        a_off[i] = id < 0 ? kOutOfRange : (unsigned)id * (unsigned)pitch + (unsigned)((chunk ^ swizzle_of_row(r)) * 16);
    }
#pragma unroll
    for (int i = 0; i < B_LOADS; ++i) {
        const int r = (wave * B_LOADS + i) * 8 + row8;
        b_off[i] = (unsigned)min(r, last_b) * (unsigned)pitch + (unsigned)((chunk ^ swizzle_of_row(r)) * 16);
    }
    // The scale loads of this wave: which operand, which group of the stage, which 64 rows.
    unsigned s_off[S_LOADS ? S_LOADS : 1];
    const int groups = pitch / 64;
    if constexpr (Op::kMx4) {
#pragma unroll
        for (int i = 0; i < S_LOADS; ++i) {
            const int u = wave + i * NW;
            if (u < BM / 32) {
                const int id = x_row(u % (BM / 64) * 64 + lane);
                s_off[i] = id < 0 ? kOutOfRange : (unsigned)id * 4u;
            } else {
                s_off[i] = (unsigned)min((u - BM / 32) % (BN / 64) * 64 + lane, last_b) * 4u;
            }
        }
    }

    const int KT = (pitch + kBK - 1) / kBK;
    const v4i qa = make_rsrc(Xt, x_extent * (unsigned)pitch), qb = make_rsrc(Wt, (unsigned)(last_b + 1) * (unsigned)pitch);
    auto load_stage = [&](int kt, int slot) {
        const unsigned koff = (unsigned)kt * kBK, dst = lds_base + (unsigned)(slot * SLOT);
        const int left = pitch - kt * kBK;  // bytes of the rows from this stage on
        if (left >= kBK) {
#pragma unroll
            for (int i = 0; i < A_LOADS; ++i) lds_dma16_first(qa, a_off[i], koff, dst + (wave * A_LOADS + i) * 1024);
#pragma unroll
            for (int i = 0; i < B_LOADS; ++i) lds_dma16_first(qb, b_off[i], koff, dst + A_BYTES + (wave * B_LOADS + i) * 1024);
        } else {  // rows end inside the stage (after a whole number of 16 bytes)
#pragma unroll
            for (int i = 0; i < A_LOADS; ++i) {
                const int c = (chunk ^ swizzle_of_row((wave * A_LOADS + i) * 8 + row8)) * 16;
                lds_dma16_first(qa, c < left ? a_off[i] : kOutOfRange, koff, dst + (wave * A_LOADS + i) * 1024);
            }
#pragma unroll
            for (int i = 0; i < B_LOADS; ++i) {
                const int c = (chunk ^ swizzle_of_row((wave * B_LOADS + i) * 8 + row8)) * 16;
                lds_dma16_first(qb, c < left ? b_off[i] : kOutOfRange, koff, dst + A_BYTES + (wave * B_LOADS + i) * 1024);
            }
        }
        if constexpr (Op::kMx4) {
#pragma unroll
            for (int i = 0; i < S_LOADS; ++i) {
                const int u = wave + i * NW;
                if (u < BM / 32) {
                    const int g = 2 * kt + u / (BM / 64);
                    lds_dma4(make_rsrc(p.xs + ((int64_t)g * p.x_count + x_first) * 4, g < groups ? x_extent * 4u : 0u), s_off[i], dst + OPERANDS + u * 256);
                } else if (u < S_UNITS) {
                    const int g = 2 * kt + (u - BM / 32) / (BN / 64);
                    lds_dma4(make_rsrc(p.ws + (((int64_t)tile.group * groups + g) * N + n0) * 4, g < groups ? (unsigned)(last_b + 1) * 4u : 0u), s_off[i],
                             dst + OPERANDS + u * 256);
                }
            }
        }
    };

    const int wm = wave / WGN, wn = wave % WGN;
    int a_row[FM], b_row[FN], a_sw[FM], b_sw[FN];
#pragma unroll
    for (int f = 0; f < FM; ++f) {
        const int r = wm * TM + f * 32 + l32;
        a_row[f] = r * kBK;
        a_sw[f] = swizzle_of_row(r);
    }
#pragma unroll
    for (int f = 0; f < FN; ++f) {
        const int r = wn * TN + f * 32 + l32;
        b_row[f] = A_BYTES + r * kBK;
        b_sw[f] = swizzle_of_row(r);
    }
    const int a_sc = OPERANDS + (hi * BM + wm * TM + l32) * 4, b_sc = OPERANDS + BM * 8 + (hi * BN + wn * TN + l32) * 4;

    typename Op::Acc acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

    if constexpr (kSlots == 2)
        if (KT) load_stage(0, 0);
    for (int kt = 0; kt < KT; ++kt) {
        if constexpr (kSlots == 1) {
            if (kt) {  // every wave has read the last stage
                __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
                __syncthreads();
            }
            load_stage(kt, 0);
            __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
            __syncthreads();
        } else {
            // own loads of stage kt have landed, own reads of stage kt - 1 are complete; its slot is free behind the barrier
            __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
            __syncthreads();
            if (kt + 1 < KT) load_stage(kt + 1, (kt + 1) & 1);
        }
        const char* stage = lds + (kSlots == 2 ? (kt & 1) * SLOT : 0);
        int sa[FM], sb[FN];
        if constexpr (Op::kMx4) {
#pragma unroll
            for (int f = 0; f < FM; ++f) sa[f] = *reinterpret_cast<const int*>(stage + a_sc + f * 128);
#pragma unroll
            for (int f = 0; f < FN; ++f) sb[f] = *reinterpret_cast<const int*>(stage + b_sc + f * 128);
        }
        v4i fa[2][FM], fb[2][FN];
        auto read_step = [&](int ks) {
#pragma unroll
            for (int f = 0; f < FM; ++f) fa[ks & 1][f] = *reinterpret_cast<const v4i*>(stage + a_row[f] + (((4 * hi + ks) ^ a_sw[f]) << 4));
#pragma unroll
            for (int f = 0; f < FN; ++f) fb[ks & 1][f] = *reinterpret_cast<const v4i*>(stage + b_row[f] + (((4 * hi + ks) ^ b_sw[f]) << 4));
        };
        read_step(0);
        static_for<0, kKS>([&](auto kc) {
            constexpr int ks = decltype(kc)::value;
            if constexpr (ks + 1 < kKS) read_step(ks + 1);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    if constexpr (kSwap)
                        acc[i][j] = Op::template mfma<ks>(fb[ks & 1][j], fa[ks & 1][i], acc[i][j], Op::kMx4 ? sb[j] : 0, Op::kMx4 ? sa[i] : 0);
                    else
                        acc[i][j] = Op::template mfma<ks>(fa[ks & 1][i], fb[ks & 1][j], acc[i][j], Op::kMx4 ? sa[i] : 0, Op::kMx4 ? sb[j] : 0);
                }
        });
    }

    // Epilogue.  Accumulator register e of lane l is row 8 (e / 4) + 4 (l / 32) + e % 4 and column l % 32 of its block (kSwap: the other way round).
    const bool gelu = p.flags & Q8_EPI_GELU;
    constexpr int kSize = kOut == Q8_TYPE_F32 ? 4 : kOut == Q8_TYPE_BF16 ? 2 : 1;
    if constexpr (kSwap) {
        const int row_bytes = N / 2;
        const __amdgpu_buffer_rsrc_t ry = __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(p.y) + (int64_t)tile.row * row_bytes, 0, tile.rows * row_bytes, 0x00020000);
        const float* bias = p.bias ? p.bias + (int64_t)tile.group * N : nullptr;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int m = wm * TM + i * 32 + l32;
            const int at = m < tile.rows ? m * row_bytes + 8 * hi : (int)kOutOfRange;
            unsigned bytes = 0;
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int nb = n0 + wn * TN + j * 32;
                if (nb >= N) break;  // columns come in whole groups of 128
                float v[16];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 b = bias ? *reinterpret_cast<const float4*>(bias + nb + 8 * q + 4 * hi) : float4{0, 0, 0, 0};
                    v[4 * q] = __fadd_rn(acc[i][j][4 * q], b.x), v[4 * q + 1] = __fadd_rn(acc[i][j][4 * q + 1], b.y);
                    v[4 * q + 2] = __fadd_rn(acc[i][j][4 * q + 2], b.z), v[4 * q + 3] = __fadd_rn(acc[i][j][4 * q + 3], b.w);
                }
                if (gelu) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = gelu_erf(v[e]);
                }
                unsigned amax = 0;
#pragma unroll
                for (int e = 0; e < 16; ++e) amax = max(amax, f32_abs_bits(v[e]));
                amax = max(amax, (unsigned)__shfl_xor((int)amax, 32));
                const unsigned byte = mx4_scale_byte(amax);
                // columns 8q + 4hi .. +3 are 16 bits of word q, this lane's the low or the high ones; each lane stores two of the four words
                const unsigned c0 = mx4_codes8(v, byte), c1 = mx4_codes8(v + 8, byte);
                const unsigned got = (unsigned)__shfl_xor((int)(hi ? c0 : c1), 32);
                const unsigned low = hi ? got : c0, high = hi ? c1 : got;
                const unsigned w0 = (low & 0xffffu) | (high << 16), w1 = (low >> 16) | (high & 0xffff0000u);
                typedef unsigned v2u __attribute__((ext_vector_type(2)));
                __builtin_amdgcn_raw_buffer_store_b64(v2u{w0, w1}, ry, at < 0 ? at : at + nb / 2, 0, 0);
                bytes |= byte << (8 * (j % 4));
                constexpr int kRun = FN < 4 ? FN : 4;  // a wave's blocks of a group, whose scale bytes lie side by side
                if ((j + 1) % kRun == 0) {
                    if (hi == 0 && m < tile.rows) {
                        uint8_t* s = p.y_scales + ((int64_t)(nb / kMxGroup) * p.M + tile.row + m) * 4 + (nb % kMxGroup) / 32 - (kRun - 1);
                        if constexpr (kRun == 4)
                            *reinterpret_cast<unsigned*>(s) = bytes;
                        else if constexpr (kRun == 2)
                            *reinterpret_cast<unsigned short*>(s) = (unsigned short)bytes;
                        else
                            *s = (uint8_t)bytes;
                    }
                    bytes = 0;
                }
            }
        }
    } else {
        static_assert(kSwap || FN == 1 || FN == 2 || FN == 4, "wave tiles of whole or half groups");
        const float sx = Op::kMx4 ? 0.0f : p.sx[0], next_scale = kOut == Q8_TYPE_I8 ? p.next_scale[0] : 0.0f;
        const __amdgpu_buffer_rsrc_t ry =
            __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(p.y) + (int64_t)tile.row * N * kSize, 0, tile.rows * N * kSize, 0x00020000);
        float famax = 0.0f;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int n = n0 + wn * TN + j * 32 + l32;
            const bool inside = n < N;
            const ProductColumn c = product_column<Op>(p, tile.group, min(n, N - 1), sx);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int m = wm * TM + i * 32 + 4 * hi;
                float v[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = product_value<Op>(acc[i][j][e], c);
                if (gelu) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = gelu_erf(v[e]);
                }
                if constexpr (!Op::kMx4) {
                    if (p.flags & Q8_EPI_ABSMAX) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (inside && m + 8 * (e >> 2) + (e & 3) < tile.rows) famax = __builtin_fmaxf(famax, __builtin_fabsf(v[e]));
                    }
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int r = m + 8 * (e >> 2) + (e & 3);
                    const int at = inside ? (r * N + n) * kSize : (int)kOutOfRange;  // rows behind the tile's are out of the descriptor's range
                    if constexpr (kOut == Q8_TYPE_F32)
                        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[e]), ry, at, 0, 0);
                    else if constexpr (kOut == Q8_TYPE_BF16)
                        __builtin_amdgcn_raw_buffer_store_b16(f32_to_bf16(v[e]), ry, at, 0, 0);
                    else
                        __builtin_amdgcn_raw_buffer_store_b8((unsigned char)quantize_code(v[e], next_scale), ry, at, 0, 0);
                }
            }
        }
        if constexpr (!Op::kMx4)
            if (p.flags & Q8_EPI_ABSMAX) publish_amax<NW>(__float_as_uint(famax), reinterpret_cast<unsigned*>(lds), p.out_amax);
    }
#endif
}

template <class Op, int BM, int BN, int WGM, int WGN, int kSlots, int kWgs>
int launch_product_tile(const Product& p, hipStream_t st)
{
    const int64_t tiles_n = (p.N + BN - 1) / BN, tiles = row_tiles(p.M, p.group_rows, p.n_groups, BM) * tiles_n;
    if (tiles * WGM * WGN * 64 >= (int64_t)1 << 32) return 1;
    const dim3 grid((unsigned)tiles), block(WGM * WGN * 64);
    const unsigned group_m = 8;
#define Q8_PT_LAUNCH(OUT) \
    hipLaunchKernelGGL((product_tile_kernel<Op, BM, BN, WGM, WGN, kSlots, kWgs, OUT>), grid, block, 0, st, p, (unsigned)tiles_n, group_m)
    if (p.y_type == Q8_TYPE_F32) {
        Q8_PT_LAUNCH(Q8_TYPE_F32);
    } else if constexpr (Op::kMx4) {
        if (p.y_type == Q8_TYPE_BF16)
            Q8_PT_LAUNCH(Q8_TYPE_BF16);
        else
            Q8_PT_LAUNCH(Q8_TYPE_MX4);
    } else {
        Q8_PT_LAUNCH(Q8_TYPE_I8);
    }
#undef Q8_PT_LAUNCH
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace q8
