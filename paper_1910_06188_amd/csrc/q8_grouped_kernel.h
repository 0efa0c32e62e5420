// Tiled kernel of the grouped and 4-bit FC products, gfx950.  Included by one translation unit per tile shape (q8_grouped_tile_*.hip).
//
// A workgroup owns BM rows of one group and BN columns of the group's weights.  It walks the reduction in stages of 128 bytes a row
// (128 int8 codes, 256 4-bit ones), loaded straight into LDS by 16 bytes a lane, swizzled so that the fragment reads of the MFMAs
// are free of bank conflicts.  The scales of a stage (4-bit: two words a row) come into LDS with it, four bytes a lane.  kSlots stage
// buffers: one (load, wait, multiply; other workgroups of the unit fill the gaps) or two (the next stage loads under this one's MFMAs).  128x128
// tiles have one: two buffers and half the workgroups are 10 to 20 % slower.  256x256 have two, as a unit holds one of them.
//
// Loads and stores go through buffer descriptors whose bounds checks take the place of branches: a lane whose row of x does not exist, or whose
// 16 bytes lie behind the end of a row, is given an offset out of range and reads zeros; outputs outside the tile's rows and columns are dropped.
#pragma once
#include "q8_gemm_kernel.h"
#include "q8_grouped_device.h"

namespace q8 {

constexpr unsigned kPanel = 8;                 // tile rows of a panel
constexpr unsigned kOutOfRange = 0x80000000u;  // above the extent of every descriptor here

// 4 bytes per lane from a buffer straight into LDS: lane l lands at lds_addr + 4 l.
__device__ __forceinline__ void lds_dma4(v4i rsrc, unsigned voff, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(lds_addr), "v"(voff), "s"(rsrc) : "memory");
}

// kOut: the type of y.  It decides which operand the MFMA takes first, that is, what a lane holds of a 32x32 block.
//   fp32, bf16    x first: one column and 16 rows.  32 lanes store 32 neighbours of a row at once, whole 128-byte lines of fp32.  (With a row and 16
//                 columns a lane, stores take 16 bytes a lane but 32 bytes of 32 rows each, four times the requests to the L2: 12288 x 1024 -> 4096 to fp32
//                 59 us against 48; through LDS to whole lines 56.)
//                 bf16: of two blocks a lane has the columns 2 l and 2 l + 1, a word of y, and 32 lanes a line.  Which column a lane has is a matter of which
//                 row of w lies in its row of LDS, so this costs nothing (24576 rows of 16 experts, 1024 -> 4096 90 us; with the columns l and 32 + l exchanged
//                 between lanes 98).  fp32 the same way, 8 bytes a lane: on 4-bit codes no difference, on int8 42.7 against 38.5 (24576 rows, 1024 -> 1024).
//   4-bit, int8   w first: one row and four times four neighbouring columns.  A block of the 4-bit format -- 32 neighbours of a row -- is two
//                 lanes', its largest magnitude one exchange away.
// The bias of int8 codes is what the sums start from, which whole numbers allow.  That of 4-bit codes is added once behind the sum: a sum that starts from it
// would be rounded at its magnitude by every matrix instruction, K / 64 of them.
template <class Op, int BM, int BN, int WGM, int WGN, int kSlots, int kAhead, int kWgs, int kOut>
__global__ __launch_bounds__(WGM* WGN * 64, kWgs* WGM* WGN / 4) void product_tile_kernel(Product p, unsigned tiles_n, unsigned panel_reciprocal, int stream_out)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool kRowLane = kOut == Q8_TYPE_MX4 || kOut == Q8_TYPE_I8;
    constexpr int NW = WGM * WGN;
    constexpr int TM = BM / WGM, TN = BN / WGN, FM = TM / 32, FN = TN / 32;
    constexpr bool kPairs = kOut == Q8_TYPE_BF16 && FN % 2 == 0;
    constexpr int A_BYTES = BM * kBK, B_BYTES = BN * kBK, OPERANDS = A_BYTES + B_BYTES;
    constexpr int SCALES = Op::kMx4 ? (BM + BN) * 8 : 0, SLOT = OPERANDS + SCALES;  // scales: [A | B][group of the stage][row]
    constexpr int A_LOADS = BM / 8 / NW, B_LOADS = BN / 8 / NW;
    constexpr int S_UNITS = Op::kMx4 ? (BM + BN) / 32 : 0, S_LOADS = (S_UNITS + NW - 1) / NW;  // 64 rows of one group each
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "tile rows must split over the waves");
    static_assert(TM % 32 == 0 && TN % 32 == 0 && BM % 64 == 0 && BN % 64 == 0, "whole MFMA blocks and whole scale loads");
    static_assert(kSlots == 1 || kSlots == 2, "the waits below are for all loads");
    static_assert(kWgs * (kSlots * SLOT + BN * 4) <= 160 * 1024, "LDS is 160 KiB per compute unit");
    using Sum = typename Op::Sum;
    __shared__ __attribute__((aligned(1024))) char lds[kSlots * SLOT];
    __shared__ __attribute__((aligned(16))) Sum bias[BN];  // of each column, int8 the quantized one

    const int lane = threadIdx.x & 63, l32 = lane & 31, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned lds_base = (unsigned)(size_t)(lds_ptr_t)lds;

    // A wave that still has loads to ask for and MFMAs to issue goes before the ones that convert and store (24576 rows of 16 experts, 1024 -> 4096 to codes with
    // GELU 93 us, without priorities 100; to fp32 and bf16 within 4 % either way).
    __builtin_amdgcn_s_setprio(3);

    // The launch has room for every group ending inside a tile; the tiles that there are go to the XCDs in equal, contiguous shares, in panels of
    // kPanel tile rows, column by column.
    const RowTiles<BM> row_tiles(p);
    const unsigned tiles_m = row_tiles.count, tiles = tiles_m * tiles_n;
    if (blockIdx.x >= tiles) return;
    const unsigned pid = (unsigned)xcd_remap((int)blockIdx.x, (int)tiles), per_panel = kPanel * tiles_n;
    // pid / per_panel by the launch's reciprocal, at most one too small; a division takes as long as a quarter of a stage
    unsigned panel = (unsigned)(((unsigned long long)pid * panel_reciprocal) >> 32);
    panel += pid - panel * per_panel >= per_panel;
    const unsigned in_panel = pid - panel * per_panel, panel_rows = min(kPanel, tiles_m - panel * kPanel);
    const unsigned col = panel_rows == kPanel ? in_panel / kPanel : in_panel / panel_rows;
    const RowTile tile = row_tiles.find(panel * kPanel + (in_panel - col * panel_rows));
    const int n0 = (int)col * BN;
    const int N = (int)p.N, pitch = (int)p.pitch;
    const int rows_b = min(BN, N - n0);

    // Offsets of this lane's 16 bytes in the operands' descriptors, of whose rows it loads every eighth; rows behind the tile's are out of range, which takes no
    // comparison: a row's offset is at least its number times the pitch.  x starts at the tile's first row, or, where rows are picked by index, at its own.
    const int64_t x_first = p.x_rows ? 0 : tile.row;
    const unsigned x_extent = p.x_rows ? (unsigned)p.x_count : (unsigned)tile.rows;
    const uint8_t* Xt = p.x + x_first * pitch;
    const uint8_t* Wt = p.w + ((int64_t)tile.group * N + n0) * pitch;
    const int chunk = lane & 7, row8 = lane >> 3;
    // swizzle_of_row(r) of row r = 8 g + row8 is row8 ^ g, three bits of each
    const auto chunk_at = [&](int g) { return (unsigned)(((chunk ^ row8) << 4) ^ ((g & 7) << 4)); };
    unsigned a_off[A_LOADS], b_off[B_LOADS];
    const int groups = pitch / 64;
    unsigned s_off[S_LOADS ? S_LOADS : 1];
#pragma unroll
    for (int i = 0; i < B_LOADS; ++i) {
        const int g = wave * B_LOADS + i;
        if constexpr (kPairs)  // row 2 (s % 32) + s / 32 % 2 of 64 in LDS row s = 8 g + row8
            b_off[i] = (unsigned)(2 * row8) * (unsigned)pitch + (unsigned)((g / 8 * 64 + g % 4 * 16 + g / 4 % 2) * pitch) + chunk_at(g);
        else
            b_off[i] = (unsigned)row8 * (unsigned)pitch + (unsigned)(g * 8 * pitch) + chunk_at(g);
    }
    // The scale loads of this wave, 64 rows of one group of a stage each.
    const auto scale_row = [&](int i) {  // row of the operand that load i takes to this lane
        const int u = wave + i * NW;
        return u < BM / 32 ? u % (BM / 64) * 64 + lane : (u - BM / 32) % (BN / 64) * 64 + (kPairs ? 2 * l32 + hi : lane);
    };
    if (p.x_rows) {
        int id[A_LOADS], scale_id[S_LOADS ? S_LOADS : 1];  // all asked for before the first is looked at
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i) id[i] = p.x_rows[tile.row + min((wave * A_LOADS + i) * 8 + row8, tile.rows - 1)];
#pragma unroll
        for (int i = 0; i < S_LOADS; ++i) scale_id[i] = p.x_rows[tile.row + min(scale_row(i), tile.rows - 1)];
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i)
            a_off[i] = (unsigned)id[i] < (unsigned)p.x_count ? (unsigned)id[i] * (unsigned)pitch + chunk_at(wave * A_LOADS + i) : kOutOfRange;
#pragma unroll
        for (int i = 0; i < S_LOADS; ++i) {
            const bool there = (unsigned)scale_id[i] < (unsigned)p.x_count;
            s_off[i] = wave + i * NW >= BM / 32 ? (unsigned)scale_row(i) * 4u : there ? (unsigned)scale_id[i] * 4u : kOutOfRange;
        }
    } else {
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i) {
            const int g = wave * A_LOADS + i;
            a_off[i] = (unsigned)row8 * (unsigned)pitch + (unsigned)(g * 8 * pitch) + chunk_at(g);
        }
#pragma unroll
        for (int i = 0; i < S_LOADS; ++i) s_off[i] = (unsigned)scale_row(i) * 4u;
    }
    // Of each scale load: the words of its group in the first stage, from one stage to the next, how far they go, which group of the stage.
    const uint8_t* s_base[S_LOADS ? S_LOADS : 1];
    int64_t s_step[S_LOADS ? S_LOADS : 1];
    unsigned s_extent[S_LOADS ? S_LOADS : 1];
    int s_group[S_LOADS ? S_LOADS : 1];
    if constexpr (Op::kMx4) {
#pragma unroll
        for (int i = 0; i < S_LOADS; ++i) {
            const int u = wave + i * NW;
            const bool of_x = u < BM / 32;
            s_group[i] = of_x ? u / (BM / 64) : (u - BM / 32) / (BN / 64);
            const int64_t rows = of_x ? p.x_count : (int64_t)N;
            const uint8_t* all = of_x ? p.xs + x_first * 4 : p.ws + ((int64_t)tile.group * groups * N + n0) * 4;
            s_base[i] = all + s_group[i] * rows * 4;
            s_step[i] = rows * 8;
            s_extent[i] = (of_x ? x_extent : (unsigned)rows_b) * 4u;
        }
    }

    const int KT = pitch / kBK, tail = pitch % kBK;  // whole stages, and the bytes behind them (a whole number of 16)
    const unsigned extent_a = x_extent * (unsigned)pitch, extent_b = (unsigned)rows_b * (unsigned)pitch;
    // Stage kt into a slot; past the end of the rows through empty descriptors, which fetch nothing.
    auto load_stage = [&](int kt, int slot, auto whole) {
        constexpr bool kWhole = decltype(whole)::value;
        const unsigned koff = (unsigned)kt * kBK, dst = lds_base + (unsigned)(slot * SLOT);
        const bool live = !kWhole || kt < KT;
        const v4i qa = make_rsrc(Xt, live ? extent_a : 0u), qb = make_rsrc(Wt, live ? extent_b : 0u);
        auto at = [&](unsigned off, int r) { return kWhole || ((chunk ^ swizzle_of_row(r)) * 16 < tail) ? off : kOutOfRange; };
#pragma unroll
        for (int i = 0; i < A_LOADS; ++i)
            lds_dma16_first(qa, at(a_off[i], (wave * A_LOADS + i) * 8 + row8), koff, dst + (wave * A_LOADS + i) * 1024);
#pragma unroll
        for (int i = 0; i < B_LOADS; ++i)
            lds_dma16_first(qb, at(b_off[i], (wave * B_LOADS + i) * 8 + row8), koff, dst + A_BYTES + (wave * B_LOADS + i) * 1024);
        if constexpr (Op::kMx4) {
#pragma unroll
            for (int i = 0; i < S_LOADS; ++i) {
                const int u = wave + i * NW;
                if (S_UNITS % NW == 0 || u < S_UNITS) lds_dma4(make_rsrc(s_base[i], live && (kWhole || s_group[i] == 0) ? s_extent[i] : 0u), s_off[i], dst + OPERANDS + u * 256);
                s_base[i] += live ? s_step[i] : 0;
            }
        }
    };

    const int wm = wave / WGN, wn = wave % WGN;
    const auto column_of = [](int j, int l) { return kPairs ? j / 2 * 64 + 2 * l + j % 2 : j * 32 + l; };  // of the wave's, lane l's of block j if it has one
    // Where this lane finds its 16 bytes of step 0 in the first block of its wave's rows.  32 rows on, a row's swizzle differs in bit 2 alone,
    // so the block behind is 4 KiB away and the chunk's bit flipped; step ks has ks in the chunk's low bits.  So neither needs an address of its own: the
    // registers that eight of them took keep 128x128 tiles from having four workgroups a unit (24576 rows of 16 experts, 1024 -> 4096 92 us with three, 84 with
    // four; -> codes with GELU 101 and 94).
    static_assert((TM == 32 || TM % 64 == 0) && (TN == 32 || TN % 64 == 0), "the swizzles of a wave's blocks");
    const int ra = wm * TM + l32, rb = wn * TN + l32;
    const int a_lane = ra * kBK + (((4 * hi) ^ swizzle_of_row(ra)) << 4), b_lane = A_BYTES + rb * kBK + (((4 * hi) ^ swizzle_of_row(rb)) << 4);
    const int a_sc = OPERANDS + (hi * BM + wm * TM + l32) * 4, b_sc = OPERANDS + BM * 8 + (hi * BN + wn * TN + l32) * 4;

    load_stage(0, 0, std::true_type{});
    const float sx = Op::kMx4 ? 0.0f : p.sx[0];
    for (int t = threadIdx.x; t < BN; t += NW * 64) {
        const ProductColumn c = product_column<Op>(p, tile.group, min(n0 + t, N - 1), sx);
        if constexpr (Op::kMx4)
            bias[t] = c.b;
        else
            bias[t] = c.bq;
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
    __syncthreads();

    // Accumulator register e of lane l is column 8 (e / 4) + 4 (l / 32) + e % 4 and row l % 32 of its block if kRowLane, else the other way round.
    typedef Sum v4s __attribute__((ext_vector_type(4)));
    typename Op::Acc acc[FM][FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        if constexpr (kRowLane && !Op::kMx4) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v4s c = *reinterpret_cast<const v4s*>(bias + wn * TN + j * 32 + 8 * q + 4 * hi);
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = c[e];
            }
        } else {
            const Sum c = Op::kMx4 ? 0 : bias[wn * TN + column_of(j, l32)];
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = c;
        }
    }

    // The MFMAs of a stage.  The fragments come kAhead - 1 steps ahead of them; as soon as the last are under way, `loads` may ask for the next stage.
    auto multiply = [&](const char* stage, auto loads) {
        int sa[FM], sb[FN];
        if constexpr (Op::kMx4) {
#pragma unroll
            for (int f = 0; f < FM; ++f) sa[f] = *reinterpret_cast<const int*>(stage + a_sc + f * 128);
#pragma unroll
            for (int f = 0; f < FN; ++f) sb[f] = *reinterpret_cast<const int*>(stage + b_sc + f * 128);
        }
        v4i fa[kAhead][FM], fb[kAhead][FN];
        auto read_step = [&](auto kc) {
            constexpr int ks = decltype(kc)::value;
            int a_at = a_lane, b_at = b_lane;
            if constexpr (ks > 0) {  // in assembly, or the compiler moves them out of the loop and keeps all eight
                asm volatile("v_xor_b32 %0, %2, %1" : "=v"(a_at) : "v"(a_lane), "i"(ks << 4));
                asm volatile("v_xor_b32 %0, %2, %1" : "=v"(b_at) : "v"(b_lane), "i"(ks << 4));
            }
#pragma unroll
            for (int f = 0; f < FM; ++f) fa[ks % kAhead][f] = *reinterpret_cast<const v4i*>(stage + (a_at ^ ((f & 1) << 6)) + f * 32 * kBK);
#pragma unroll
            for (int f = 0; f < FN; ++f) fb[ks % kAhead][f] = *reinterpret_cast<const v4i*>(stage + (b_at ^ ((f & 1) << 6)) + f * 32 * kBK);
        };
        static_for<0, kAhead - 1>([&](auto kc) { read_step(kc); });
        static_for<0, kKS>([&](auto kc) {
            constexpr int ks = decltype(kc)::value, next = ks + kAhead - 1;
            if constexpr (next < kKS) read_step(std::integral_constant<int, next>{});
            if constexpr (next == kKS - 1) {
                __builtin_amdgcn_sched_barrier(0);
                loads();
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    if constexpr (kRowLane)
                        acc[i][j] = Op::template mfma<ks>(fb[ks % kAhead][j], fa[ks % kAhead][i], acc[i][j], Op::kMx4 ? sb[j] : 0, Op::kMx4 ? sa[i] : 0);
                    else
                        acc[i][j] = Op::template mfma<ks>(fa[ks % kAhead][i], fb[ks % kAhead][j], acc[i][j], Op::kMx4 ? sa[i] : 0, Op::kMx4 ? sb[j] : 0);
            __builtin_amdgcn_sched_barrier(0);  // fragments of later steps would only take registers
        });
    };
    // One slot: the next stage loads as soon as every wave holds the last fragments of this one, under the MFMAs that are left.  Two: into the
    // other slot from the start.
    for (int kt = 0; kt < KT; ++kt) {
        if constexpr (kSlots == 2) load_stage(kt + 1, (kt + 1) & 1, std::true_type{});
        multiply(lds + (kSlots == 2 ? (kt & 1) * SLOT : 0), [&] {
            if constexpr (kSlots == 1) {
                __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
                __syncthreads();
                load_stage(kt + 1, 0, std::true_type{});
            }
        });
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));  // own loads have landed and own reads are complete
        __syncthreads();
    }
    if (tail) {
        load_stage(KT, 0, std::false_type{});
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
        __syncthreads();
        multiply(lds, [] {});
    }

    __builtin_amdgcn_s_setprio(0);

    // Epilogue.  The lane's number is counted anew, so that it takes no register through the loop.
    const int out_lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)), out_l32 = out_lane & 31, out_hi = out_lane >> 5;
    const auto column = [&](int j) { return column_of(j, out_l32); };
    typedef unsigned v2u __attribute__((ext_vector_type(2)));
    typedef unsigned v4u __attribute__((ext_vector_type(4)));
    const bool gelu = p.flags & Q8_EPI_GELU;
    constexpr int kSize = kOut == Q8_TYPE_F32 ? 4 : kOut == Q8_TYPE_BF16 ? 2 : 1;
    const int row_bytes = kOut == Q8_TYPE_MX4 ? N / 2 : N * kSize;
    const __amdgpu_buffer_rsrc_t ry = __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(p.y) + (int64_t)tile.row * row_bytes, 0, tile.rows * row_bytes, 0x00020000);
    const float r = Op::kMx4 ? 1.0f : dequant_factor(sx, p.sw[tile.group]);
    const float next_scale = kOut == Q8_TYPE_I8 ? p.next_scale[0] : 0.0f;
    float famax = 0.0f;
    // Block (i, j) as fp32 values.
    auto block_values = [&](int i, int j, float* v) {
        if constexpr (Op::kMx4 && kRowLane) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v4s c = *reinterpret_cast<const v4s*>(bias + wn * TN + j * 32 + 8 * q + 4 * out_hi);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * q + e] = __fadd_rn(acc[i][j][4 * q + e], c[e]);
            }
        } else if constexpr (Op::kMx4) {
            const float c = bias[wn * TN + column(j)];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = __fadd_rn(acc[i][j][e], c);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = (float)acc[i][j][e] * r;
        }
        if (gelu) {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = product_gelu<Op>(v[e]);
        }
        if constexpr (!Op::kMx4) {
            if (p.flags & Q8_EPI_ABSMAX) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int along = 8 * (e >> 2) + 4 * out_hi + (e & 3), m = wm * TM + i * 32 + (kRowLane ? out_l32 : along), n = n0 + wn * TN + (kRowLane ? j * 32 + along : column(j));
                    if (m < tile.rows && n < N) famax = __builtin_fmaxf(famax, __builtin_fabsf(v[e]));
                }
            }
        }
    };
    if constexpr (kOut == Q8_TYPE_MX4) {
        static_assert(kOut != Q8_TYPE_MX4 || FN == 1 || FN == 2 || FN == 4, "wave tiles of a group, or of a half or a quarter of one");
        constexpr int kPair = FN < 2 ? 1 : 2;  // blocks that one store takes
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int m = wm * TM + i * 32 + out_l32;
            const unsigned row_at = m < tile.rows ? (unsigned)(m * row_bytes) : kOutOfRange;
            const int nw = n0 + wn * TN;
            if (nw >= N) break;  // columns come in whole groups of 128
            unsigned bytes = 0;  // scale bytes, side by side in a group's word
#pragma unroll
            for (int j = 0; j < FN; j += kPair) {
                unsigned c[kPair][2];
#pragma unroll
                for (int h = 0; h < kPair; ++h) {
                    float v[16];
                    block_values(i, j + h, v);
                    float a = __builtin_fabsf(v[0]);
#pragma unroll
                    for (int e = 1; e < 15; e += 2) a = __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, __builtin_fabsf(v[e])), __builtin_fabsf(v[e + 1]));
                    a = __builtin_elementwise_maximum(a, __builtin_fabsf(v[15]));
                    const v2u both = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(a), false, false);  // the two lanes of the row
                    const unsigned byte = mx4_scale_byte(max(both[0], both[1]));
                    c[h][0] = mx4_codes8(v, byte), c[h][1] = mx4_codes8(v + 8, byte);
                    bytes |= byte << (8 * (j + h));
                }
                // Columns 8q + 4hi .. +3 are 16 bits of word q of a block, this lane's the low or the high ones.  Lanes l and l + 32 exchange halves of two
                // blocks, so that each holds four whole words of one.
                if constexpr (kPair == 2) {
                    const v2u p0 = __builtin_amdgcn_permlane32_swap(c[0][0], c[1][0], false, false), p1 = __builtin_amdgcn_permlane32_swap(c[0][1], c[1][1], false, false);
                    const v4u w = {(p0[0] & 0xffffu) | (p0[1] << 16), (p0[0] >> 16) | (p0[1] & 0xffff0000u), (p1[0] & 0xffffu) | (p1[1] << 16), (p1[0] >> 16) | (p1[1] & 0xffff0000u)};
                    __builtin_amdgcn_raw_buffer_store_b128(w, ry, row_at + (unsigned)((nw + (j + out_hi) * 32) / 2), 0, 0);
                } else {
                    const v2u p0 = __builtin_amdgcn_permlane32_swap(c[0][0], c[0][1], false, false);
                    __builtin_amdgcn_raw_buffer_store_b64(v2u{(p0[0] & 0xffffu) | (p0[1] << 16), (p0[0] >> 16) | (p0[1] & 0xffff0000u)}, ry, row_at + (unsigned)((nw + j * 32) / 2 + 8 * out_hi), 0, 0);
                }
            }
            if (out_hi == 0 && m < tile.rows) {
                uint8_t* s = p.y_scales + ((int64_t)(nw / kMxGroup) * p.M + tile.row + m) * 4 + (nw % kMxGroup) / 32;
                if constexpr (FN == 4)
                    *reinterpret_cast<unsigned*>(s) = bytes;
                else if constexpr (FN == 2)
                    *reinterpret_cast<unsigned short*>(s) = (unsigned short)bytes;
                else
                    *s = (uint8_t)bytes;
            }
        }
    } else if constexpr (kOut == Q8_TYPE_I8) {
        const bool wide = N % 4 == 0 && reinterpret_cast<uintptr_t>(p.y) % 4 == 0;  // four codes start on a word and no row ends inside them
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int m = wm * TM + i * 32 + out_l32;
            const unsigned row_at = m < tile.rows ? (unsigned)(m * row_bytes) : kOutOfRange;
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                float v[16];
                block_values(i, j, v);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = n0 + wn * TN + j * 32 + 8 * q + 4 * out_hi;
                    unsigned code[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) code[e] = (unsigned)quantize_code(v[4 * q + e], next_scale) & 0xffu;
                    if (wide) {
                        __builtin_amdgcn_raw_buffer_store_b32(code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24, ry, n < N ? row_at + (unsigned)n : kOutOfRange, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b8((unsigned char)code[e], ry, n + e < N ? row_at + (unsigned)(n + e) : kOutOfRange, 0, 0);
                    }
                }
            }
        }
    } else {
        // Rows of a block lie in registers, so a row's place is a scalar offset -- which the bounds check does not see: tiles that are cut short add it to
        // the lane's own.
        constexpr int kStep = kPairs ? 2 : 1;
        const bool words = kPairs && N % 2 == 0 && reinterpret_cast<uintptr_t>(p.y) % 4 == 0;
        auto store_tile = [&](auto fullc, auto streamc) {
            constexpr bool kFull = decltype(fullc)::value;
            constexpr int kAux = decltype(streamc)::value ? 2 : 0;  // aux bit 1: non-temporal
            auto store = [&](auto value, unsigned at, int row) {
                const unsigned to = kFull ? at : at + (unsigned)(row * row_bytes);
                const int uniform = kFull ? row * row_bytes : 0;
                if constexpr (sizeof(value) == 4)
                    __builtin_amdgcn_raw_buffer_store_b32(value, ry, to, uniform, kAux);
                else
                    __builtin_amdgcn_raw_buffer_store_b16(value, ry, to, uniform, kAux);
            };
#pragma unroll
            for (int j = 0; j < FN; j += kStep) {
                const int n = n0 + wn * TN + column(j);
                const unsigned at = n < N ? (unsigned)(4 * out_hi * row_bytes + n * kSize) : kOutOfRange, beside = n + 1 < N ? at + kSize : kOutOfRange;
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    const int m = wm * TM + i * 32;
                    float v[kStep][16];
#pragma unroll
                    for (int h = 0; h < kStep; ++h) block_values(i, j + h, v[h]);
                    if (words) {
                        if constexpr (kPairs) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) store(f32_to_bf16x2(v[0][e], v[1][e]), at, m + 8 * (e >> 2) + (e & 3));
                        }
                    } else {
#pragma unroll
                        for (int h = 0; h < kStep; ++h)
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                if constexpr (kOut == Q8_TYPE_F32)
                                    store(__float_as_uint(v[h][e]), h ? beside : at, m + 8 * (e >> 2) + (e & 3));
                                else
                                    store(f32_to_bf16(v[h][e]), h ? beside : at, m + 8 * (e >> 2) + (e & 3));
                            }
                    }
                }
            }
        };
        if (tile.rows < BM)
            store_tile(std::false_type{}, std::false_type{});
        else if (stream_out)
            store_tile(std::true_type{}, std::true_type{});
        else
            store_tile(std::true_type{}, std::false_type{});
    }
    if constexpr (!Op::kMx4)
        if (p.flags & Q8_EPI_ABSMAX) publish_amax<NW>(__float_as_uint(famax), reinterpret_cast<unsigned*>(lds), p.out_amax);
#endif
}

template <class Op, int BM, int BN, int WGM, int WGN, int kSlots, int kAhead, int kWgs>
int launch_product_tile(const Product& p, hipStream_t st)
{
    const int64_t tiles_n = (p.N + BN - 1) / BN, tiles = row_tiles(p.M, p.n_groups, BM) * tiles_n;
    if (tiles * WGM * WGN * 64 >= (int64_t)1 << 32) return 1;
    const dim3 grid((unsigned)tiles), block(WGM * WGN * 64);
    // Outputs that the L2s (32 MB together) do not hold anyway are stored past the caches: lying dirty in the 256 MB behind the L2s, they are written back under the
    // next launch.  K = 1024, N = 4096, us, with ordinary stores and with these, four sets of tensors in turn, as the layers of a model have them: 96 MB of fp32 31.8 and
    // 27.5, 192 MB 56.3 and 48.2, 320 MB 88.2 and 76.1; 48 MB of bf16 23.4 and 21.7, 128 MB 62.4 and 51.8.  With the next layer's quantizer behind each: 47.5
    // and 51.1, 96.2 and 95.2, 165.1 and 153.9; 36.8 and 36.1, 91.8 and 95.2.  The other way round only where all of it stays in the caches: one set, 192 MB with the
    // quantizer 77.2 and 87.0, by itself 47.7 and 47.8.
    const int stream_out = p.M * p.N * (p.y_type == Q8_TYPE_BF16 ? 2 : 4) >= (int64_t)32 << 20;
#define Q8_PT_LAUNCH(OUT) \
    hipLaunchKernelGGL((product_tile_kernel<Op, BM, BN, WGM, WGN, kSlots, kAhead, kWgs, OUT>), grid, block, 0, st, p, (unsigned)tiles_n, (unsigned)(((int64_t)1 << 32) / (kPanel * tiles_n)), stream_out)
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
