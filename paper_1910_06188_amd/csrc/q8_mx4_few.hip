// The 4-bit FC layer on an fp32 or bf16 x of few rows, in one launch: such a layer is bound by launch latency and by how fast the weights come in, and
// a second launch for the quantizer costs as much again.  Blocks of the format need nothing from outside themselves, so every workgroup quantizes its
// rows of x into its own LDS while its first weights are on the way.
//
//   workgroup = KW waves, one tile of up to 32 rows and 32 columns
//   wave w    = the 128-byte units w, w + KW, ... of the reduction: four 1 KiB loads of whole lines of w, through LDS of its own
//
// As two launches and as one, us a call in a loop on one set of tensors: 1 x 1024 -> 4096 6.4 and 3.4, 8 x 1024 -> 4096 6.3 and 4.0, 256 x 512 -> 512 6.6 and 5.0,
// 128 x 768 -> 768 6.6 and 6.0; from 32 rows of 1024 on two are as fast (6.5 and 7.0), and many tiles slower as one (512 x 1024 -> 1024 7.8 and 10.5).  With the
// tensors of several layers in turn 1 x 1024 -> 4096 takes 4.6 to 4.8 a call; the kernel itself 3.8.
#include "q8_grouped_device.h"
#include "q8_load16.h"

namespace q8 {

constexpr int kFewMaxK = 4096, kFewElements = 24576, kFewTiles = 512;
constexpr int kFewRows = 32, kFewUnit = 128, kFewSteps = kFewUnit / 32, kFewUnitBytes = kFewRows * kFewUnit;
constexpr int kFewRow = kFewRows + 8;  // words of a row of partial sums: the halves of an accumulator store on different banks

__device__ __forceinline__ int few_swizzle(int r) { return (r ^ (r >> 3)) & 7; }

// LDS: the codes of x by units, their scales [group][row], the waves' staged weights; the partial sums take the place of all that.
constexpr int few_lds(int units, int waves)
{
    const int operands = units * (kFewUnitBytes + 2 * kFewRows * 4) + waves * kFewUnitBytes, sums = waves * kFewRows * kFewRow * 4;
    return operands > sums ? operands : sums;
}

// kUnits: units of a row at most.
template <class T, int KW, int kUnits>
__global__ __launch_bounds__(KW * 64, KW / 4) void product_few_kernel(const T* __restrict__ x, int64_t K, Product p)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ __attribute__((aligned(16))) char lds[few_lds(kUnits, KW)];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, hi = lane >> 5, chunk = lane & 7, row8 = lane >> 3;
    const int pitch = (int)p.pitch, units = (pitch + kFewUnit - 1) / kFewUnit, full = pitch / kFewUnit, groups = pitch / 64;
    const int row0 = (int)blockIdx.y * kFewRows, rows = (int)min(p.M - row0, (int64_t)kFewRows);
    char* x_scales = lds + kUnits * kFewUnitBytes;
    char* stage = x_scales + kUnits * 2 * kFewRows * 4 + wave * kFewUnitBytes;
    const int64_t n0 = (int64_t)blockIdx.x * 32;
    const int last_b = (int)min((int64_t)32, p.N - n0) - 1;

    const uint8_t* row[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) row[i] = p.w + (n0 + min(8 * i + row8, last_b)) * pitch;
    const int64_t ws_row = n0 + min(l32, last_b);
    v4i in[4];
    int sb = 0;
    auto load_unit = [&](int u) {
        const int at = u * kFewUnit + 16 * chunk;
        if (u < full) {
#pragma unroll
            for (int i = 0; i < 4; ++i) in[i] = load16_any(reinterpret_cast<const int8_t*>(row[i]) + at);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) in[i] = load16_bounded(reinterpret_cast<const int8_t*>(row[i]) + at, pitch - at, pitch);
        }
        const int64_t g = 2 * u + hi;
        sb = g < groups ? *reinterpret_cast<const int*>(p.ws + (g * p.N + ws_row) * 4) : 0;
    };
    if (wave < units) load_unit(wave);

    // Codes and scales of x.  Rows that it does not have stay as they are: their sums go nowhere.
    const unsigned words = (unsigned)pitch / 4;  // of a row's codes
    for (unsigned i = threadIdx.x; i < words * (unsigned)rows; i += KW * 64) {
        const unsigned r = i / words, c = i - r * words;
        float v[8];
        load8(x + (row0 + (int64_t)r) * K + c * 8, (int)max(min(K - (int64_t)c * 8, (int64_t)8), (int64_t)0), v);
        const unsigned byte = mx4_scale_byte(quad_max_u32(amax8(v)));
        const int at = (int)c * 4;
        *reinterpret_cast<unsigned*>(lds + at / kFewUnit * kFewUnitBytes + r * kFewUnit + (((at % kFewUnit / 16) ^ few_swizzle(r)) << 4) + at % 16) = mx4_codes8(v, byte);
        if (c % 4 == 0) x_scales[(c / 16 * kFewRows + r) * 4 + c % 16 / 4] = (char)byte;
    }
    if (groups % 2 && threadIdx.x < kFewRows) reinterpret_cast<int*>(x_scales)[groups * kFewRows + threadIdx.x] = 0;  // the last unit's other group: w reads as zeros there
    __syncthreads();

    v16f acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0;
    for (int u = wave; u < units; u += KW) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<v4i*>(stage + (8 * i + row8) * kFewUnit + ((chunk ^ few_swizzle(8 * i + row8)) << 4)) = in[i];
        const int ub = sb;
        if (u + KW < units) load_unit(u + KW);
        const int ua = *reinterpret_cast<const int*>(x_scales + ((2 * u + hi) * kFewRows + l32) * 4);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the lanes read what other lanes of this wave wrote
        __builtin_amdgcn_wave_barrier();
        v4i fa[kFewSteps], fb[kFewSteps];
#pragma unroll
        for (int s = 0; s < kFewSteps; ++s) {
            const int at = l32 * kFewUnit + (((4 * hi + s) ^ few_swizzle(l32)) << 4);
            fa[s] = *reinterpret_cast<const v4i*>(lds + u * kFewUnitBytes + at);
            fb[s] = *reinterpret_cast<const v4i*>(stage + at);
        }
        acc = OpMx4::mfma<0>(fa[0], fb[0], acc, ua, ub);
        acc = OpMx4::mfma<1>(fa[1], fb[1], acc, ua, ub);
        acc = OpMx4::mfma<2>(fa[2], fb[2], acc, ua, ub);
        acc = OpMx4::mfma<3>(fa[3], fb[3], acc, ua, ub);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();  // the partial sums lie where the operands were
    float* part = reinterpret_cast<float*>(lds);
    // Accumulator register e of lane (l32, hi) is row 8 (e / 4) + 4 hi + e % 4, column l32.
#pragma unroll
    for (int e = 0; e < 16; ++e) part[(wave * kFewRows + 8 * (e >> 2) + 4 * hi + (e & 3)) * kFewRow + l32] = acc[e];
    __syncthreads();
    finish_tile<OpMx4, KW>(p, RowTile{0, row0, rows}, n0, part, kFewRow);
#endif
}

// Few rows, or few tiles of short ones, whose quantization in every workgroup takes less than a launch.
bool mx4_few_eligible(int64_t M, int64_t N, int64_t K)
{
    const int64_t rows = M < kFewRows ? M : kFewRows, tiles = (M + kFewRows - 1) / kFewRows * ((N + 31) / 32);
    return M >= 1 && K >= 1 && K <= kFewMaxK && rows * K <= kFewElements && tiles <= kFewTiles;
}

template <class T>
static int launch(const T* x, int64_t K, const Product& p, hipStream_t st)
{
    const dim3 grid((unsigned)((p.N + 31) / 32), (unsigned)((p.M + kFewRows - 1) / kFewRows));
    if (p.pitch <= 4 * kFewUnit)
        hipLaunchKernelGGL((product_few_kernel<T, 8, 4>), grid, dim3(512), 0, st, x, K, p);
    else
        hipLaunchKernelGGL((product_few_kernel<T, 8, kFewMaxK / 256>), grid, dim3(512), 0, st, x, K, p);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

int launch_mx4_few(const void* x, bool bf16, int64_t K, const Product& p, hipStream_t st)
{
    return bf16 ? launch(static_cast<const unsigned short*>(x), K, p, st) : launch(static_cast<const float*>(x), K, p, st);
}

}  // namespace q8
