// Quantization to the 4-bit microscaled format (q8_mx4_device.h) and back: codes and scales for the products, or in training the
// value of each element's code.  Blocks of 32 need nothing from outside themselves, so one pass over the tensor does it, with no
// reduction over it first.
//
// Four lanes share a block, eight elements each: two 16-byte loads of fp32 (one of bf16), a maximum over the quad in the vector
// ALU, four conversions of two elements, a store of 4 bytes of codes (or of the values).  Sixteen lanes are a storage group of 128
// elements, and a wave takes the same group of four neighbouring rows, whose 4 x 4 scale bytes lie side by side.
#include "q8_launch.h"
#include "q8_mx4_device.h"

namespace q8 {

typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned short u16;

// The values of E2M1 codes have two significant bits: rounding them to bf16 changes nothing (2^-128, the smallest, is a bf16 number).
__device__ __forceinline__ void store8(float* p, int left, const float* v)
{
    if (left >= 8) {
        __builtin_memcpy(p, v, 32);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = v[i];
    }
}
__device__ __forceinline__ void store8(u16* p, int left, const float* v)
{
    if (left >= 8) {
        unsigned a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xffff0000u);
        __builtin_memcpy(p, a, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (u16)(__float_as_uint(v[i]) >> 16);
    }
}

// The general kernel.  kCodes: codes and scales; else the values, in place if x is xq.  A wave takes kUnits times four neighbouring rows of one
// group, all loads in front; the rows of a workgroup fill half a 128-byte line of scales or all of it.
template <class T, bool kCodes, int kWaves, int kUnits>
__global__ __launch_bounds__(kWaves * 64) void mx4_quantize_kernel(const T* x, int64_t M, int64_t K, unsigned groups, uint8_t* __restrict__ codes,
                                                                   uint8_t* __restrict__ scales, T* xq)
{
    constexpr int kRows = kWaves * 4;  // from one unit to the next
    const unsigned group = blockIdx.x % groups;
    const int64_t row0 = (int64_t)(blockIdx.x / groups) * (kRows * kUnits) + threadIdx.x / 16;
    const int in_group = (threadIdx.x % 16) * 8;
    const int64_t k = (int64_t)group * kMxGroup + in_group;
    const int left = (int)min(K - k, (int64_t)8);
    float v[kUnits][8];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int64_t row = row0 + u * kRows;
        if (row < M && left > 0) {
            load8(x + row * K + k, left, v[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = 0.0f;
        }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int64_t row = row0 + u * kRows;
        const unsigned byte = mx4_scale_byte(quad_max_u32(amax8(v[u])));
        const unsigned c = mx4_codes8(v[u], byte);
        if (row >= M) return;
        if constexpr (kCodes) {
            *reinterpret_cast<unsigned*>(codes + (row * groups + group) * (kMxGroup / 2) + in_group / 2) = c;
            if (threadIdx.x % 4 == 0) scales[((int64_t)group * M + row) * 4 + in_group / 32] = (uint8_t)byte;
        } else if (left > 0) {
            mx4_values8(c, byte, v[u]);
            store8(xq + row * K + k, left, v[u]);
        }
    }
}

// Values of rows that are whole blocks: the tensor is one run of blocks, and a lane takes the 16 bytes of its own place in it, workgroups of
// one wave in address order, which moves the most bytes on this part (12288 x 4096 to bf16 31 us, to fp32 60, the time of a copy; the general kernel 37 and 72).
template <class T>
__global__ __launch_bounds__(64) void mx4_fake_quantize_kernel(const T* x, T* xq, int64_t vectors)
{
    constexpr int kElems = 16 / sizeof(T);
    const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (i >= vectors) return;  // whole blocks leave
    const v4u in = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(x) + i);
    float v[8];
    if constexpr (kElems == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(in[e]), v[4 + e] = 0.0f;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[2 * e] = __uint_as_float(in[e] << 16), v[2 * e + 1] = __uint_as_float(in[e] & 0xffff0000u);
    }
    unsigned a = quad_max_u32(amax8(v));
    if constexpr (kElems == 4) a = max(a, (unsigned)__builtin_amdgcn_update_dpp(0, (int)a, 0x141, 0xf, 0xf, true));  // row_half_mirror: the block's other quad
    const unsigned byte = mx4_scale_byte(a);
    mx4_values8(mx4_codes8(v, byte), byte, v);
    v4u out;
    if constexpr (kElems == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = __float_as_uint(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = (__float_as_uint(v[2 * e]) >> 16) | (__float_as_uint(v[2 * e + 1]) & 0xffff0000u);
    }
    __builtin_nontemporal_store(out, reinterpret_cast<v4u*>(xq) + i);
}

template <class T, bool kCodes>
static int launch(const T* x, int64_t M, int64_t K, uint8_t* codes, uint8_t* scales, T* xq, hipStream_t st)
{
    constexpr int64_t kElems = 16 / sizeof(T);
    const bool aligned = reinterpret_cast<uintptr_t>(x) % 16 == 0 && reinterpret_cast<uintptr_t>(xq) % 16 == 0;
    if constexpr (!kCodes) {
        const int64_t vectors = M * K / kElems;
        if (aligned && K % 32 == 0 && vectors <= ((int64_t)1 << 32) - 64) {  // a launch is limited to 2^32 threads, less a workgroup
            hipLaunchKernelGGL(mx4_fake_quantize_kernel<T>, dim3((unsigned)((vectors + 63) / 64)), dim3(64), 0, st, x, xq, vectors);
            return hipGetLastError() == hipSuccess ? 0 : 1;
        }
    }
    const int64_t groups = mx4_groups(K);
    // one unit for fp32 (12288 x 4096: 39.3 us, two 40.5, four 42.5), two for bf16, whose loads are half as wide (22.3, 20.5, 21.8)
    constexpr int kWaves = 4, kUnits = sizeof(T) == 4 ? 1 : 2;
    const int64_t blocks = (M + kWaves * 4 * kUnits - 1) / (kWaves * 4 * kUnits) * groups;
    if (blocks * kWaves * 64 >= (int64_t)1 << 32) return 1;
    hipLaunchKernelGGL((mx4_quantize_kernel<T, kCodes, kWaves, kUnits>), dim3((unsigned)blocks), dim3(kWaves * 64), 0, st, x, M, K, (unsigned)groups, codes, scales, xq);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

int launch_mx4_quantize(const void* x, bool bf16, int64_t M, int64_t K, uint8_t* codes, uint8_t* scales, hipStream_t st)
{
    return bf16 ? launch<u16, true>(static_cast<const u16*>(x), M, K, codes, scales, nullptr, st)
                : launch<float, true>(static_cast<const float*>(x), M, K, codes, scales, nullptr, st);
}

int launch_mx4_fake_quantize(const void* x, bool bf16, int64_t M, int64_t K, void* xq, hipStream_t st)
{
    return bf16 ? launch<u16, false>(static_cast<const u16*>(x), M, K, nullptr, nullptr, static_cast<u16*>(xq), st)
                : launch<float, false>(static_cast<const float*>(x), M, K, nullptr, nullptr, static_cast<float*>(xq), st);
}

}  // namespace q8
