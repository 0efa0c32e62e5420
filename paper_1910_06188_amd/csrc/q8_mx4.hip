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

typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned short u16;

// Elements k .. k+7 of a row, zeros from K on.  kVec: k + 7 < K and the address is a multiple of 16 bytes.
template <bool kVec>
__device__ __forceinline__ void load8(const float* p, int left, float* v)
{
    if constexpr (kVec) {
        const v4f a = *reinterpret_cast<const v4f*>(p), b = *reinterpret_cast<const v4f*>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.0f;
    }
}
template <bool kVec>
__device__ __forceinline__ void load8(const u16* p, int left, float* v)
{
    if constexpr (kVec) {
        const v4u a = *reinterpret_cast<const v4u*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(a[i] << 16), v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? bf16_to_f32(p[i]) : 0.0f;
    }
}

// The values of E2M1 codes have two significant bits: rounding them to bf16 changes nothing (2^-128, the smallest, is a bf16 number).
template <bool kVec>
__device__ __forceinline__ void store8(float* p, int left, const float* v)
{
    if constexpr (kVec) {
        *reinterpret_cast<v4f*>(p) = v4f{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<v4f*>(p + 4) = v4f{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = v[i];
    }
}
template <bool kVec>
__device__ __forceinline__ void store8(u16* p, int left, const float* v)
{
    if constexpr (kVec) {
        v4u a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xffff0000u);
        *reinterpret_cast<v4u*>(p) = a;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (u16)(__float_as_uint(v[i]) >> 16);
    }
}

__device__ __forceinline__ unsigned amax8(const float* v)
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}

constexpr int kMxThreads = 256;
constexpr int kMxRows = kMxThreads / 16;  // rows of a workgroup's step, one group of each

// kCodes: codes and scales; else the values, in place if x is xq.
template <class T, bool kVec, bool kCodes>
__global__ __launch_bounds__(kMxThreads) void mx4_quantize_kernel(const T* x, int64_t M, int64_t K, unsigned groups, uint8_t* __restrict__ codes,
                                                                  uint8_t* __restrict__ scales, T* xq)
{
    const unsigned group = blockIdx.x % groups;
    const int64_t row = (int64_t)(blockIdx.x / groups) * kMxRows + threadIdx.x / 16;
    if (row >= M) return;  // whole quads leave
    const int in_group = (threadIdx.x % 16) * 8;
    const int64_t k = (int64_t)group * kMxGroup + in_group;
    const int left = (int)min(K - k, (int64_t)8);
    float v[8];
    if (kVec ? left > 0 : true)
        load8<kVec>(x + row * K + k, left, v);
    else
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    const unsigned byte = mx4_scale_byte(quad_max_u32(amax8(v)));
    const unsigned c = mx4_codes8(v, byte);
    if constexpr (kCodes) {
        *reinterpret_cast<unsigned*>(codes + (row * groups + group) * (kMxGroup / 2) + in_group / 2) = c;
        if (threadIdx.x % 4 == 0) scales[((int64_t)group * M + row) * 4 + in_group / 32] = (uint8_t)byte;
    } else if (left > 0) {
        mx4_values8(c, byte, v);
        store8<kVec>(xq + row * K + k, left, v);
    }
}

template <class T, bool kCodes>
static int launch(const T* x, int64_t M, int64_t K, uint8_t* codes, uint8_t* scales, T* xq, hipStream_t st)
{
    const int64_t groups = mx4_groups(K), blocks = (M + kMxRows - 1) / kMxRows * groups;
    if (blocks > 0x7fffffffLL) return 1;
    // eight elements at a time where all of them start on 16 bytes
    const bool vec = K % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0 && reinterpret_cast<uintptr_t>(xq) % 16 == 0;
    if (vec)
        hipLaunchKernelGGL((mx4_quantize_kernel<T, true, kCodes>), dim3((unsigned)blocks), dim3(kMxThreads), 0, st, x, M, K, (unsigned)groups, codes, scales, xq);
    else
        hipLaunchKernelGGL((mx4_quantize_kernel<T, false, kCodes>), dim3((unsigned)blocks), dim3(kMxThreads), 0, st, x, M, K, (unsigned)groups, codes, scales, xq);
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
