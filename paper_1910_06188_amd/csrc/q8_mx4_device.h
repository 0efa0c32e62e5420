// The 4-bit microscaled format (MXFP4 of the OCP Microscaling Formats specification, version 1.0) on the device: blocks of 32
// neighbours of a row share a power of two, and each element is an E2M1 number -- 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives.
//
//   a = max |x| of the block, s = max(floor(log2 a) - 2, -127), scale byte = s + 127, code = nearest E2M1 number of x / 2^s
//
// floor(log2 a) of a normal binary32 number is its exponent field - 127, so the scale byte is that field - 2, not below 0: no
// logarithm and no division anywhere.  a / 2^s lies in [4, 8); what is above 6 takes the code of 6, as the specification has it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace q8 {

constexpr int kMxGroup = 128;       // elements of a storage group: four blocks, 64 bytes of codes and 4 of scales
constexpr unsigned kMxNan = 255;    // the scale byte of a block with an infinity or a NaN in it: all its elements are NaN

__host__ __device__ constexpr int64_t mx4_groups(int64_t K) { return (K + kMxGroup - 1) / kMxGroup; }

// Scale byte of a block from the bit pattern of its largest |x| (the unsigned order of |x| puts infinities and NaN on top).
__device__ __forceinline__ unsigned mx4_scale_byte(unsigned amax_bits)
{
    const unsigned e = amax_bits >> 23;
    return e == 255u ? kMxNan : max(e, 2u) - 2u;
}

// 2^(byte - 127); 2^-127 is no normal number.
__device__ __forceinline__ float mx4_scale(unsigned byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

// Eight elements of one block to eight codes, the first in the low half of the low byte.  v_cvt_scalef32_pk_fp4_f32 divides by
// the power of two, rounds to the nearest code with ties to even, keeps the sign and takes magnitudes above 6 to 6 (tested on
// all quotients of 12 bits below 8, both signs, in blocks of ten magnitudes from subnormal ones to 2^126).
__device__ __forceinline__ unsigned mx4_codes8(const float* v, unsigned byte)
{
    const float s = mx4_scale(byte);
    unsigned c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
    return byte == kMxNan ? 0u : c;
}

// The values that eight codes stand for.
__device__ __forceinline__ void mx4_values8(unsigned codes, unsigned byte, float* v)
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    const float s = mx4_scale(byte);
    const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
    const v2f c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
    const float nan = __uint_as_float(0x7fc00000u);
    v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
    if (byte == kMxNan)
        for (int i = 0; i < 8; ++i) v[i] = nan;
}

// Maximum over the four lanes of a quad.
__device__ __forceinline__ unsigned quad_max_u32(unsigned v)
{
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));  // quad_perm [1, 0, 3, 2]
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));  // quad_perm [2, 3, 0, 1]
    return v;
}

__device__ __forceinline__ float bf16_to_f32(unsigned short b) { return __uint_as_float((unsigned)b << 16); }

// Round to nearest even; a NaN stays one.
__device__ __forceinline__ unsigned f32_to_bf16x2(float low, float high)
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector((v2f{low, high}), v2b));
}
__device__ __forceinline__ unsigned short f32_to_bf16(float f) { return __builtin_bit_cast(unsigned short, (__bf16)f); }

// The first `left` (at most eight) of eight elements at whatever address, zeros behind them.
__device__ __forceinline__ void load8(const float* p, int left, float* v)
{
    if (left >= 8) {
        __builtin_memcpy(v, p, 32);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void load8(const unsigned short* p, int left, float* v)
{
    if (left >= 8) {
        unsigned a[4];
        __builtin_memcpy(a, p, 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(a[i] << 16), v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? bf16_to_f32(p[i]) : 0.0f;
    }
}

// The largest |v|, as bits.
__device__ __forceinline__ unsigned amax8(const float* v)
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}

}  // namespace q8
