// 16-byte vectors of operand rows that may start at any byte and end anywhere, shared by the kernels that load operands through registers.
#pragma once
#include "q8_device.h"

namespace q8 {

__device__ __forceinline__ v4i load16_any(const int8_t* p)
{
    v4i v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// 16 bytes at p of which the first `left` belong to the row (none if left <= 0), zeros behind them.  The row is K bytes
// long and ends at p + left; nothing outside it is read: a vector that would end behind the row starts earlier instead,
// and the bytes in front of p are shifted out (rows of less than 16 bytes: the same with words, less than 4: bytes).
__device__ __forceinline__ v4i load16_bounded(const int8_t* p, int left, int K)
{
    v4i v = {0, 0, 0, 0};
    if (K >= 16) {
        unsigned __int128 u;
        __builtin_memcpy(&u, p + min(left - 16, 0), 16);
        const int drop = max(16 - left, 0);
        u = drop < 16 ? u >> (8 * drop) : 0;
        __builtin_memcpy(&v, &u, 16);
    } else if (left > 0 && K >= 4) {  // the row's only chunk: left = K
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const int rest = K - 4 * d;  // bytes of the row from word d on
            unsigned u;
            __builtin_memcpy(&u, p + 4 * d + min(rest - 4, 0), 4);
            const int drop = max(4 - rest, 0);
            v[d] = drop < 4 ? (int)(u >> (8 * drop)) : 0;
        }
    } else if (left > 0) {
#pragma unroll
        for (int j = 0; j < 3; ++j) v[0] |= (j < K ? (int)(unsigned char)p[min(j, K - 1)] : 0) << (8 * j);
    }
    return v;
}

}  // namespace q8
