// Microscaled 4-bit floating point on the device: blocks of 32 values, e2m1 codes, one power of two each.
#pragma once
#include "vq_types.h"

namespace vq {

constexpr int kMxBlock = 32;
constexpr int kMxNan = 255;      // the scale of a block with a value that is not finite

__host__ __device__ __forceinline__ int mx_scale_stride(int K) { return (K / kMxBlock + 3) / 4 * 4; }

// Magnitude bits of a float: they order like the magnitudes, infinity and NaN above every number.
__device__ __forceinline__ unsigned magnitude(float t) { return __builtin_bit_cast(unsigned, t) & 0x7FFFFFFFu; }

// The scale's byte from the largest magnitude of the block: floor(log2) is the float's exponent, 2 less is that of
// a block whose largest code is 4 or 6.  Numbers below 2^-126 count as that small (byte 0 is 2^-127 in any case).
__device__ __forceinline__ int mx_scale_of(unsigned top) {
    const int e = (int)(top >> 23);
    return e == 255 ? kMxNan : max(e - 2, 0);
}

// Four neighbouring lanes hold a block: the largest of their numbers.
__device__ __forceinline__ unsigned largest_of_block(unsigned top) {
    top = max(top, (unsigned)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true));          // the neighbour's
    return max(top, (unsigned)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true));         // the other pair's
}

// Eight values of a block as codes, the first in the lowest bits.  The conversion divides by the power of two in
// `scale`'s exponent, rounds to nearest even and saturates.
__device__ __forceinline__ unsigned mx_encode(const float* t, int byte) {
    const float scale = __builtin_bit_cast(float, byte << 23);
    unsigned d = 0;
    d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, t[0], t[1], scale, 0);
    d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, t[2], t[3], scale, 1);
    d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, t[4], t[5], scale, 2);
    d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, t[6], t[7], scale, 3);
    return byte == kMxNan ? 0 : d;
}

}  // namespace vq
