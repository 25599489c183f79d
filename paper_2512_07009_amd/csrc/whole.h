// whole.h - numbers in 8 bits with a scale, as the norm and the pages of tracks
// make them.
#ifndef FLOCK_WHOLE_H
#define FLOCK_WHOLE_H

#include "encoder_common.h"

namespace flock {
namespace whole {

// |x| as bits, in the order of the numbers: infinity above all of them, NaN above it.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// x / scale to the nearest whole number, ties to even, given 1 / scale: the low byte of
// what is left of x / scale beside 1.5 x 2^23 (|x / scale| is below 128).
__device__ __forceinline__ uint32_t rounded(float x, float per) { return __float_as_uint(__builtin_fmaf(x, per, 12582912.0f)); }

// Four low bytes in one word.
__device__ __forceinline__ int bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return (int)__builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

}  // namespace whole
}  // namespace flock

#endif  // FLOCK_WHOLE_H
