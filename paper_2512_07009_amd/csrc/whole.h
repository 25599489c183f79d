// whole.h - numbers in 8 bits with a scale, as the norm and the pages of tracks
// make them.
#ifndef FLOCK_WHOLE_H
#define FLOCK_WHOLE_H

#include "encoder_common.h"

namespace flock {
namespace whole {

// |x| as bits, in the order of the numbers: infinity above all of them, NaN above it.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// How numbers go to whole ones: x / scale in 32 bits, rounded as a division is, and that to
// the nearest, ties to even.  A product with 1 / scale alone would take x on either side where
// x / scale is a half (16-bit numbers of half their row's largest, 63.5, are), so its remainder
// goes over it once more.  |x / scale| is below 128.
struct Quotient {
    float scale, per;
    __device__ __forceinline__ explicit Quotient(float scale) : scale(scale), per(scale > 0.0f ? 1.0f / scale : 0.0f) {}
    // As the low byte of a sum with 1.5 x 2^23.
    __device__ __forceinline__ uint32_t rounded(float x) const {
        const float q = x * per;
        return __float_as_uint(__builtin_fmaf(__builtin_fmaf(-q, scale, x), per, q) + 12582912.0f);
    }
};

// A whole number times a quotient of scales to the nearest, likewise.
__device__ __forceinline__ uint32_t rounded_again(float whole, float quotient) {
    return __float_as_uint(__builtin_fmaf(whole, quotient, 12582912.0f));
}

// Four low bytes in one word.
__device__ __forceinline__ int bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return (int)__builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

}  // namespace whole
}  // namespace flock

#endif  // FLOCK_WHOLE_H
