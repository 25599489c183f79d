// linear_common.h - the LDS of 8-bit products in tiles: stages of rows' bytes,
// and where in them waves put the outputs that they store.
#ifndef FLOCK_LINEAR_COMMON_H
#define FLOCK_LINEAR_COMMON_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace flock {
namespace linear {

constexpr int kStep = 128, kAhead = 1, kStages = kAhead + 1, kChunks = kStep / 16;

template <int BM, int BN>
struct __attribute__((aligned(16))) LinearShared {
    int8_t x[kStages][BM * kStep], w[kStages][BN * kStep];
    float x_scale[kStages][BM], w_scale[kStages][BN], bias[kStages][BN];  // of tiles in turn: a tile may be one step
};

// Bytes that a wave's outputs of 16 bits go through: 32 rows of 32 KN.
template <int KN>
constexpr int kRoom = 32 * 32 * KN * 2;

// A wave's own room of four in a stage that nobody multiplies: two in the rows' part of it,
// two in the weights'.  Each lies within its part, so none reaches into a stage beside it.
template <int KN, int BM, int BN>
__host__ __device__ inline int8_t *stage_room(LinearShared<BM, BN> &s, int stage, int wave) {
    static_assert(2 * kRoom<KN> <= BM * kStep && 2 * kRoom<KN> <= BN * kStep, "two rooms in each part of a stage");
    return (wave < 2 ? s.x[stage] : s.w[stage]) + (wave & 1) * kRoom<KN>;
}

}  // namespace linear
}  // namespace flock

#endif  // FLOCK_LINEAR_COMMON_H
