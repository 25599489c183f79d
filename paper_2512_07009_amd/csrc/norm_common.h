// norm_common.h - what the norms of rows share: sums over a row's lanes, the
// shapes of rows, launches by parts, and the joining of the blocks' shares of
// the weights' gradients.
#ifndef FLOCK_NORM_COMMON_H
#define FLOCK_NORM_COMMON_H

#include <algorithm>
#include <type_traits>

#include "encoder_common.h"

namespace flock {
namespace norm {

constexpr int kThreads = 256;

// Sum over the TPR lanes that share a row; every lane gets it.  slot: LDS for
// the four waves' sums (TPR = 256), a different one in each of the calls
// between two barriers.
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float *slot) {
    constexpr int kLanes = TPR < 64 ? TPR : 64;
    x = over_lanes<kLanes>(x, [](float u, float v) { return u + v; });
    if (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) slot[wave] = x;
        __syncthreads();
        x = (slot[0] + slot[1]) + (slot[2] + slot[3]);
    }
    return x;
}

// Sum of the blocks' shares [n][columns] (the weights' gradients, then the biases' from
// column `width` on), in a fixed order: 16 columns a block, 64 lanes of shares each, 5 us
// for 1024 shares of 512 columns (64 columns and 16 lanes: 16 workgroups, 20 us).
static __global__ void __launch_bounds__(1024) columns_kernel(const float *partial, int n, int columns, int width,
                                                              float *dw, float *db) {
    __shared__ float part[64][16];
    const int lane = threadIdx.x & 15, share = threadIdx.x >> 4;
    const int c = blockIdx.x * 16 + lane;
    float s = 0.0f;
    if (c < columns) {
#pragma unroll 4
        for (int i = share; i < n; i += 64) s += partial[(int64_t)i * columns + c];
    }
    part[share][lane] = s;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        __syncthreads();
        if (share < d) part[share][lane] += part[share + d][lane];
    }
    if (share != 0 || c >= columns) return;
    if (c < width) {
        if (dw) dw[c] = part[0][lane];
    } else if (db) {
        db[c - width] = part[0][lane];
    }
}

// fn(ITER, TPR) for a row of `width`: TPR lanes a row, ITER packs a lane.  A pack a
// lane up to a wave (the fewest lanes of 8, 16, 32 and 64), then 2 or 4 packs a lane
// of a wave, then of four waves; wide() above 4 packs x 256 lanes.  2 or 3 packs over
// 32 lanes instead were slower (30000 rows of 333 fp32 64 -> 69 us with the backward
// pass).  64 million bfloat16 elements, forward and backward: rows of 1500 300 us, of
// 2048 230, of 6000 280, of 20000 (wide) 558; the bytes alone take 126.
template <int VEC, typename F, typename W>
hipError_t with_shape(int32_t width, F &&fn, W &&wide) {
    const int packs = (width + VEC - 1) / VEC;
    if (packs <= 8) return fn(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{});
    if (packs <= 16) return fn(std::integral_constant<int, 1>{}, std::integral_constant<int, 16>{});
    if (packs <= 32) return fn(std::integral_constant<int, 1>{}, std::integral_constant<int, 32>{});
    if (packs <= 64) return fn(std::integral_constant<int, 1>{}, std::integral_constant<int, 64>{});
    if (packs <= 128) return fn(std::integral_constant<int, 2>{}, std::integral_constant<int, 64>{});
    if (packs <= 256) return fn(std::integral_constant<int, 4>{}, std::integral_constant<int, 64>{});
    if (packs <= 512) return fn(std::integral_constant<int, 2>{}, std::integral_constant<int, 256>{});
    if (packs <= 1024) return fn(std::integral_constant<int, 4>{}, std::integral_constant<int, 256>{});
    return wide();
}

// launch(part, blocks) over the rows of a, by as many as a launch holds.  Parts
// begin at a group of rows, so that a row gets the same lanes in any of them.
template <typename T, typename A, typename F>
hipError_t by_parts(A a, int rows_per_block, F &&launch) {
    const int64_t rows = a.rows, most = kMaxWorkgroups * rows_per_block;
    hipError_t err = hipSuccess;
    for (int64_t first = 0; first < rows && err == hipSuccess; first += most) {
        A part = a;
        part.rows = std::min(rows - first, most);
        part.advance(first, sizeof(T));
        launch(part, dim3((uint32_t)((part.rows + rows_per_block - 1) / rows_per_block)));
        err = hipGetLastError();
    }
    return err;
}

constexpr int kWideShares = 64;

// Blocks of the backward pass: enough to fill the card (four of 256 threads a
// compute unit; with 4 packs of 16-bit elements a lane registers let two of them
// run at a time, the others follow), and each block's share of the weight's gradient
// is one row of the workspace, 4 MB at 512 columns beside the 524 MB of the case above.
inline int backward_blocks(int64_t rows, int n_cus) {
    const int64_t blocks = (rows + 3) / 4;
    return (int)std::min<int64_t>(std::max<int64_t>(blocks, 1), 4 * (int64_t)n_cus);
}

}  // namespace norm
}  // namespace flock

#endif  // FLOCK_NORM_COMMON_H
