// norm.hip - layer norm of rows (a bird's features each) and its backward
// pass, with the reduction of the weight's and bias's gradients.
//
//   h = x (+ residual, rounded to the type it is kept in)
//   y = (h - mean) * rstd * weight + bias,  rstd = 1 / sqrt(var + eps)
//   g = dy * weight, xh = (h - mean) * rstd
//   dh = rstd * (g - mean(g) - xh * mean(g * xh)) (+ dsum)
//   dweight = sum over rows of dy * xh,  dbias = sum over rows of dy
//
// Both passes are bound by memory: a row is read once, held in registers, and
// its statistics are taken there in 32 bits (the variance from the centred
// values, so that a large mean costs no digits).  TPR lanes share a row, a
// part of a wave for narrow rows and four waves for wide ones.  128000 rows of
// 512 in bfloat16 with residual: forward 96 us (5.5 TB/s), backward 106 us
// (5.0 TB/s) and 4 us for the columns' sums; 500 rows: 3.7 us, less than a call
// takes on the host.

#include "encoder_common.h"

namespace flock {
namespace {

constexpr int kThreads = 256;

// Sum over the TPR lanes that share a row; every lane gets it.  slot: LDS for
// the four waves' sums (TPR = 256), a different one in each of the calls
// between two barriers.
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float *slot) {
    constexpr int kLanes = TPR < 64 ? TPR : 64;
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) x += __shfl_xor(x, d);
    if (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) slot[wave] = x;
        __syncthreads();
        x = (slot[0] + slot[1]) + (slot[2] + slot[3]);
    }
    return x;
}

template <typename T, int VEC, int ITER, int TPR>
__global__ void __launch_bounds__(kThreads) norm_kernel(NormArgs a) {
    __shared__ float sums[2][4];
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR;
    if (TPR <= 64 && row >= a.rows) return;  // whole groups of lanes (one row a block otherwise)
    const int width = a.width;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    float h[ITER][VEC];
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * TPR + lane) * VEC;
        load_some<T, VEC>(x + c, width - c, h[i]);
    }
    if (a.residual) {
        const T *r = static_cast<const T *>(a.residual) + row * a.residual_stride;
        T *s = static_cast<T *>(a.sum) + row * a.sum_stride;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TPR + lane) * VEC;
            float t[VEC];
            load_some<T, VEC>(r + c, width - c, t);
            // what is normalised is the sum as it is kept
#pragma unroll
            for (int e = 0; e < VEC; ++e) h[i][e] = static_cast<float>(static_cast<T>(h[i][e] + t[e]));
            store_some<T, VEC>(s + c, width - c, h[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) total += h[i][e];
    const float mean = row_sum<TPR>(total, sums[0]) / (float)width;
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * TPR + lane) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            h[i][e] -= mean;
            if (c + e < width) sq += h[i][e] * h[i][e];
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(sq, sums[1]) / (float)width + a.eps);
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * TPR + lane) * VEC;
        if (c < width) {
            float w[VEC], o[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] = h[i][e] * rstd;
            if (a.weight) {
                load_some<float, VEC>(a.weight + c, width - c, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] *= w[e];
            }
            if (a.bias) {
                load_some<float, VEC>(a.bias + c, width - c, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] += w[e];
            }
            store_some<T, VEC>(y + c, width - c, o);
        }
    }
}

// Rows too wide for registers: the row is read again for each step.
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_wide_kernel(NormArgs a) {
    __shared__ float sums[2][4];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    if (a.residual) {
        const T *r = static_cast<const T *>(a.residual) + row * a.residual_stride;
        T *s = static_cast<T *>(a.sum) + row * a.sum_stride;
        for (int c = threadIdx.x; c < a.width; c += kThreads)
            s[c] = static_cast<T>(static_cast<float>(x[c]) + static_cast<float>(r[c]));
        x = s;  // each thread reads back what it wrote itself
    }
    float total = 0.0f;
    for (int c = threadIdx.x; c < a.width; c += kThreads) total += static_cast<float>(x[c]);
    const float mean = row_sum<256>(total, sums[0]) / (float)a.width;
    float sq = 0.0f;
    for (int c = threadIdx.x; c < a.width; c += kThreads) {
        const float d = static_cast<float>(x[c]) - mean;
        sq += d * d;
    }
    const float rstd = 1.0f / sqrtf(row_sum<256>(sq, sums[1]) / (float)a.width + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    for (int c = threadIdx.x; c < a.width; c += kThreads) {
        float o = (static_cast<float>(x[c]) - mean) * rstd;
        if (a.weight) o *= a.weight[c];
        if (a.bias) o += a.bias[c];
        y[c] = static_cast<T>(o);
    }
}

// Gradient of the rows, and each block's share of the weight's and bias's
// gradients: a block takes every gridDim.x-th group of rows, its lanes keep
// the sums of their own columns in registers, and the groups of a block are
// joined in LDS, in the groups' order.  Rows go to blocks by their index
// alone, so the sums do not depend on timing.
template <typename T, int VEC, int ITER, int TPR>
__global__ void __launch_bounds__(kThreads) norm_backward_kernel(NormBackwardArgs a) {
    constexpr int kGroups = kThreads / TPR;
    __shared__ float sums[2][2][4];
    __shared__ float joined[TPR < 256 ? kThreads * VEC : 1];
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int width = a.width;
    float dw[ITER][VEC], db[ITER][VEC], w[ITER][VEC];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * TPR + lane) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            dw[i][e] = db[i][e] = 0.0f;
            w[i][e] = 1.0f;
        }
        if (a.weight) load_some<float, VEC>(a.weight + c, width - c, w[i]);
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kGroups + group; row < a.rows; row += (int64_t)gridDim.x * kGroups) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const T *gy = static_cast<const T *>(a.grad_y) + row * a.grad_y_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float xh[ITER][VEC], g[ITER][VEC];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TPR + lane) * VEC;
            load_some<T, VEC>(x + c, width - c, xh[i]);
            load_some<T, VEC>(gy + c, width - c, g[i]);  // zeros beyond the row: nothing there counts
        }
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                xh[i][e] = (xh[i][e] - mean) * rstd;
                dw[i][e] += g[i][e] * xh[i][e];
                db[i][e] += g[i][e];
                g[i][e] *= w[i][e];
                s1 += g[i][e];
                s2 += g[i][e] * xh[i][e];
            }
        // four waves of a row: the slots of one row are read before the next row but one writes them
        s1 = row_sum<TPR>(s1, sums[turn][0]) / (float)width;
        s2 = row_sum<TPR>(s2, sums[turn][1]) / (float)width;
        turn ^= 1;
        T *dx = static_cast<T *>(a.grad_x) + row * a.grad_x_stride;
        const T *gs = a.grad_sum ? static_cast<const T *>(a.grad_sum) + row * a.grad_sum_stride : nullptr;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TPR + lane) * VEC;
            if (c < width) {
                float o[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = rstd * (g[i][e] - s1 - xh[i][e] * s2);
                if (gs) {
                    float t[VEC];
                    load_some<T, VEC>(gs + c, width - c, t);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) o[e] += t[e];
                }
                store_some<T, VEC>(dx + c, width - c, o);
            }
        }
    }
    if (!a.partial) return;
    float *part = a.partial + (int64_t)blockIdx.x * 2 * width;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float(&d)[VEC] = which ? db[i] : dw[i];
            if (kGroups > 1) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < VEC; ++e) joined[threadIdx.x * VEC + e] = d[e];
                __syncthreads();
                if (group == 0) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        for (int g = 1; g < kGroups; ++g) d[e] += joined[(g * TPR + lane) * VEC + e];
                }
            }
            const int c = (i * TPR + lane) * VEC;
            if (group == 0 && c < width) {
                store_some<float, VEC>(part + (int64_t)which * width + c, width - c, d);
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) norm_backward_wide_kernel(NormBackwardArgs a) {
    __shared__ float sums[2][4];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *gy = static_cast<const T *>(a.grad_y) + row * a.grad_y_stride;
    const T *gs = a.grad_sum ? static_cast<const T *>(a.grad_sum) + row * a.grad_sum_stride : nullptr;
    T *dx = static_cast<T *>(a.grad_x) + row * a.grad_x_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < a.width; c += kThreads) {
        const float g = static_cast<float>(gy[c]) * (a.weight ? a.weight[c] : 1.0f);
        s1 += g;
        s2 += g * (static_cast<float>(x[c]) - mean) * rstd;
    }
    s1 = row_sum<256>(s1, sums[0]) / (float)a.width;
    s2 = row_sum<256>(s2, sums[1]) / (float)a.width;
    for (int c = threadIdx.x; c < a.width; c += kThreads) {
        const float g = static_cast<float>(gy[c]) * (a.weight ? a.weight[c] : 1.0f);
        const float xh = (static_cast<float>(x[c]) - mean) * rstd;
        float o = rstd * (g - s1 - xh * s2);
        if (gs) o += static_cast<float>(gs[c]);
        dx[c] = static_cast<T>(o);
    }
}

// The wide rows' shares of the weight's and bias's gradients: a thread per
// column, blockIdx.y takes every gridDim.y-th row.
template <typename T>
__global__ void __launch_bounds__(kThreads) norm_columns_kernel(NormBackwardArgs a) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.width) return;
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float g = static_cast<float>((static_cast<const T *>(a.grad_y) + row * a.grad_y_stride)[c]);
        const float x = static_cast<float>((static_cast<const T *>(a.x) + row * a.x_stride)[c]);
        dw += g * ((x - a.mean[row]) * a.rstd[row]);
        db += g;
    }
    a.partial[(int64_t)blockIdx.y * 2 * a.width + c] = dw;
    a.partial[(int64_t)blockIdx.y * 2 * a.width + a.width + c] = db;
}

// Sum of the blocks' shares, in a fixed order: 16 columns a block, 64 lanes of
// shares each (64 columns and 16 lanes: 16 workgroups for 512 columns, 20 us for
// 1024 shares).
__global__ void __launch_bounds__(1024) norm_reduce_kernel(const float *partial, int n, int width, float *dw,
                                                           float *db) {
    __shared__ float part[64][16];
    const int lane = threadIdx.x & 15, share = threadIdx.x >> 4;
    const int c = blockIdx.x * 16 + lane;
    float s = 0.0f;
    if (c < 2 * width) {
#pragma unroll 4
        for (int i = share; i < n; i += 64) s += partial[(int64_t)i * 2 * width + c];
    }
    part[share][lane] = s;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        __syncthreads();
        if (share < d) part[share][lane] += part[share + d][lane];
    }
    if (share != 0 || c >= 2 * width) return;
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
int backward_blocks(int64_t rows, int n_cus) {
    const int64_t blocks = (rows + 3) / 4;
    return (int)std::min<int64_t>(std::max<int64_t>(blocks, 1), 4 * (int64_t)n_cus);
}

}  // namespace

size_t norm_backward_workspace_bytes(int64_t rows, int32_t width, int n_cus) {
    if (rows <= 0 || width <= 0) return 0;
    const int64_t shares = std::max(backward_blocks(rows, n_cus), kWideShares);
    return (size_t)shares * 2 * (size_t)width * sizeof(float);
}

hipError_t launch_norm(const NormArgs &a, int32_t dtype, hipStream_t stream) {
    return with_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        constexpr int kVec = 16 / (int)sizeof(T);
        return with_shape<kVec>(
                a.width,
                [&](auto iter, auto tpr) {
                    constexpr int ITER = decltype(iter)::value, TPR = decltype(tpr)::value;
                    return by_parts<T>(a, kThreads / TPR, [&](const NormArgs &part, dim3 grid) {
                        hipLaunchKernelGGL((norm_kernel<T, kVec, ITER, TPR>), grid, dim3(kThreads), 0, stream, part);
                    });
                },
                [&] {
                    return by_parts<T>(a, 1, [&](const NormArgs &part, dim3 grid) {
                        hipLaunchKernelGGL((norm_wide_kernel<T>), grid, dim3(kThreads), 0, stream, part);
                    });
                });
    });
}

hipError_t launch_norm_backward(NormBackwardArgs a, int32_t dtype, void *workspace, int n_cus, float *grad_weight,
                                float *grad_bias, hipStream_t stream) {
    a.partial = grad_weight || grad_bias ? static_cast<float *>(workspace) : nullptr;
    int shares = a.rows > 0 ? backward_blocks(a.rows, n_cus) : 0;
    hipError_t err = a.rows == 0 ? hipSuccess : with_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        constexpr int kVec = 16 / (int)sizeof(T);
        return with_shape<kVec>(
                a.width,
                [&](auto iter, auto tpr) {
                    constexpr int ITER = decltype(iter)::value, TPR = decltype(tpr)::value;
                    constexpr int kRows = kThreads / TPR;
                    shares = (int)std::min<int64_t>(shares, (a.rows + kRows - 1) / kRows);
                    hipLaunchKernelGGL((norm_backward_kernel<T, kVec, ITER, TPR>), dim3(shares), dim3(kThreads), 0,
                                       stream, a);
                    return hipGetLastError();
                },
                [&] {
                    hipError_t e = by_parts<T>(a, 1, [&](const NormBackwardArgs &part, dim3 grid) {
                        hipLaunchKernelGGL((norm_backward_wide_kernel<T>), grid, dim3(kThreads), 0, stream, part);
                    });
                    if (e != hipSuccess || !a.partial) return e;
                    shares = (int)std::min<int64_t>(kWideShares, a.rows);
                    hipLaunchKernelGGL((norm_columns_kernel<T>), dim3((a.width + kThreads - 1) / kThreads, shares),
                                       dim3(kThreads), 0, stream, a);
                    return hipGetLastError();
                });
    });
    if (err != hipSuccess || !(grad_weight || grad_bias)) return err;
    hipLaunchKernelGGL(norm_reduce_kernel, dim3((2 * a.width + 15) / 16), dim3(1024), 0, stream, a.partial, shares,
                       a.width, grad_weight, grad_bias);
    return hipGetLastError();
}

}  // namespace flock
