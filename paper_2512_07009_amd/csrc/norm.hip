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

#include "norm_common.h"

namespace flock {
namespace {

using namespace norm;

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
    hipLaunchKernelGGL(columns_kernel, dim3((2 * a.width + 15) / 16), dim3(1024), 0, stream, a.partial, shares,
                       2 * a.width, a.width, grad_weight, grad_bias);
    return hipGetLastError();
}

}  // namespace flock
