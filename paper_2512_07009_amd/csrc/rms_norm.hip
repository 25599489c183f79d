// rms_norm.hip - root-mean-square norm of rows, its backward pass, and rows in
// 8 bits with a scale each: the norm's output or any features.
//
//   h = x (+ residual, rounded to the type it is kept in)
//   y = h * rstd * weight,  rstd = 1 / sqrt(sum h^2 / width + eps)
//   8 bits: scale = max |y| / 127 over the row, q = y / scale to the nearest, ties to even
//   g = dy * weight, xh = h * rstd
//   dh = rstd * (g - xh * mean(g * xh)) (+ dsum),  dweight = sum over rows of dy * xh
//
// Both passes are bound by memory, and a row is read once and held in registers
// over the lanes that norm_common.h gives it.  In 8 bits y stays in 32 bits up
// to its one rounding: the largest |y| is found over the row's registers, and
// nothing but whole numbers and a scale a row is written.
//
// 128000 x 512 in bfloat16 with a residual: forward 87 us (5.9 TB/s), backward 107
// (4.9), in 8 bits 82 (5.5; a copy of 2 GiB 4.8).  500 rows 3.8.  Wider rows, 64
// million elements, follow the layer norm's shapes.

#include "norm_common.h"
#include "whole.h"

namespace flock {
namespace {

using namespace norm;
using namespace whole;

// Largest |x| over the TPR lanes that share a row, as bits: those of NaN are above
// those of infinity, and both above those of any number.
template <int TPR>
__device__ __forceinline__ uint32_t row_largest(uint32_t x, uint32_t *slot) {
    constexpr int kLanes = TPR < 64 ? TPR : 64;
    x = over_lanes<kLanes>(x, [](uint32_t u, uint32_t v) { return max(u, v); });
    if (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) slot[wave] = x;
        __syncthreads();
        x = max(max(slot[0], slot[1]), max(slot[2], slot[3]));
    }
    return x;
}

// How a row whose largest |y| has these bits goes to 8 bits.  Rows below 2^-100
// are zeros (1 / scale would leave 32 bits), those with values that are not
// finite zeros with a scale of NaN, which every product with them then is.
__device__ __forceinline__ float scale_of(uint32_t largest) {
    const float most = __uint_as_float(largest);
    return largest >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : most >= 0x1p-100f ? most / 127.0f : 0.0f;
}

struct Steps {
    float scale;
    Quotient by;
    int kept;  // bits of a whole number: none of one that is zero by this
    __device__ __forceinline__ explicit Steps(uint32_t largest)
        : scale(scale_of(largest)), by(scale), kept(scale > 0.0f ? -1 : 0) {}
    __device__ __forceinline__ int round(float y) const { return (int)by.rounded(y) & kept; }
    __device__ __forceinline__ int round(float y0, float y1, float y2, float y3) const {
        return bytes(by.rounded(y0), by.rounded(y1), by.rounded(y2), by.rounded(y3)) & kept;
    }
};

template <int N>
__device__ __forceinline__ void store_whole(int8_t *p, int n, const float (&y)[N], const Steps &s) {
    struct __attribute__((packed, aligned(1))) Words { int v[N / 4]; } a;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) a.v[i] = s.round(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
    if (n >= N) {
        *reinterpret_cast<Words *>(p) = a;
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = (int8_t)(a.v[i / 4] >> (8 * (i % 4)));
}

// What is made of a row: its norm in the features' type, in 8 bits, or the row as
// it is in 8 bits.
constexpr int kNormed = 0, kNormedWhole = 1, kWhole = 2;

template <typename T, int VEC, int ITER, int TPR, int FORM>
__global__ void __launch_bounds__(kThreads) rms_kernel(RmsArgs a) {
    __shared__ float sums[4];
    __shared__ uint32_t most[4];
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR;
    if (TPR <= 64 && row >= a.rows) return;  // whole groups of lanes (one row a block otherwise)
    const int width = a.width;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    float h[ITER][VEC];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * TPR + lane) * VEC;
        load_some<T, VEC>(x + c, width - c, h[i]);
    }
    if (FORM != kWhole && a.residual) {
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
    if (FORM != kWhole) {
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sq += h[i][e] * h[i][e];
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(sq, sums) / (float)width + a.eps);
        if (lane == 0 && a.rstd) a.rstd[row] = rstd;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TPR + lane) * VEC;
            if (c < width) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) h[i][e] *= rstd;
                if (a.weight) {
                    float w[VEC];
                    load_some<float, VEC>(a.weight + c, width - c, w);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) h[i][e] *= w[e];
                }
                if (FORM == kNormed) store_some<T, VEC>(static_cast<T *>(a.y) + row * a.y_stride + c, width - c, h[i]);
            }
        }
    }
    if (FORM == kNormed) return;
    // (what lies beyond the row was loaded as zeros)
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < ITER; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) largest = max(largest, magnitude(h[i][e]));
    const Steps steps(row_largest<TPR>(largest, most));
    if (lane == 0) a.scale[row] = steps.scale;
    int8_t *q = static_cast<int8_t *>(a.y) + row * a.y_stride;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * TPR + lane) * VEC;
        if (c < width) store_whole<VEC>(q + c, width - c, h[i], steps);
    }
}

// Rows too wide for registers: the row is read again for each step.
template <typename T, int FORM>
__global__ void __launch_bounds__(kThreads) rms_wide_kernel(RmsArgs a) {
    __shared__ float sums[4];
    __shared__ uint32_t most[4];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    float rstd = 1.0f;
    if (FORM != kWhole) {
        if (a.residual) {
            const T *r = static_cast<const T *>(a.residual) + row * a.residual_stride;
            T *s = static_cast<T *>(a.sum) + row * a.sum_stride;
            for (int c = threadIdx.x; c < a.width; c += kThreads)
                s[c] = static_cast<T>(static_cast<float>(x[c]) + static_cast<float>(r[c]));
            x = s;  // each thread reads back what it wrote itself
        }
        float sq = 0.0f;
        for (int c = threadIdx.x; c < a.width; c += kThreads) sq += static_cast<float>(x[c]) * static_cast<float>(x[c]);
        rstd = 1.0f / sqrtf(row_sum<256>(sq, sums) / (float)a.width + a.eps);
        if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
    }
    const auto value = [&](int c) {
        float o = static_cast<float>(x[c]);
        if (FORM != kWhole) o *= rstd;
        if (FORM != kWhole && a.weight) o *= a.weight[c];
        return o;
    };
    if (FORM == kNormed) {
        T *y = static_cast<T *>(a.y) + row * a.y_stride;
        for (int c = threadIdx.x; c < a.width; c += kThreads) y[c] = static_cast<T>(value(c));
        return;
    }
    uint32_t largest = 0;
    for (int c = threadIdx.x; c < a.width; c += kThreads) largest = max(largest, magnitude(value(c)));
    const Steps steps(row_largest<256>(largest, most));
    if (threadIdx.x == 0) a.scale[row] = steps.scale;
    int8_t *q = static_cast<int8_t *>(a.y) + row * a.y_stride;
    for (int c = threadIdx.x; c < a.width; c += kThreads) q[c] = (int8_t)steps.round(value(c));
}

// Gradient of the rows, and each block's share of the weight's gradient: a block
// takes every gridDim.x-th group of rows, its lanes keep the sums of their own
// columns in registers, and the groups of a block are joined in LDS, in the
// groups' order.  Rows go to blocks by their index alone, so the sums do not
// depend on timing.
template <typename T, int VEC, int ITER, int TPR>
__global__ void __launch_bounds__(kThreads) rms_backward_kernel(RmsBackwardArgs a) {
    constexpr int kGroups = kThreads / TPR;
    __shared__ float sums[2][4];
    __shared__ float joined[TPR < 256 ? kThreads * VEC : 1];
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int width = a.width;
    float dw[ITER][VEC], w[ITER][VEC];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * TPR + lane) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            dw[i][e] = 0.0f;
            w[i][e] = 1.0f;
        }
        if (a.weight) load_some<float, VEC>(a.weight + c, width - c, w[i]);
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kGroups + group; row < a.rows; row += (int64_t)gridDim.x * kGroups) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const T *gy = static_cast<const T *>(a.grad_y) + row * a.grad_y_stride;
        const float rstd = a.rstd[row];
        float xh[ITER][VEC], g[ITER][VEC];
        float s = 0.0f;
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
                xh[i][e] *= rstd;
                dw[i][e] += g[i][e] * xh[i][e];
                g[i][e] *= w[i][e];
                s += g[i][e] * xh[i][e];
            }
        // four waves of a row: the slots of one row are read before the next row but one writes them
        s = row_sum<TPR>(s, sums[turn]) / (float)width;
        turn ^= 1;
        T *dx = static_cast<T *>(a.grad_x) + row * a.grad_x_stride;
        const T *gs = a.grad_sum ? static_cast<const T *>(a.grad_sum) + row * a.grad_sum_stride : nullptr;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * TPR + lane) * VEC;
            if (c < width) {
                float o[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = rstd * (g[i][e] - xh[i][e] * s);
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
    float *part = a.partial + (int64_t)blockIdx.x * width;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        if (kGroups > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < VEC; ++e) joined[threadIdx.x * VEC + e] = dw[i][e];
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    for (int g = 1; g < kGroups; ++g) dw[i][e] += joined[(g * TPR + lane) * VEC + e];
            }
        }
        const int c = (i * TPR + lane) * VEC;
        if (group == 0 && c < width) store_some<float, VEC>(part + c, width - c, dw[i]);
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rms_backward_wide_kernel(RmsBackwardArgs a) {
    __shared__ float sums[4];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *gy = static_cast<const T *>(a.grad_y) + row * a.grad_y_stride;
    const T *gs = a.grad_sum ? static_cast<const T *>(a.grad_sum) + row * a.grad_sum_stride : nullptr;
    T *dx = static_cast<T *>(a.grad_x) + row * a.grad_x_stride;
    const float rstd = a.rstd[row];
    float s = 0.0f;
    for (int c = threadIdx.x; c < a.width; c += kThreads)
        s += static_cast<float>(gy[c]) * (a.weight ? a.weight[c] : 1.0f) * static_cast<float>(x[c]) * rstd;
    s = row_sum<256>(s, sums) / (float)a.width;
    for (int c = threadIdx.x; c < a.width; c += kThreads) {
        const float g = static_cast<float>(gy[c]) * (a.weight ? a.weight[c] : 1.0f);
        float o = rstd * (g - static_cast<float>(x[c]) * rstd * s);
        if (gs) o += static_cast<float>(gs[c]);
        dx[c] = static_cast<T>(o);
    }
}

// The wide rows' shares of the weight's gradient: a thread per column, blockIdx.y
// takes every gridDim.y-th row.
template <typename T>
__global__ void __launch_bounds__(kThreads) rms_columns_kernel(RmsBackwardArgs a) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.width) return;
    float dw = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y)
        dw += static_cast<float>((static_cast<const T *>(a.grad_y) + row * a.grad_y_stride)[c]) *
              (static_cast<float>((static_cast<const T *>(a.x) + row * a.x_stride)[c]) * a.rstd[row]);
    a.partial[(int64_t)blockIdx.y * a.width + c] = dw;
}

template <typename T, int FORM>
hipError_t launch_form(const RmsArgs &a, hipStream_t stream) {
    constexpr int kVec = 16 / (int)sizeof(T);
    return with_shape<kVec>(
            a.width,
            [&](auto iter, auto tpr) {
                constexpr int ITER = decltype(iter)::value, TPR = decltype(tpr)::value;
                return by_parts<T>(a, kThreads / TPR, [&](const RmsArgs &part, dim3 grid) {
                    hipLaunchKernelGGL((rms_kernel<T, kVec, ITER, TPR, FORM>), grid, dim3(kThreads), 0, stream, part);
                });
            },
            [&] {
                return by_parts<T>(a, 1, [&](const RmsArgs &part, dim3 grid) {
                    hipLaunchKernelGGL((rms_wide_kernel<T, FORM>), grid, dim3(kThreads), 0, stream, part);
                });
            });
}

}  // namespace

size_t rms_backward_workspace_bytes(int64_t rows, int32_t width, int n_cus) {
    if (rows <= 0 || width <= 0) return 0;
    return (size_t)std::max(backward_blocks(rows, n_cus), kWideShares) * (size_t)width * sizeof(float);
}

hipError_t launch_rms(const RmsArgs &a, int32_t dtype, hipStream_t stream) {
    return with_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        if (a.as_is) return launch_form<T, kWhole>(a, stream);
        return a.scale ? launch_form<T, kNormedWhole>(a, stream) : launch_form<T, kNormed>(a, stream);
    });
}

hipError_t launch_rms_backward(RmsBackwardArgs a, int32_t dtype, void *workspace, int n_cus, float *grad_weight,
                               hipStream_t stream) {
    a.partial = grad_weight ? static_cast<float *>(workspace) : nullptr;
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
                    hipLaunchKernelGGL((rms_backward_kernel<T, kVec, ITER, TPR>), dim3(shares), dim3(kThreads), 0, stream, a);
                    return hipGetLastError();
                },
                [&] {
                    hipError_t e = by_parts<T>(a, 1, [&](const RmsBackwardArgs &part, dim3 grid) {
                        hipLaunchKernelGGL((rms_backward_wide_kernel<T>), grid, dim3(kThreads), 0, stream, part);
                    });
                    if (e != hipSuccess || !a.partial) return e;
                    shares = (int)std::min<int64_t>(kWideShares, a.rows);
                    hipLaunchKernelGGL((rms_columns_kernel<T>), dim3((a.width + kThreads - 1) / kThreads, shares),
                                       dim3(kThreads), 0, stream, a);
                    return hipGetLastError();
                });
    });
    if (err != hipSuccess || !grad_weight) return err;
    hipLaunchKernelGGL(columns_kernel, dim3((a.width + 15) / 16), dim3(1024), 0, stream, a.partial, shares, a.width, a.width,
                       grad_weight, static_cast<float *>(nullptr));
    return hipGetLastError();
}

}  // namespace flock
