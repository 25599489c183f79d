// linear.hip - products of rows in 8 bits with weights in 8 bits, a scale for
// each row and each output:
//
//   y[m, n] = act(x_scale[m] * w_scale[n] * sum_k x[m, k] w[n, k] + bias[n])
//
// Sums are whole numbers of 32 bits on the matrix cores, exact up to a width of
// 2^17 - 1, so they do not depend on their order; what follows is in 32 bits with
// one rounding to the output's type.

#include "encoder_common.h"

namespace flock {
namespace {

constexpr int kThreads = 256;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// 16 bytes of a row from `k` on, zeros beyond its width.
__device__ __forceinline__ i32x4 load_chunk(const int8_t *row, int k, int width) {
    if (k + 16 <= width) {
        const Pack<int8_t, 16> a = *reinterpret_cast<const Pack<int8_t, 16> *>(row + k);
        return __builtin_bit_cast(i32x4, a);
    }
    i32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int b = 0; b < 16; ++b)
        if (k + b < width) v[b / 4] |= (int)(uint8_t)row[k + b] << (8 * (b % 4));
    return v;
}

// x Phi(x), Phi the normal distribution.  With z = |x| / sqrt 2 and t = 1 / (1 + 0.51 z),
// e^(z^2) erfc(z) / t is a polynomial of t to 9e-7 of itself (fitted to erfc over z <= 10, 7
// terms; 6 are off by 5e-6), so that the tail of negative x keeps its digits: 6.5e-6 of the
// result in all, against 3.9e-3 for half a step of bfloat16.  The library's erfc takes some
// three times the instructions, which the products do not cover.
__device__ __forceinline__ float gelu(float x) {
    const float z = fabsf(x);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.36062445840513924f, z, 1.0f));
    float p = 0.047249945f;
    p = __builtin_fmaf(p, t, -0.1795673f);
    p = __builtin_fmaf(p, t, 0.17922265f);
    p = __builtin_fmaf(p, t, 0.027526545f);
    p = __builtin_fmaf(p, t, 0.13953302f);
    p = __builtin_fmaf(p, t, 0.142076165f);
    p = __builtin_fmaf(p, t, 0.14395875f);
    const float tail = p * t * __builtin_amdgcn_exp2f(x * x * -0.72134752044448170368f);  // 1 - Phi(|x|)
    return __builtin_fmaf(-z, tail, fmaxf(x, 0.0f));
}

// ---------------------------------------------------------------------------
// Many rows: BM x BN outputs a workgroup, a quarter of them a wave.
//
// The weights are the left factor (32 outputs), the rows the right one (32 rows),
// so that a lane holds four outputs of one row side by side.  Tiles of BK bytes of
// every row go to LDS without registers in between (16 bytes a lane), one while the
// one before is multiplied, with one barrier a tile.  A row's chunks of 16 bytes are
// stored in an order that turns with the row, so that the 32 rows that a wave reads
// a chunk of lie in different banks.
// ---------------------------------------------------------------------------

template <int BK>
__device__ __forceinline__ int turned(int row, int chunk) {
    return BK == 128 ? chunk ^ (row & 7) : chunk ^ ((row >> 1) & 3);
}

// A tile of ROWS rows: where its lanes load from, in the order in which they store.
template <int ROWS, int BK>
struct Loader {
    static constexpr int kChunks = BK / 16, kLoads = ROWS * kChunks / kThreads;
    const int8_t *base;
    int left;               // rows there are
    uint32_t at[kLoads];    // of the lane's chunk, from base
    uint32_t pitch;

    __device__ __forceinline__ Loader(const int8_t *p, int64_t stride, int rows) {
        base = p;
        left = rows;
        pitch = (uint32_t)stride;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int slot = i * kThreads + threadIdx.x, row = slot / kChunks;
            // (rows beyond the last are the last: what they give is not stored)
            at[i] = (uint32_t)min(row, left - 1) * pitch + 16u * turned<BK>(row, slot % kChunks);
        }
    }

    __device__ __forceinline__ void direct(int8_t *tile, int k0) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void *)(base + k0 + at[i]),
                    (__attribute__((address_space(3))) void *)(tile + 16 * (i * kThreads + 64 * wave)), 16, 0, 0);
    }

    // The row's end, or rows that do not begin at 16 bytes.
    __device__ __forceinline__ void by_registers(int8_t *tile, int k0, int width) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int slot = i * kThreads + threadIdx.x, row = slot / kChunks;
            const int8_t *p = base + (uint32_t)min(row, left - 1) * pitch;
            *reinterpret_cast<i32x4 *>(tile + 16 * slot) = load_chunk(p, k0 + 16 * turned<BK>(row, slot % kChunks), width);
        }
    }
};

template <typename T, int BM, int BN, int BK>
__global__ void __launch_bounds__(kThreads, 2) linear_kernel(LinearArgs a) {
    constexpr int kMT = BM / 64, kNT = BN / 64;      // 32 x 32 parts of a wave
    constexpr int kPitch = 32 * kNT + 16 / (int)sizeof(T);
    constexpr int kTiles = 2 * (BM + BN) * BK, kStage = 4 * 32 * kPitch * (int)sizeof(T);
    __shared__ __attribute__((aligned(16))) int8_t shared[kTiles > kStage ? kTiles : kStage];
    __shared__ float scales[2][BN];

    const int64_t tile = blockIdx.x;
    const int64_t m0 = tile / a.column_tiles * BM;
    const int n0 = (int)(tile % a.column_tiles) * BN;
    const int rows = (int)min((int64_t)BM, a.rows - m0), columns = min(BN, a.outputs - n0);
    for (int i = threadIdx.x; i < BN; i += kThreads) {
        scales[0][i] = i < columns ? a.w_scale[n0 + i] : 0.0f;
        scales[1][i] = i < columns && a.bias ? a.bias[n0 + i] : 0.0f;
    }
    const Loader<BM, BK> load_x(a.x + m0 * a.x_stride, a.x_stride, rows);
    const Loader<BN, BK> load_w(a.w + n0 * a.w_stride, a.w_stride, columns);
    const auto fetch = [&](int t) {
        int8_t *x = shared + (t & 1) * (BM + BN) * BK, *w = x + BM * BK;
        const int k0 = t * BK;
        if (a.aligned && k0 + BK <= a.width) {
            load_x.direct(x, k0);
            load_w.direct(w, k0);
        } else {
            load_x.by_registers(x, k0, a.width);
            load_w.by_registers(w, k0, a.width);
        }
    };

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, col = lane & 31;
    const int wm = (wave & 1) * (BM / 2), wn = (wave >> 1) * (BN / 2);
    i32x16 acc[kNT][kMT] = {};
    const int steps = (a.width + BK - 1) / BK;
    fetch(0);
    for (int t = 0; t < steps; ++t) {
        __syncthreads();  // this tile is there, and the one before has been read
        if (t + 1 < steps) fetch(t + 1);
        const int8_t *x = shared + (t & 1) * (BM + BN) * BK, *w = x + BM * BK;
#pragma unroll
        for (int k = 0; k < BK / 32; ++k) {
            i32x4 wf[kNT], xf[kMT];
#pragma unroll
            for (int i = 0; i < kNT; ++i) {
                const int row = wn + 32 * i + col;
                wf[i] = *reinterpret_cast<const i32x4 *>(w + row * BK + 16 * turned<BK>(row, 2 * k + h));
            }
#pragma unroll
            for (int j = 0; j < kMT; ++j) {
                const int row = wm + 32 * j + col;
                xf[j] = *reinterpret_cast<const i32x4 *>(x + row * BK + 16 * turned<BK>(row, 2 * k + h));
            }
#pragma unroll
            for (int i = 0; i < kNT; ++i)
#pragma unroll
                for (int j = 0; j < kMT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[i], xf[j], acc[i][j], 0, 0, 0);
        }
    }
    __syncthreads();  // the tiles' memory is free

    // by 32 rows of a wave through LDS, so that a row's outputs are stored side by side
    T *stage = reinterpret_cast<T *>(shared) + wave * 32 * kPitch;
    constexpr int kVec = 16 / (int)sizeof(T), kLanes = 32 * kNT / kVec;  // of a row
#pragma unroll
    for (int j = 0; j < kMT; ++j) {
        const int m = wm + 32 * j + col;
        const float xs = m < rows ? a.x_scale[m0 + m] : 0.0f;
#pragma unroll
        for (int i = 0; i < kNT; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int n = 32 * i + 2 * r + 4 * h;
                float o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[e] = (float)acc[i][j][r + e] * xs * scales[0][wn + n + e] + scales[1][wn + n + e];
                    if (a.gelu) o[e] = gelu(o[e]);
                }
                store_pack<T, 4>(stage + col * kPitch + n, o);
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 32 * kLanes / 64; ++i) {
            const int part = i * 64 + lane, row = part / kLanes, n = part % kLanes * kVec;
            const int left = columns - wn - n;
            if (wm + 32 * j + row < rows && left > 0) {
                T *y = static_cast<T *>(a.y) + (m0 + wm + 32 * j + row) * a.y_stride + n0 + wn + n;
                const T *s = stage + row * kPitch + n;
                if (left >= kVec) {
                    *reinterpret_cast<Pack<T, kVec> *>(y) = *reinterpret_cast<const Pack<T, kVec> *>(s);
                } else {
                    for (int e = 0; e < left; ++e) y[e] = s[e];
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// ---------------------------------------------------------------------------
// Few rows: the weights are what is read, so a workgroup takes 16 outputs and its
// eight waves share the width, 256 bytes of each output a wave and turn (a lane 64
// of them in four loads).  Factors go from memory to the matrix cores as they are:
// both sides take their bytes in the same order, and that order is free.  The
// waves' sums are joined in LDS.
// ---------------------------------------------------------------------------

constexpr int kFewWaves = 8;

template <typename T, int MT>
__global__ void __launch_bounds__(64 * kFewWaves) linear_few_kernel(LinearArgs a) {
    __shared__ int sums[kFewWaves][MT][16][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, part = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const int8_t *w = a.w + (int64_t)min(n0 + row, a.outputs - 1) * a.w_stride;
    const int8_t *x[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) x[j] = a.x + min((int64_t)(16 * j + row), a.rows - 1) * a.x_stride;
    i32x4 acc[MT] = {};
    for (int k0 = wave * 256; k0 < a.width; k0 += 256 * kFewWaves) {
        i32x4 wf[4], xf[MT][4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k = k0 + 64 * s + 16 * part;
            wf[s] = load_chunk(w, k, a.width);
#pragma unroll
            for (int j = 0; j < MT; ++j) xf[j][s] = load_chunk(x[j], k, a.width);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[s], xf[j][s], acc[j], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][j][row][4 * part + r] = acc[j][r];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 256; i += 64 * kFewWaves) {
        const int n = i & 15, m = i >> 4;
        if (m >= a.rows || n0 + n >= a.outputs) continue;
        int total = 0;
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) total += sums[v][m >> 4][m & 15][n];
        float o = (float)total * a.x_scale[m] * a.w_scale[n0 + n] + (a.bias ? a.bias[n0 + n] : 0.0f);
        if (a.gelu) o = gelu(o);
        static_cast<T *>(a.y)[m * a.y_stride + n0 + n] = static_cast<T>(o);
    }
}

template <typename T, int BM, int BN, int BK>
hipError_t launch_tiles(LinearArgs a, hipStream_t stream) {
    a.column_tiles = (a.outputs + BN - 1) / BN;
    // by as many rows as a launch holds
    const int64_t rows = a.rows, most = kMaxWorkgroups / a.column_tiles * BM;
    hipError_t err = hipSuccess;
    for (int64_t first = 0; first < rows && err == hipSuccess; first += most) {
        LinearArgs part = a;
        part.rows = std::min(rows - first, most);
        part.advance(first, sizeof(T));
        const dim3 grid((uint32_t)((part.rows + BM - 1) / BM * a.column_tiles));
        hipLaunchKernelGGL((linear_kernel<T, BM, BN, BK>), grid, dim3(kThreads), 0, stream, part);
        err = hipGetLastError();
    }
    return err;
}

template <typename T, int MT>
hipError_t launch_few(const LinearArgs &a, hipStream_t stream) {
    hipLaunchKernelGGL((linear_few_kernel<T, MT>), dim3((a.outputs + 15) / 16), dim3(64 * kFewWaves), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(LinearArgs a, int32_t dtype, int n_cus, hipStream_t stream) {
    const auto fits = [](const void *p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 16 == 0; };
    a.aligned = fits(a.x, a.x_stride) && fits(a.w, a.w_stride);
    return with_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        if (a.rows <= 16) return launch_few<T, 1>(a, stream);
        if (a.rows <= 32) return launch_few<T, 2>(a, stream);
        const int64_t tiles = (a.rows + 127) / 128 * ((a.outputs + 127) / 128);
        if (tiles < 2 * (int64_t)n_cus) return launch_tiles<T, 64, 64, 128>(a, stream);
        return launch_tiles<T, 128, 128, 128>(a, stream);
    });
}

}  // namespace flock
