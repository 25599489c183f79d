// rotary.hip - rotary positions with three axes: a bird's queries and keys are
// turned, pair of dimensions by pair, by angles that grow with its time, its y
// and its x.
//
//   angle_p = position on p's axis * freq_p;  (a, b) -> (a cos - b sin, a sin + b cos)
//
// Positions are whole numbers (frames, 1/16 px) and frequencies come as
// 64-bit fractions of a turn per unit, so the phase is one integer product
// whose overflow drops the whole turns: it has no rounding error, however far
// the bird is from the origin, and its upper 32 bits go to the hardware's sine
// and cosine, which take turns (largest error found: 7.3e-8).
//
// The turns of a bird serve all its heads: a block takes a few birds, puts
// their cosines and sines into LDS, and then streams the heads, bound by
// memory (each element is read once and written once): 128000 birds of 16 heads
// of 64 in bfloat16 111 us, 4.7 TB/s (140 us where a block made its table before
// it began to load); 500 birds 6.4 us, a chain of two loads and the table.

#include "encoder_common.h"

namespace flock {
namespace {

constexpr int kThreads = 256;
constexpr int kTable = 1024;  // (cos, sin) pairs in LDS

// n / d for m = ceil(2^32 / d), 0 for d = 1: exact while n d < 2^32 (here at
// most 2^23: the items of a block are at most 4 x 256, or one bird's 512 heads
// of 64 chunks).
__device__ __forceinline__ uint32_t quotient(uint32_t n, uint32_t m) { return m ? __umulhi(n, m) : n; }

// A block's work items are (bird, head, chunk of VEC pairs, then of VEC
// dimensions that are only passed on), at most kItems a thread.  Their loads
// are started first, the table is made while they run.
constexpr int kItems = 4;

template <typename T, int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs a) {
    __shared__ float2 table[kTable];
    const int pairs = a.pairs;
    const int64_t first = (int64_t)blockIdx.x * a.birds_per_block;
    const int birds = (int)min((int64_t)a.birds_per_block, a.total - first);
    const int heads = a.q_heads + a.k_heads;
    const int turned = (pairs + VEC - 1) / VEC;
    const int chunks = turned + (a.tail + VEC - 1) / VEC;
    const int items = birds * heads * chunks;
    float u[kItems][VEC], v[kItems][VEC];
    T *out[kItems];
    int bird_of[kItems], chunk[kItems];
    for (int base = 0; base < items; base += kItems * kThreads) {
#pragma unroll
        for (int n = 0; n < kItems; ++n) {
            const int e = base + n * kThreads + threadIdx.x;
            if (e >= items) continue;
            const int bh = quotient(e, a.chunk_reciprocal), c = e - bh * chunks;
            const int b = quotient(bh, a.head_reciprocal), hd = bh - b * heads;
            const int64_t bird = first + b;
            const T *in;
            if (hd < a.q_heads) {
                in = static_cast<const T *>(a.q) + bird * a.q_stride + hd * a.head_dim;
                out[n] = static_cast<T *>(a.q_out) + bird * a.q_out_stride + hd * a.head_dim;
            } else {
                in = static_cast<const T *>(a.k) + bird * a.k_stride + (hd - a.q_heads) * a.head_dim;
                out[n] = static_cast<T *>(a.k_out) + bird * a.k_out_stride + (hd - a.q_heads) * a.head_dim;
            }
            bird_of[n] = b;
            chunk[n] = c;
            if (c >= turned) {
                const int d = (c - turned) * VEC;
                load_some<T, VEC>(in + 2 * pairs + d, a.tail - d, u[n]);
            } else if (INTERLEAVED) {
                load_some<T, VEC>(in + 2 * c * VEC, 2 * (pairs - c * VEC), u[n]);
                load_some<T, VEC>(in + 2 * c * VEC + VEC, 2 * (pairs - c * VEC) - VEC, v[n]);
            } else {
                load_some<T, VEC>(in + c * VEC, pairs - c * VEC, u[n]);
                load_some<T, VEC>(in + pairs + c * VEC, pairs - c * VEC, v[n]);
            }
        }
        if (base == 0) {
            for (int e = threadIdx.x; e < birds * pairs; e += kThreads) {
                const int b = quotient(e, a.pair_reciprocal), p = e - b * pairs;
                const int64_t bird = first + b;
                int64_t pos;
                if (p < a.n_time) pos = a.time[bird];
                else pos = a.xy[2 * bird + (p < a.n_time + a.n_y ? 1 : 0)];
                const uint64_t phase = (uint64_t)pos * a.step[p];
                const float turns = (float)(int32_t)(phase >> 32) * 0x1p-32f;
                const float sn = __builtin_amdgcn_sinf(turns);
                table[e] = make_float2(__builtin_amdgcn_cosf(turns), a.inverse ? -sn : sn);
            }
            __syncthreads();
        }
#pragma unroll
        for (int n = 0; n < kItems; ++n) {
            if (base + n * kThreads + (int)threadIdx.x >= items) continue;
            const int c = chunk[n];
            if (c >= turned) {
                const int d = (c - turned) * VEC;
                store_some<T, VEC>(out[n] + 2 * pairs + d, a.tail - d, u[n]);
                continue;
            }
            const float2 *t = table + bird_of[n] * pairs + c * VEC;
            const int left = pairs - c * VEC;
            if (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float2 w = t[min(i, left - 1)];
                    float &x = i < VEC / 2 ? u[n][2 * i] : v[n][2 * i - VEC];
                    float &y = i < VEC / 2 ? u[n][2 * i + 1] : v[n][2 * i + 1 - VEC];
                    const float z = x * w.x - y * w.y;
                    y = x * w.y + y * w.x;
                    x = z;
                }
                store_some<T, VEC>(out[n] + 2 * c * VEC, 2 * left, u[n]);
                store_some<T, VEC>(out[n] + 2 * c * VEC + VEC, 2 * left - VEC, v[n]);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float2 w = t[min(i, left - 1)];
                    const float z = u[n][i] * w.x - v[n][i] * w.y;
                    v[n][i] = u[n][i] * w.y + v[n][i] * w.x;
                    u[n][i] = z;
                }
                store_some<T, VEC>(out[n] + c * VEC, left, u[n]);
                store_some<T, VEC>(out[n] + pairs + c * VEC, left, v[n]);
            }
        }
    }
}

uint32_t reciprocal(uint32_t d) { return d > 1 ? (uint32_t)(((1ull << 32) + d - 1) / d) : 0; }

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int32_t dtype, hipStream_t stream) {
    // dimensions beyond the pairs are copied, unless the call works in place
    a.tail = a.q == a.q_out && a.k == a.k_out ? 0 : a.head_dim - 2 * a.pairs;
    return with_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        constexpr int kVec = 16 / (int)sizeof(T);
        const int heads = a.q_heads + a.k_heads;
        const int chunks = (a.pairs + kVec - 1) / kVec + (a.tail + kVec - 1) / kVec;
        a.birds_per_block = 1;
        // as many birds as keep a thread at kItems items, the table within LDS
        while (a.birds_per_block < 64 && 2 * a.birds_per_block * a.pairs <= kTable &&
               2 * a.birds_per_block * heads * chunks <= kItems * kThreads)
            a.birds_per_block *= 2;
        a.chunk_reciprocal = reciprocal(chunks);
        a.head_reciprocal = reciprocal(heads);
        a.pair_reciprocal = reciprocal(a.pairs);
        // by as many birds as a launch holds
        const int64_t total = a.total, most = kMaxWorkgroups * a.birds_per_block;
        hipError_t err = hipSuccess;
        for (int64_t first = 0; first < total && err == hipSuccess; first += most) {
            RotaryArgs part = a;
            part.total = std::min(total - first, most);
            part.advance(first, sizeof(T));
            const dim3 grid((uint32_t)((part.total + a.birds_per_block - 1) / a.birds_per_block));
            if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<T, kVec, true>), grid, dim3(kThreads), 0, stream, part);
            else hipLaunchKernelGGL((rotary_kernel<T, kVec, false>), grid, dim3(kThreads), 0, stream, part);
            err = hipGetLastError();
        }
        return err;
    });
}

}  // namespace flock
