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
// memory (each element is read once and written once).

#include "encoder_common.h"

namespace flock {
namespace {

constexpr int kThreads = 256;
constexpr int kTable = 1024;  // (cos, sin) pairs in LDS

// n / d for m = ceil(2^32 / d), 0 for d = 1: exact while n d < 2^32 (here at
// most 2^25: the items of a block are at most 4 x 256, or one bird's 512 heads
// of 256 dimensions).
__device__ __forceinline__ uint32_t quotient(uint32_t n, uint32_t m) { return m ? __umulhi(n, m) : n; }

template <typename T, int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs a) {
    __shared__ float2 table[kTable];
    const int pairs = a.pairs;
    const int64_t first = (int64_t)blockIdx.x * a.birds_per_block;
    const int birds = (int)min((int64_t)a.birds_per_block, a.total - first);
    for (int e = threadIdx.x; e < birds * pairs; e += kThreads) {
        const int b = e / pairs, p = e - b * pairs;
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
    // work items: bird, head, chunk of VEC pairs (then of VEC dimensions that are only passed on)
    const int heads = a.q_heads + a.k_heads;
    const int turned = pairs / VEC;
    const int chunks = turned + a.tail / VEC;
    const int items = birds * heads * chunks;
    for (int e = threadIdx.x; e < items; e += kThreads) {
        const int bh = quotient(e, a.chunk_reciprocal), c = e - bh * chunks;
        const int b = quotient(bh, a.head_reciprocal), hd = bh - b * heads;
        const int64_t bird = first + b;
        const T *in;
        T *out;
        if (hd < a.q_heads) {
            in = static_cast<const T *>(a.q) + bird * a.q_stride + hd * a.head_dim;
            out = static_cast<T *>(a.q_out) + bird * a.q_out_stride + hd * a.head_dim;
        } else {
            in = static_cast<const T *>(a.k) + bird * a.k_stride + (hd - a.q_heads) * a.head_dim;
            out = static_cast<T *>(a.k_out) + bird * a.k_out_stride + (hd - a.q_heads) * a.head_dim;
        }
        if (c >= turned) {
            const int d = 2 * pairs + (c - turned) * VEC;
            float z[VEC];
            load_pack<T, VEC>(in + d, z);
            store_pack<T, VEC>(out + d, z);
            continue;
        }
        const float2 *t = table + b * pairs + c * VEC;
        float u[VEC], v[VEC];
        if (INTERLEAVED) {
            load_pack<T, VEC>(in + 2 * c * VEC, u);
            load_pack<T, VEC>(in + 2 * c * VEC + VEC, v);
            if (VEC == 1) {
                const float2 w = t[0];
                const float x = u[0] * w.x - v[0] * w.y;
                v[0] = u[0] * w.y + v[0] * w.x;
                u[0] = x;
            } else {
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) {
                    const float2 w0 = t[i], w1 = t[VEC / 2 + i];
                    const float x0 = u[2 * i] * w0.x - u[2 * i + 1] * w0.y;
                    u[2 * i + 1] = u[2 * i] * w0.y + u[2 * i + 1] * w0.x;
                    u[2 * i] = x0;
                    const float x1 = v[2 * i] * w1.x - v[2 * i + 1] * w1.y;
                    v[2 * i + 1] = v[2 * i] * w1.y + v[2 * i + 1] * w1.x;
                    v[2 * i] = x1;
                }
            }
            store_pack<T, VEC>(out + 2 * c * VEC, u);
            store_pack<T, VEC>(out + 2 * c * VEC + VEC, v);
        } else {
            load_pack<T, VEC>(in + c * VEC, u);
            load_pack<T, VEC>(in + pairs + c * VEC, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float2 w = t[i];
                const float x = u[i] * w.x - v[i] * w.y;
                v[i] = u[i] * w.y + v[i] * w.x;
                u[i] = x;
            }
            store_pack<T, VEC>(out + c * VEC, u);
            store_pack<T, VEC>(out + pairs + c * VEC, v);
        }
    }
}

uint32_t reciprocal(uint32_t d) { return d > 1 ? (uint32_t)(((1ull << 32) + d - 1) / d) : 0; }

bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int32_t dtype, hipStream_t stream) {
    // dimensions beyond the pairs are copied, unless the call works in place
    a.tail = a.q == a.q_out && a.k == a.k_out ? 0 : a.head_dim - 2 * a.pairs;
    return with_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        constexpr int kVec = 16 / (int)sizeof(T);
        const bool packs = a.pairs % kVec == 0 && a.head_dim % kVec == 0 && on16(a.q) && on16(a.k) && on16(a.q_out) &&
                           on16(a.k_out) && a.q_stride % kVec == 0 && a.k_stride % kVec == 0 &&
                           a.q_out_stride % kVec == 0 && a.k_out_stride % kVec == 0;
        const int vec = packs ? kVec : 1;
        const int heads = a.q_heads + a.k_heads;
        const int chunks = a.pairs / vec + a.tail / vec;
        a.birds_per_block = 1;
        // a few items a thread, and the table within LDS
        while (a.birds_per_block < 64 && 2 * a.birds_per_block * a.pairs <= kTable &&
               2 * a.birds_per_block * heads * chunks <= 4 * kThreads)
            a.birds_per_block *= 2;
        a.chunk_reciprocal = reciprocal(chunks);
        a.head_reciprocal = reciprocal(heads);
        const dim3 grid((uint32_t)((a.total + a.birds_per_block - 1) / a.birds_per_block));
        if (packs) {
            if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<T, kVec, true>), grid, dim3(kThreads), 0, stream, a);
            else hipLaunchKernelGGL((rotary_kernel<T, kVec, false>), grid, dim3(kThreads), 0, stream, a);
        } else {
            if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<T, 1, true>), grid, dim3(kThreads), 0, stream, a);
            else hipLaunchKernelGGL((rotary_kernel<T, 1, false>), grid, dim3(kThreads), 0, stream, a);
        }
        return hipGetLastError();
    });
}

}  // namespace flock
