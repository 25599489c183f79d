// tracks.hip - new detections' keys and values into the pages of their tracks.
//
//   key: pairs of dimensions turned by time, y and x as rotary_frames turns them,
//        in 32 bits, and rounded once, to the page's whole numbers
//   scale = max(scale the page had, if it held tokens before, max |new| / 127)
//   held tokens, where the scale grew: whole number * old / new scale, to the nearest
//   new tokens: value / scale, to the nearest; ties to even
//
// A workgroup takes the keys or the values of one page and kv head, so that no two
// meet in memory: values stay in LDS in 32 bits between the search for the largest and
// the rounding.  Tokens that the page does not get yet are left as they are.

#include "tracks_common.h"

namespace flock {
namespace {

using namespace tracks;

constexpr int kThreads = 256;
constexpr int kVec = 8;

// Largest |x| over the workgroup, as bits (those of NaN are the largest).
__device__ __forceinline__ uint32_t block_largest(uint32_t x, uint32_t *slot) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, d));
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = x;
    __syncthreads();
    return max(max(slot[0], slot[1]), max(slot[2], slot[3]));
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// x / scale to the nearest whole number, given what to multiply by instead (0: zeros).
__device__ __forceinline__ uint32_t rounded(float x, float per) {
    return per > 0.0f ? (uint32_t)(int)fminf(fmaxf(rintf(x * per), -127.0f), 127.0f) & 0xffu : 0u;
}

__device__ __forceinline__ float byte_of(const i32x4 &c, int i) { return (float)(int8_t)(c[i >> 2] >> (8 * (i & 3))); }

// Numbers of pages that the rows may touch: a track of n rows at most n / 64 + 2.
__host__ __device__ inline int64_t append_pages(int32_t n_tracks, int32_t total) {
    return (int64_t)total / kPage + 2 * (int64_t)n_tracks;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) append_kernel(AppendArgs a) {
    extern __shared__ float fresh[];    // [new tokens of the page][dim]
    __shared__ uint32_t slot[4];
    const int dim = a.cache.dim, heads = a.cache.kv_heads;
    const bool values = blockIdx.x & 1;
    const int64_t item = blockIdx.x >> 1;
    const int head = (int)(item % heads);
    int64_t within;
    const Track track = find_track(a.tracks, item / heads, append_pages(a.tracks.n_tracks, a.tracks.total),
                                   [](int offset, int t) { return (int64_t)(offset / kPage) + 2 * (int64_t)t; }, &within);
    if (!track.ok || track.n > track.length || within < 0) return;
    const int start = track.length - track.n;
    const int64_t first = (start / kPage + within) * kPage;  // the page's first token
    if (first >= track.length) return;
    const int s0 = (int)max((int64_t)start - first, (int64_t)0), s1 = (int)min((int64_t)track.length - first, (int64_t)kPage);
    const int n = s1 - s0;  // new tokens of this page
    if (n <= 0) return;
    const int page = a.tracks.table[(int64_t)track.index * a.tracks.table_stride + first / kPage];
    if (page < 0 || page >= a.cache.pages) return;
    const int64_t row0 = track.row0 + (first + s0 - start);
    const int64_t block = (int64_t)page * heads + head;

    // the new tokens, in 32 bits
    const T *in = static_cast<const T *>(values ? a.v : a.k) + row0 * (values ? a.v_stride : a.k_stride) + head * dim;
    const int64_t stride = values ? a.v_stride : a.k_stride;
    const int packs = dim / kVec;
    uint32_t largest = 0;
    for (int i = threadIdx.x; i < n * packs; i += kThreads) {
        const int token = i / packs, d = i % packs * kVec;
        float x[kVec];
        load_pack<T, kVec>(in + token * stride + d, x);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            fresh[token * dim + d + e] = x[e];
            if (values || d + e >= 2 * a.pairs) largest = max(largest, magnitude(x[e]));
        }
    }
    if (!values && a.pairs) {
        __syncthreads();
        for (int i = threadIdx.x; i < n * a.pairs; i += kThreads) {
            const int token = i / a.pairs, p = i % a.pairs;
            const int64_t bird = row0 + token;
            const int64_t pos = p < a.n_time ? a.time[bird] : a.xy[2 * bird + (p < a.n_time + a.n_y ? 1 : 0)];
            const uint64_t phase = (uint64_t)pos * a.step[p];
            const float turns = (float)(int32_t)(phase >> 32) * 0x1p-32f;
            const float sn = __builtin_amdgcn_sinf(turns), cs = __builtin_amdgcn_cosf(turns);
            float *u = fresh + token * dim + (a.interleaved ? 2 * p : p), *v = u + (a.interleaved ? 1 : a.pairs);
            const float x = *u, y = *v;
            *u = x * cs - y * sn;
            *v = x * sn + y * cs;
            largest = max(largest, max(magnitude(*u), magnitude(*v)));
        }
    }
    largest = block_largest(largest, slot);

    // the page's scale; one with values that are not finite has NaN, and zeros
    float *scales = values ? a.cache.v_scale : a.cache.k_scale;
    const float old = s0 > 0 ? scales[block] : 0.0f;
    float scale = largest < 0x7f800000u ? __uint_as_float(largest) / 127.0f : __uint_as_float(0x7fc00000u);
    if (largest < __float_as_uint(0x1p-100f)) scale = 0.0f;
    scale = old > scale || old != old ? old : scale;
    const float per = scale > 0.0f ? 1.0f / scale : 0.0f;
    const float again = old == scale ? 1.0f : per * old;  // what held tokens are multiplied by
    const bool held = s0 > 0 && old != scale;             // ... and have to be
    __syncthreads();                                      // (every wave has read the old scale)
    if (threadIdx.x == 0) scales[block] = scale;

    if (!values) {
        int8_t *k = a.cache.k + block * (kPage * dim);
        const int chunks = dim / 16, begin = held ? 0 : s0 * chunks;
        for (int i = begin + threadIdx.x; i < s1 * chunks; i += kThreads) {
            const int token = i / chunks, d = i % chunks * 16;
            i32x4 *at = reinterpret_cast<i32x4 *>(k + token * dim + d);
            i32x4 c = {0, 0, 0, 0};
            if (token < s0) {
                const i32x4 before = *at;
#pragma unroll
                for (int e = 0; e < 16; ++e) c[e >> 2] |= rounded(byte_of(before, e), again) << (8 * (e & 3));
            } else {
                const float *x = fresh + (token - s0) * dim + d;
#pragma unroll
                for (int e = 0; e < 16; ++e) c[e >> 2] |= rounded(x[e], per) << (8 * (e & 3));
            }
            *at = c;
        }
        return;
    }
    int8_t *v = a.cache.v + block * (kPage * dim);
    for (int i = threadIdx.x; i < 4 * dim; i += kThreads) {
        const int d = i % dim, part = i / dim;  // 16 places of a dimension
        // whether any of its tokens is written
        bool some = false, all = true;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int token = token_at(16 * part + e);
            const bool writes = token < s1 && (token >= s0 || held);
            some |= writes;
            all &= writes && token >= s0;
        }
        if (!some) continue;
        i32x4 *at = reinterpret_cast<i32x4 *>(v + d * kPage + 16 * part);
        i32x4 before = {0, 0, 0, 0}, c = {0, 0, 0, 0};
        if (!all) before = *at;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int token = token_at(16 * part + e);
            uint32_t b = (uint32_t)(before[e >> 2] >> (8 * (e & 3))) & 0xffu;
            if (token >= s0 && token < s1) b = rounded(fresh[(token - s0) * dim + d], per);
            else if (token < s0 && held) b = rounded(byte_of(before, e), again);
            c[e >> 2] |= b << (8 * (e & 3));
        }
        *at = c;
    }
}

}  // namespace

int64_t append_workgroups(int32_t n_tracks, int32_t total, int32_t kv_heads) {
    return append_pages(n_tracks, total) * kv_heads * 2;
}

hipError_t launch_append(const AppendArgs &a, int32_t dtype, hipStream_t stream) {
    const dim3 grid((uint32_t)append_workgroups(a.tracks.n_tracks, a.tracks.total, a.cache.kv_heads));
    const size_t lds = (size_t)std::min<int64_t>(kPage, a.tracks.total) * a.cache.dim * sizeof(float);
    return with_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL((append_kernel<T>), grid, dim3(kThreads), lds, stream, a);
        return hipGetLastError();
    });
}

}  // namespace flock
