// tracks.hip - new detections' keys and values into the pages of their tracks.
//
//   key: pairs of dimensions turned by time, y and x as rotary_frames turns them,
//        in 32 bits, and rounded once, to the page's whole numbers
//   scale = max(scale the page had, if it held tokens before, max |new| / 127)
//   held tokens, where the scale grew: whole number * old / new scale, to the nearest
//   new tokens: value / scale, to the nearest; ties to even
//
// A workgroup takes the keys or the values of one page and kv head, so that no two
// meet in memory: they stay in LDS as they came between the search for the largest and
// the rounding.  Tokens that the page does not get yet are left as they are.
//
// The time is that of a workgroup's trips to memory one after the other (the track, its
// page, the rows with their positions and the page's scale), not of bytes: as many
// workgroups run beside each other as LDS allows.  With a token or a few a track one is
// a wave; clips take four.  500 tracks of a token, 2 kv heads of 64: 8 us for 7 MB;
// 700 clips of up to 120, 4 heads of 128: 78 us for 200 MB, vector instructions 68%.
// Rows in LDS as 32 bits left room for half the workgroups (99 us), keys turned twice
// took 83, and four tokens of values a lane at a time 88 for 82.

#include "tracks_common.h"
#include "whole.h"

namespace flock {
namespace {

using namespace tracks;
using namespace whole;

constexpr int kVec = 8, kItems = 4;
constexpr int kPad = 8;  // between tokens in LDS: those of four parts of a dimension's places lie in other banks

// Largest |x| over the workgroup, as bits (those of NaN are the largest).
template <int WAVES>
__device__ __forceinline__ uint32_t block_largest(uint32_t x, uint32_t *slot) {
    x = over_lanes<64>(x, [](uint32_t u, uint32_t v) { return max(u, v); });
    if (WAVES == 1) return x;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) x = max(x, slot[w]);
    return x;
}

// A byte of ones for each of the four low bits.
__device__ __forceinline__ int of_bits(uint32_t bits) { return (int)(((bits & 0xf) * 0x00204081u & 0x01010101u) * 0xffu); }

__device__ __forceinline__ float byte_of(const i32x4 &c, int i) { return (float)(int8_t)(c[i >> 2] >> (8 * (i & 3))); }

// Pages that rows go to are numbered as a first one of every track, and after those the
// others: a track of n rows has at most (n + 62) / 64 of them, so that those of the track
// whose rows begin at `offset` begin at other_pages().
__host__ __device__ inline int64_t other_pages(int32_t offset, int32_t track) {
    const int64_t each = (int64_t)(offset / kPage) + track, pairs = offset / 2;
    return each < pairs ? each : pairs;
}

template <typename T, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) append_kernel(AppendArgs a) {
    constexpr int kThreads = 64 * WAVES;
    extern __shared__ __attribute__((aligned(16))) char shared[];
    __shared__ uint32_t slot[WAVES];
    __shared__ int32_t places[3][kPage];   // time, y, x of the new tokens
    const int dim = a.cache.dim, pitch = dim + kPad, heads = a.cache.kv_heads;
    T *const fresh = reinterpret_cast<T *>(shared);                                    // [token of the page][pitch]
    int8_t *const whole = reinterpret_cast<int8_t *>(shared) + kPage * pitch * sizeof(T);  // keys: [new token][dim]
    const bool values = blockIdx.x & 1;
    const uint32_t item = blockIdx.x >> 1, number = item / (uint32_t)heads;
    const int head = (int)(item - number * heads);
    const int64_t others = (int64_t)number - a.tracks.n_tracks;
    int64_t within = 0;
    Track track;
    if (others < 0) {
        track = track_of(a.tracks, (int)number);
    } else {
        track = find_track(a.tracks, others, other_pages(a.tracks.total, a.tracks.n_tracks), other_pages, &within);
        if (within < 0) return;
        ++within;
    }
    if (!track.ok || track.n > track.length) return;
    const int start = track.length - track.n;
    const int64_t first = (start / kPage + within) * kPage;  // the page's first token
    if (first >= track.length) return;
    const int s0 = (int)max((int64_t)start - first, (int64_t)0), s1 = (int)min((int64_t)track.length - first, (int64_t)kPage);
    const int n = s1 - s0;  // new tokens of this page
    if (n <= 0) return;
    const int page = a.tracks.table[(int64_t)track.index * a.tracks.table_stride + first / kPage];
    const int64_t row0 = track.row0 + (first + s0 - start);

    // a new token is 2^pack_shift packs, its turns 2^pair_shift pairs: some of them none.
    // A thread's pairs are the same of every token.
    const int pairs = values ? 0 : a.pairs, p = threadIdx.x & ((1 << a.pair_shift) - 1);
    const uint64_t step = p < pairs ? a.step[p] : 0;
    if (page < 0 || page >= a.cache.pages) return;
    const int64_t block = (int64_t)page * heads + head;
    float *scales = values ? a.cache.v_scale : a.cache.k_scale;
    const float old = s0 > 0 ? scales[block] : 0.0f;
    int8_t *const v = a.cache.v + block * (kPage * dim);
    if (pairs && (int)threadIdx.x < n) {
        const int64_t bird = row0 + threadIdx.x;
        if (a.n_time) places[0][threadIdx.x] = a.time[bird];
        if (pairs > a.n_time) {
            const int2 xy = reinterpret_cast<const int2 *>(a.xy)[bird];
            places[1][threadIdx.x] = xy.y;
            places[2][threadIdx.x] = xy.x;
        }
    }

    // the new tokens, kItems packs of a thread on their way at a time
    const int64_t stride = values ? a.v_stride : a.k_stride;
    const T *in = static_cast<const T *>(values ? a.v : a.k) + row0 * stride + head * dim;
    uint32_t largest = 0;
    for (int first_item = threadIdx.x; first_item < n << a.pack_shift; first_item += kItems * kThreads) {
        Pack<T, kVec> x[kItems];
#pragma unroll
        for (int m = 0; m < kItems; ++m) {
            const int i = first_item + m * kThreads, token = i >> a.pack_shift, d = (i & ((1 << a.pack_shift) - 1)) * kVec;
            if (token < n && d < dim) x[m] = *reinterpret_cast<const Pack<T, kVec> *>(in + token * stride + d);
        }
#pragma unroll
        for (int m = 0; m < kItems; ++m) {
            const int i = first_item + m * kThreads, token = i >> a.pack_shift, d = (i & ((1 << a.pack_shift) - 1)) * kVec;
            if (token >= n || d >= dim) continue;
            *reinterpret_cast<Pack<T, kVec> *>(__builtin_assume_aligned(fresh + (s0 + token) * pitch + d, 16)) = x[m];
            if (pairs == 0) {
#pragma unroll
                for (int e = 0; e < kVec; ++e) largest = max(largest, magnitude(static_cast<float>(x[m].v[e])));
            }
        }
    }
    __syncthreads();
    // keys, turned: a pair of a token at a time, and what is beyond the pairs
    const int axis = p < a.n_time ? 0 : p < a.n_time + a.n_y ? 1 : 2;
    const int d0 = a.interleaved ? 2 * p : p, d1 = d0 + (a.interleaved ? 1 : pairs);
    const int first_token = threadIdx.x >> a.pair_shift, apart = kThreads >> a.pair_shift;
    const auto turn = [&](int token) {
        const uint64_t phase = (uint64_t)(int64_t)places[axis][token] * step;
        const float turned = (float)(int32_t)(phase >> 32) * 0x1p-32f;
        const float sn = __builtin_amdgcn_sinf(turned), cs = __builtin_amdgcn_cosf(turned);
        const T *row = fresh + (s0 + token) * pitch;
        const float x = static_cast<float>(row[d0]), y = static_cast<float>(row[d1]);
        return make_float2(x * cs - y * sn, x * sn + y * cs);
    };
    const auto others_of = [&](auto &&each) {
        for (int token = threadIdx.x >> 6; token < n; token += WAVES)
            for (int d = 2 * pairs + (threadIdx.x & 63); d < dim; d += 64)
                each(token, d, static_cast<float>(fresh[(s0 + token) * pitch + d]));
    };
    // (four waves keep what they turned, at most 64 x 64 pairs; one has a few tokens, and turns them again)
    constexpr int kTurns = WAVES == 4 ? kPage * 64 / kThreads : 1;
    float2 mine[kTurns];
    const auto note = [&](float x) { largest = max(largest, magnitude(x)); };
    if (pairs) {
        if (p < pairs) {
            if constexpr (WAVES == 4) {
#pragma unroll
                for (int m = 0; m < kTurns; ++m) {
                    const int token = first_token + m * apart;
                    if (token >= n) break;
                    mine[m] = turn(token);
                    note(mine[m].x);
                    note(mine[m].y);
                }
            } else {
                for (int token = first_token; token < n; token += apart) {
                    const float2 z = turn(token);
                    note(z.x);
                    note(z.y);
                }
            }
        }
        others_of([&](int, int, float x) { note(x); });
    }
    largest = block_largest<WAVES>(largest, slot);
    __syncthreads();  // (every wave has read the old scale)

    // the page's scale; one with values that are not finite has NaN, and zeros
    float scale = largest < 0x7f800000u ? __uint_as_float(largest) / 127.0f : __uint_as_float(0x7fc00000u);
    if (largest < __float_as_uint(0x1p-100f)) scale = 0.0f;
    scale = old > scale || old != old ? old : scale;
    const Quotient to(scale);
    const float again = scale > 0.0f ? old / scale : 0.0f;  // what held tokens are multiplied by
    const bool held = s0 > 0 && old != scale;  // ... and have to be
    const int kept = scale == scale ? -1 : 0;  // bits (a page with NaN holds zeros)
    if (threadIdx.x == 0) scales[block] = scale;

    if (!values) {
        int8_t *k = a.cache.k + block * (kPage * dim);
        const auto keep = [&](int token, int d, float x) { whole[token * dim + d] = (int8_t)(kept & to.rounded(x)); };
        if (p < pairs) {
            if constexpr (WAVES == 4) {
#pragma unroll
                for (int m = 0; m < kTurns; ++m) {
                    const int token = first_token + m * apart;
                    if (token >= n) break;
                    keep(token, d0, mine[m].x);
                    keep(token, d1, mine[m].y);
                }
            } else {
                for (int token = first_token; token < n; token += apart) {
                    const float2 z = turn(token);
                    keep(token, d0, z.x);
                    keep(token, d1, z.y);
                }
            }
        }
        others_of(keep);
        __syncthreads();
        const int shift = a.pack_shift - 1;  // chunks of 16
        for (int i = ((held ? 0 : s0) << shift) + threadIdx.x; i < s1 << shift; i += kThreads) {
            const int token = i >> shift, d = (i & ((1 << shift) - 1)) * 16;
            if (d >= dim) continue;
            i32x4 *at = reinterpret_cast<i32x4 *>(k + token * dim + d);
            if (token >= s0) {
                *at = *reinterpret_cast<const i32x4 *>(whole + (token - s0) * dim + d);
                continue;
            }
            const i32x4 before = *at;
            i32x4 c;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                c[e] = kept & bytes(rounded_again(byte_of(before, 4 * e), again), rounded_again(byte_of(before, 4 * e + 1), again),
                                    rounded_again(byte_of(before, 4 * e + 2), again), rounded_again(byte_of(before, 4 * e + 3), again));
            *at = c;
        }
        return;
    }
    // 16 places of a dimension at a time, which hold tokens 4 part + 0 .. 3 of each 16
    const uint64_t ends = s1 == 64 ? ~0ull : (1ull << s1) - 1, begins = (1ull << s0) - 1;
    for (int i = threadIdx.x; i < 4 * dim; i += kThreads) {
        const int part = i & 3, d = i >> 2;
        const auto of_part = [&](uint64_t tokens) {
            const uint64_t m = tokens >> (4 * part);
            return (uint32_t)(m & 0xf) | (uint32_t)(m >> 12 & 0xf0) | (uint32_t)(m >> 24 & 0xf00) | (uint32_t)(m >> 36 & 0xf000);
        };
        const uint32_t brings = of_part(ends & ~begins), holds = held ? of_part(begins) : 0;
        if (!(brings | holds)) continue;
        i32x4 *at = reinterpret_cast<i32x4 *>(v + d * kPage + 16 * part);
        // (no branches: what the places of other tokens have in LDS is read and left out)
        const T *x = fresh + 4 * part * pitch + d;
        const auto value = [&](int e, int i) { return to.rounded(static_cast<float>(x[(16 * e + i) * pitch])); };
        i32x4 c, before = {0, 0, 0, 0};
        if (brings != 0xffff) before = *at;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c[e] = kept & bytes(value(e, 0), value(e, 1), value(e, 2), value(e, 3));
            c[e] = (c[e] & of_bits(brings >> (4 * e))) | (before[e] & ~of_bits(brings >> (4 * e)));
        }
        if (held) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int again_4 = kept & bytes(rounded_again(byte_of(before, 4 * e), again), rounded_again(byte_of(before, 4 * e + 1), again),
                                                 rounded_again(byte_of(before, 4 * e + 2), again), rounded_again(byte_of(before, 4 * e + 3), again));
                c[e] = (again_4 & of_bits(holds >> (4 * e))) | (c[e] & ~of_bits(holds >> (4 * e)));
            }
        }
        *at = c;
    }
}

}  // namespace

int64_t append_workgroups(int32_t n_tracks, int32_t total, int32_t kv_heads) {
    return (n_tracks + other_pages(total, n_tracks)) * kv_heads * 2;
}

hipError_t launch_append(AppendArgs a, int32_t dtype, hipStream_t stream) {
    const dim3 grid((uint32_t)append_workgroups(a.tracks.n_tracks, a.tracks.total, a.cache.kv_heads));
    const auto shift = [](int n) {
        int s = 0;
        while ((1 << s) < n) ++s;
        return s;
    };
    a.pack_shift = shift(a.cache.dim / kVec);
    a.pair_shift = shift(a.pairs);
    return with_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        const size_t lds = kPage * (a.cache.dim + kPad) * sizeof(T) + kPage * a.cache.dim;
        if (a.tracks.total <= 8 * (int64_t)a.tracks.n_tracks) hipLaunchKernelGGL((append_kernel<T, 1>), grid, dim3(64), lds, stream, a);
        else hipLaunchKernelGGL((append_kernel<T, 4>), grid, dim3(256), lds, stream, a);
        return hipGetLastError();
    });
}

}  // namespace flock
