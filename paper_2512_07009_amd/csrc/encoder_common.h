// encoder_common.h - element types of the per-bird encoder's kernels (layer
// norm, rotary positions, attention): loads of packs, and conversions that
// round to nearest even.
#ifndef FLOCK_ENCODER_COMMON_H
#define FLOCK_ENCODER_COMMON_H

#include <hip/hip_runtime.h>

#include "flock.h"
#include "internal.h"

namespace flock {

using half_t = _Float16;
using bf16_t = __bf16;

// N elements moved by loads or stores of 16 bytes at most.  Memory may hold a
// pack at any element: the hardware's wide accesses need no more.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T v[N];
};

template <typename T, int N>
__device__ __forceinline__ void load_pack(const T *p, float (&out)[N]) {
    const Pack<T, N> a = *reinterpret_cast<const Pack<T, N> *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = static_cast<float>(a.v[i]);
}

template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const float (&in)[N]) {
    Pack<T, N> a;
#pragma unroll
    for (int i = 0; i < N; ++i) a.v[i] = static_cast<T>(in[i]);
    *reinterpret_cast<Pack<T, N> *>(p) = a;
}

// The first n (of N) elements of a pack, zeros after them.
template <typename T, int N>
__device__ __forceinline__ void load_some(const T *p, int n, float (&out)[N]) {
    if (n >= N) {
        load_pack<T, N>(p, out);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = i < n ? static_cast<float>(p[i]) : 0.0f;
}

template <typename T, int N>
__device__ __forceinline__ void store_some(T *p, int n, const float (&in)[N]) {
    if (n >= N) {
        store_pack<T, N>(p, in);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = static_cast<T>(in[i]);
}

// f over the values (32 bits) of each LANES lanes beside each other, pairs that are farthest
// apart first: the lanes 32 and 16 away by swaps of rows, the others by turns of a row of 16,
// which is a lane 8, and then, where all that are 8 apart are alike, 4 away.  All lanes of
// the LANES are active.  (Norms of 128000 rows of 512 in 8 bits, two of these a row: by
// way of LDS, as __shfl_xor goes, 63 us, so 50.)
template <int LANES, typename V, typename F>
__device__ __forceinline__ V over_lanes(V x, F &&f) {
    static_assert(LANES == 8 || LANES == 16 || LANES == 32 || LANES == 64, "a row's lanes");
    const auto bits = [](V v) { return __builtin_bit_cast(uint32_t, v); };
    const auto value = [](uint32_t v) { return __builtin_bit_cast(V, v); };
    if constexpr (LANES >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(bits(x), bits(x), false, false);
        x = f(value(p[0]), value(p[1]));
    }
    if constexpr (LANES >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(bits(x), bits(x), false, false);
        x = f(value(p[0]), value(p[1]));
    }
    if constexpr (LANES >= 16) {
        x = f(x, value(__builtin_amdgcn_update_dpp(0, bits(x), 0x128, 0xf, 0xf, false)));  // row_ror:8
        x = f(x, value(__builtin_amdgcn_update_dpp(0, bits(x), 0x124, 0xf, 0xf, false)));  // row_ror:4
    } else {
        x = f(x, value(__shfl_xor(bits(x), 4)));
    }
    x = f(x, value(__builtin_amdgcn_update_dpp(0, bits(x), 0x4e, 0xf, 0xf, false)));  // quad_perm:[2,3,0,1]
    return f(x, value(__builtin_amdgcn_update_dpp(0, bits(x), 0xb1, 0xf, 0xf, false)));  // quad_perm:[1,0,3,2]
}

// fn(T{}) with the element type of `dtype`.
template <typename F>
inline hipError_t with_dtype(int32_t dtype, F &&fn) {
    if (dtype == FLOCK_F32) return fn(float{});
    if (dtype == FLOCK_F16) return fn(half_t{});
    return fn(bf16_t{});
}

}  // namespace flock

#endif  // FLOCK_ENCODER_COMMON_H
