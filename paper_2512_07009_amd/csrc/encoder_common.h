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

// fn(T{}) with the element type of `dtype`.
template <typename F>
inline hipError_t with_dtype(int32_t dtype, F &&fn) {
    if (dtype == FLOCK_F32) return fn(float{});
    if (dtype == FLOCK_F16) return fn(half_t{});
    return fn(bf16_t{});
}

}  // namespace flock

#endif  // FLOCK_ENCODER_COMMON_H
