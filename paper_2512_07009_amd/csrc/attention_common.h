// attention_common.h - what the attention kernels share: the arithmetic of the
// scores, the matrix cores' layouts, the tiles' numbers.
#ifndef FLOCK_ATTENTION_COMMON_H
#define FLOCK_ATTENTION_COMMON_H

#include "encoder_common.h"

namespace flock {
namespace attention {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kPxPerQuantum = 1.0f / 16.0f;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef half_t f16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x16 mfma(f16x8 a, f16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

template <typename T> struct Frag;
template <> struct Frag<half_t> { using type = f16x8; };
template <> struct Frag<bf16_t> { using type = bf16x8; };

// Value of the lane 32 away, both halves' values combined by f.
template <typename F>
__device__ __forceinline__ float across(float x, F &&f) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// tanh from one exponential: 1 - 2 / (e^2x + 1), exact at both ends.
__device__ __forceinline__ float tanh_fast(float x) {
    return 1.0f - 2.0f * __builtin_amdgcn_rcpf(exp2_fast(2.0f * kLog2e * x) + 1.0f);
}

__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = max(x, __shfl_xor(x, d));
    return __builtin_amdgcn_readfirstlane(x);
}

// n / group for m = ceil(2^32 / group), 0 for a group of one: exact for
// n < 2^16, group <= 256.
__device__ __forceinline__ uint32_t group_quotient(uint32_t n, uint32_t m) { return m ? __umulhi(n, m) : n; }

// Row (of 32) that register r of a lane in half h holds of a product.
__device__ __forceinline__ constexpr int out_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// A frame's part of the batch.
struct Span {
    int32_t q0, nq, k0, nk;
    bool ok;
};

__device__ __forceinline__ Span frame_span(const AttentionArgs &a, int f) {
    Span s;
    s.q0 = a.q_offsets[f];
    s.k0 = a.k_offsets[f];
    const int32_t q1 = a.q_offsets[f + 1], k1 = a.k_offsets[f + 1];
    s.ok = s.q0 >= 0 && q1 >= s.q0 && q1 <= a.total_q && s.k0 >= 0 && k1 >= s.k0 && k1 <= a.total_k;
    s.nq = q1 - s.q0;
    s.nk = k1 - s.k0;
    return s;
}

// A run of rows of a frame and kv head, row r of it being head g of query i:
// only the run's beginning is divided by the heads in full.
struct RowRun {
    int first_query, first_g;
    __device__ __forceinline__ RowRun(const AttentionArgs &a, int row0) {
        first_query = (int)((uint32_t)row0 / (uint32_t)a.group);
        first_g = row0 - first_query * a.group;
    }
    __device__ __forceinline__ void find(const AttentionArgs &a, int r, int &query, int &g) const {
        const uint32_t u = first_g + r, n = group_quotient(u, a.group_reciprocal);
        query = first_query + (int)n;
        g = (int)(u - __umul24(n, a.group));
    }
    __device__ __forceinline__ int query(const AttentionArgs &a, int r) const {
        return first_query + (int)group_quotient(first_g + r, a.group_reciprocal);
    }
    __device__ __forceinline__ void advance(const AttentionArgs &a, int rows) {
        const int whole = (int)group_quotient(first_g + rows, a.group_reciprocal);
        first_query += whole;
        first_g += rows - whole * a.group;
    }
};

// The first key that query i of a frame does not see (without hidden keys).
__device__ __forceinline__ int seen_limit(const AttentionArgs &a, const Span &sp, int prefix, int i) {
    return a.causal ? (int)min(max((int64_t)prefix, (int64_t)i + sp.nk - sp.nq + 1), (int64_t)sp.nk) : sp.nk;
}

inline uint32_t group_reciprocal(int group) {
    return group > 1 ? (uint32_t)(((1ull << 32) + group - 1) / group) : 0;
}

// Tiles of `tile` rows are numbered without knowing the frames on the host:
// frame f's begin at offsets[f] * group / tile + f, which leaves it at least as
// many numbers as it has tiles.  Returns the frame of tile number `slot`, and
// the tile's place within it.
__device__ __forceinline__ int find_frame(const int32_t *offsets, int n_frames, int group, int tile, int64_t slot,
                                          int64_t *within) {
    int lo = 0, hi = n_frames - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((int64_t)offsets[mid] * group / tile + mid <= slot) lo = mid;
        else hi = mid - 1;
    }
    *within = slot - ((int64_t)offsets[lo] * group / tile + lo);
    return lo;
}

// Workgroups are dealt to the eight XCDs in turn; consecutive work items,
// which share keys, go to one XCD and meet in its L2.
__device__ __forceinline__ int64_t xcd_order(int64_t id, int64_t n) {
    const int64_t per = n / 8;
    return id < per * 8 ? (id % 8) * per + id / 8 : id;
}

// Copies rows of a [rows][dim] matrix into LDS rows of DP + 8 elements, zeros
// for rows that are absent and dimensions at and above dim.
template <int DP, int ROWS, typename P>
__device__ __forceinline__ void stage_rows(i16x8 *lds, int dim, P &&row_pointer) {
    constexpr int kChunks = DP / 8;
    constexpr int kPitch = DP / 8 + 1;
#pragma unroll
    for (int e = threadIdx.x; e < ROWS * kChunks; e += kThreads) {
        const int r = e / kChunks, c = e % kChunks;
        const short *p = row_pointer(r);
        i16x8 z = {};
        if (p != nullptr && c * 8 < dim) z = *reinterpret_cast<const i16x8 *>(p + c * 8);
        lds[r * kPitch + c] = z;
    }
}

// Left factor from LDS rows: lane's row, 8 dimensions from 16 step + 8 h.
template <typename T, int DP>
__device__ __forceinline__ typename Frag<T>::type read_rows(const i16x8 *lds, int row, int step, int h) {
    const i16x8 z = lds[row * (DP / 8 + 1) + 2 * step + h];
    return __builtin_bit_cast(typename Frag<T>::type, z);
}

// Left factor from LDS columns: dimension 32 block + lane % 32 of the LDS rows
// first + {4h .. 4h + 3, 8 + 4h .. 8 + 4h + 3}.
template <typename T, int DP>
__device__ __forceinline__ typename Frag<T>::type read_columns(const i16x8 *lds, int first, int block, int lane) {
    typedef __attribute__((address_space(3))) i16x4 *LdsPtr;
    const int h = lane >> 5, i = lane & 15, part = (lane >> 4) & 1;
    const short *p = reinterpret_cast<const short *>(lds) + (first + 4 * h + (i >> 2)) * (DP + 8) + 32 * block +
                     16 * part + 4 * (i & 3);
    const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)p);
    const i16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(p + 8 * (DP + 8)));
    const i16x8 z = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    return __builtin_bit_cast(typename Frag<T>::type, z);
}

// Right factor from global memory: 8 dimensions from 16 step + 8 h of a row.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type load_frag(const short *row, int step, int h, int dim) {
    i16x8 z = {};
    const int c = 16 * step + 8 * h;
    if (row != nullptr && c < dim) z = *reinterpret_cast<const i16x8 *>(row + c);
    return __builtin_bit_cast(typename Frag<T>::type, z);
}

// Waits for the loads so far.  Before a loop that keeps loads in flight: else the
// first use of what was loaded before it waits, in every turn, for those too.
__device__ __forceinline__ void wait_for_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// Half of a product's registers as the right factor of the next one.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type round_frag(const f32x16 &s, int part) {
    typename Frag<T>::type z;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = static_cast<T>(s[8 * part + i]);
    return z;
}

// Keys of a 32-key tile that a query sees, as bits of this lane's registers'
// rows (bit out_row(r, 0)): those in `bits` and below the query's limit.
__device__ __forceinline__ uint32_t seen_bits(uint32_t bits, int limit, int first_key, int h) {
    const int n = limit - first_key;
    if (n <= 0) return 0;
    if (n < 32) bits &= (1u << n) - 1u;
    return bits >> (4 * h);
}

// A tile of 64 keys (or KEYS) and its values on its way from memory to LDS: load() starts
// the loads into registers, so that they run under the products of the tile
// before, store() puts them into an LDS buffer.  Hidden and absent keys become
// zeros there and get a penalty of -infinity on their scores, so that nothing
// else need tell them apart; `seen` has a bit for each key that takes part, 64 a word.
//
// A tile is one buffer resource whose end is the end of its last key, so that
// loads beyond it (absent keys, dimensions beyond the head's, which are sent
// there) return zeros without a test; offsets within it stay below 2^31
// (kAttentionMaxStride), tiles begin at 64-bit addresses.
constexpr int kTileKeys = 64;
constexpr int kBeyond = 0x7ffffff0;

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_resource(const void *base, int64_t first_element, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(
        const_cast<short *>(static_cast<const short *>(base) + first_element), 0, bytes, 0x00027000);
}

template <int DP, int KEYS = kTileKeys>
struct KeyTile {
    static constexpr int kChunks = DP / 8;                       // of 16 bytes in a row
    static constexpr int kPitch = DP / 8 + 1;                    // LDS row, one chunk of padding
    static constexpr int kLoads = KEYS * kChunks / kThreads;
    static constexpr int kRowChunks = KEYS * kPitch;
    static constexpr int kBytes = 2 * kRowChunks * 16 + 3 * KEYS * 4 + 16;

    struct Lds {
        i16x8 *k, *v;
        float *x, *y, *penalty;
        uint64_t *seen;
        __device__ __forceinline__ explicit Lds(char *base) {
            k = reinterpret_cast<i16x8 *>(base);
            v = k + kRowChunks;
            x = reinterpret_cast<float *>(v + kRowChunks);
            y = x + KEYS;
            penalty = y + KEYS;
            seen = reinterpret_cast<uint64_t *>(penalty + KEYS);
        }
    };

    i32x4 k[kLoads], v[kLoads];
    // as loaded: what is made of them waits for the loads, so it is made in store()
    uint8_t kept[kLoads], key_kept;
    int2 place;

    template <bool DIST>
    __device__ __forceinline__ void load(const AttentionArgs &a, const Span &sp, int head, int first, int end) {
        const int rows = min(end - first, KEYS);
        const int64_t row0 = sp.k0 + first;
        const int k_step = (int)a.k_stride * 2, v_step = (int)a.v_stride * 2;
        const auto kr = tile_resource(a.k, row0 * a.k_stride + head * a.dim, (rows - 1) * k_step + a.dim * 2);
        const auto vr = tile_resource(a.v, row0 * a.v_stride + head * a.dim, (rows - 1) * v_step + a.dim * 2);
        constexpr bool kEven = kThreads % kChunks == 0;  // a thread's loads are of one column
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int e = threadIdx.x + (kEven ? 0 : n * kThreads);
            const int r = e / kChunks, c = e % kChunks;
            const bool in = c * 8 < a.dim;
            const int more = kEven ? n * (kThreads / kChunks) : 0;
            k[n] = __builtin_amdgcn_raw_buffer_load_b128(kr, in ? r * k_step + c * 16 : kBeyond, more * k_step, 0);
            v[n] = __builtin_amdgcn_raw_buffer_load_b128(vr, in ? r * v_step + c * 16 : kBeyond, more * v_step, 0);
            if (a.keep) kept[n] = a.keep[row0 + min(r + more, rows - 1)];
        }
        if (threadIdx.x < KEYS) {
            key_kept = (int)threadIdx.x < rows;
            const int64_t row = row0 + min((int)threadIdx.x, rows - 1);
            if (a.keep && key_kept) key_kept = a.keep[row];
            if (DIST) place = reinterpret_cast<const int2 *>(a.k_xy)[row];
        }
    }

    template <bool DIST>
    __device__ __forceinline__ void store(const AttentionArgs &a, const Lds &lds) {
        if (a.keep) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                if (kept[n] == 0) k[n] = v[n] = i32x4{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int e = threadIdx.x + n * kThreads;
            const int at = e / kChunks * kPitch + e % kChunks;
            lds.k[at] = __builtin_bit_cast(i16x8, k[n]);
            lds.v[at] = __builtin_bit_cast(i16x8, v[n]);
        }
        if (threadIdx.x < KEYS) {  // whole waves
            if (DIST) {
                lds.x[threadIdx.x] = (float)place.x * kPxPerQuantum;
                lds.y[threadIdx.x] = (float)place.y * kPxPerQuantum;
            }
            lds.penalty[threadIdx.x] = key_kept != 0 ? 0.0f : -INFINITY;
            const uint64_t seen = __ballot(key_kept != 0);
            if ((threadIdx.x & 63) == 0) lds.seen[threadIdx.x >> 6] = seen;
        }
    }
};

// Four floats of consecutive rows of a product, from LDS.
__device__ __forceinline__ float4 read4(const float *p, int first, int r, int h) {
    return *reinterpret_cast<const float4 *>(p + first + out_row(r, h));
}

// Squared distance in px^2, and the scores in units of log 2 from a product of
// queries and keys.  The products' order is written out, so that every kernel
// gets the same bits: P = exp(s - lse) of the backward pass is then right even
// where all of a query's keys are far and its scores are large (th: tanh(t / cap),
// kept for the gradient).
__device__ __forceinline__ float distance2(float dx, float dy) { return __builtin_fmaf(dx, dx, dy * dy); }

template <bool DIST, bool CAP>
__device__ __forceinline__ float score(float qk, float scale, float cap2, float d2, float slope2, float &th) {
    float s;
    if (CAP) {
        th = tanh_fast(qk * scale);  // scale holds scale / cap
        s = cap2 * th;
    } else {
        s = qk * scale;              // scale holds scale * log2 e
    }
    if (DIST) s = __builtin_fmaf(-slope2, d2, s);
    return s;
}

// log sum exp of a query in 64 bits: with large scores, 32 would not hold it
// to a weight's digits.  top is the largest score in units of log 2, sum the
// sum of 2^(s - top).
__device__ __forceinline__ double row_lse(float top, float sum) {
    return sum > 0.0f ? ((double)top + (double)__builtin_log2f(sum)) * 0.693147180559945309417 : -INFINITY;
}

// A query's lse in units of log 2 as shift, and the factor that is left:
// P = 2^(s - shift) * rest.  A query that sees no key has P = 0.
__device__ __forceinline__ void split_lse(double lse, float &shift, float &rest) {
    const double lse2 = lse * 1.44269504088896340736;
    shift = (float)lse2;
    rest = exp2_fast((float)((double)shift - lse2));
    if (shift == -INFINITY) {
        shift = INFINITY;
        rest = 0.0f;
    }
}

// fn<T, DP, DIST, CAP>() of the call.
template <typename F>
inline hipError_t with_kernel(const AttentionArgs &a, int32_t dtype, F &&fn) {
    auto flags = [&](auto t, auto dp) {
        auto yes = std::true_type{};
        auto no = std::false_type{};
        const bool dist = a.slopes != nullptr, cap = a.cap > 0.0f;
        if (dist) return cap ? fn(t, dp, yes, yes) : fn(t, dp, yes, no);
        return cap ? fn(t, dp, no, yes) : fn(t, dp, no, no);
    };
    auto dims = [&](auto t) {
        if (a.dim <= 32) return flags(t, std::integral_constant<int, 32>{});
        if (a.dim <= 64) return flags(t, std::integral_constant<int, 64>{});
        if (a.dim <= 96) return flags(t, std::integral_constant<int, 96>{});
        return flags(t, std::integral_constant<int, 128>{});
    };
    return dtype == FLOCK_F16 ? dims(half_t{}) : dims(bf16_t{});
}

inline size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace attention
}  // namespace flock

#endif  // FLOCK_ATTENTION_COMMON_H
