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

// Caps, cap tanh(t / cap), in two forms.  Low ones: r = 1 / (e^2x + 1) from
// 2 x log2 e, tanh x = 1 - 2 r, and its derivative 1 - tanh^2 x = 4 r (1 - r).  Small
// scores are then differences of numbers as large as the cap, off by 1.5e-7 of it:
// up to kLowCap that is 1e-5, what 32-bit sums of products leave them as well.
// Higher caps take tanh itself, to 2.5e-7 of its size: below 1/2 the continued
// fraction x / (1 + x^2 / (3 + x^2 / (5 + x^2 / 7))) (its next part is x^2 / 9: off by
// 4e-8), 1 - 2 r above.  That costs a cap of 100 14% of a forward pass (64 x 2000: 1.10
// -> 1.25 ms) and 8% of a training step (4.74 -> 5.13 ms).
constexpr int kNoCap = 0, kLow = 1, kHigh = 2;
constexpr float kLowCap = 64.0f;
// A cap from here on changes no score by a rounding of it below 2^83.
constexpr float kLargestCap = 0x1p96f;
__device__ __forceinline__ float tanh_part(float x2) { return __builtin_amdgcn_rcpf(exp2_fast(x2) + 1.0f); }
__device__ __forceinline__ float tanh_low(float x) {
    const float n = x * x;
    return x * __builtin_fmaf(10.0f, n, 105.0f) * __builtin_amdgcn_rcpf(__builtin_fmaf(n, n + 45.0f, 105.0f));
}
// What a score's gradient is multiplied by, from cap_parts below.
template <int CAP>
__device__ __forceinline__ float cap_slope(float r) {
    return CAP == kLow ? 4.0f * __builtin_fmaf(-r, r, r) : __builtin_fmaf(-r, r, 1.0f);
}
// The parts of capped scores that their gradients take, from products and
// score_scale(), and the score in units of log 2 from one; other may be added.
template <int CAP>
__device__ __forceinline__ void cap_parts(f32x16 &s, float scale) {
    if (CAP == kLow) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = tanh_part(s[r] * scale);
    } else if (CAP == kHigh) {
        float most = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] *= scale;
            most = fmaxf(most, fabsf(s[r]));
        }
        // where a high cap does its work no score comes near it
        if (__all(most < 0.5f)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = tanh_low(s[r]);
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float high = __builtin_fmaf(-2.0f, tanh_part(s[r] * (2.0f * kLog2e)), 1.0f);
                s[r] = fabsf(s[r]) < 0.5f ? tanh_low(s[r]) : high;
            }
        }
    }
}
template <int CAP>
__device__ __forceinline__ float capped(float r, float cap2, float other) {
    return __builtin_fmaf(CAP == kLow ? -2.0f * cap2 : cap2, r, other);
}
template <int CAP>
__device__ __forceinline__ float cap_constant(float cap2) { return CAP == kLow ? cap2 : 0.0f; }
// What products are multiplied by first (finite, so that a hidden key's zero stays
// one under caps near the smallest number).
template <int CAP>
__device__ __forceinline__ float score_scale(const AttentionArgs &a) {
    if (CAP == kHigh) return a.scale / a.cap;
    return CAP == kLow ? fminf(2.0f * kLog2e * a.scale / a.cap, 0x1p127f) : a.scale * kLog2e;
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

// Workgroups are dealt to the eight XCDs in turn; each XCD gets an eighth of the
// work items in one piece, so that those that share keys meet in its L2.  Against
// the plain order: 256 queries over 8000 keys 481 -> 427 us, training steps 8%;
// against runs of 32 items an XCD: 513 -> 427 us, and 2%.
__device__ __forceinline__ int64_t xcd_order(int64_t id, int64_t n) {
    const int64_t per = n / 8;
    return id < per * 8 ? (id % 8) * per + id / 8 : id;
}

// Rows of DP / 8 chunks of 16 bytes lie a pitch of chunks apart in LDS.  Read as
// rows (16 lanes a chunk each of 16 rows) they want an odd pitch, read as columns
// (4 chunks of 4 rows a time) one of 4 or 12 modulo 16; rows read both ways take
// the odd pitch that leaves 2 chunks of 4 rows apart, the best there is.
template <int DP>
struct Pitch {
    static constexpr int kRows = DP / 8 + 1;
    static constexpr int kColumns = DP == 128 ? 20 : DP == 32 ? 4 : 12;
    static constexpr int kBoth = DP == 128 ? 19 : DP == 32 ? 7 : DP / 8 + 1;
};

// Left factor from LDS rows: lane's row, 8 dimensions from 16 step + 8 h.
template <typename T, int PITCH>
__device__ __forceinline__ typename Frag<T>::type read_rows(const i16x8 *lds, int row, int step, int h) {
    const i16x8 z = lds[row * PITCH + 2 * step + h];
    return __builtin_bit_cast(typename Frag<T>::type, z);
}

// Left factor from LDS columns: dimension 32 block + lane % 32 of the LDS rows
// first + {4h .. 4h + 3, 8 + 4h .. 8 + 4h + 3}.
template <typename T, int PITCH>
__device__ __forceinline__ typename Frag<T>::type read_columns(const i16x8 *lds, int first, int block, int lane) {
    typedef __attribute__((address_space(3))) i16x4 *LdsPtr;
    const int h = lane >> 5, i = lane & 15, part = (lane >> 4) & 1;
    const short *p = reinterpret_cast<const short *>(lds) + (first + 4 * h + (i >> 2)) * (8 * PITCH) + 32 * block +
                     16 * part + 4 * (i & 3);
    const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)p);
    const i16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(p + 8 * (8 * PITCH)));
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

// Distances on the matrix cores.  Relative to a common origin, with row a and key
// b, -slope d2 = 2 slope a.b - slope |b|^2 - slope |a|^2; the last term is a
// constant of the row, and the first two are one more step of the product of
// queries and keys: 16 products of bfloat16 parts (8 bits each) that hold x, y
// (two parts, whole numbers of 1/16 px below 2^16), |b|^2 and the slope's factors
// (three parts) to 2^-24.  That takes five vector operations off each score,
// where they bound the kernels (64 x 2000 without lse 1.07 -> 0.87 ms, 24 x 8000 9.6 ->
// 8.9 ms, a training step, in the keys' gradients, 4.08 -> 3.90).  The sums pass
// through numbers as large as slope |b|^2, so scores are off by 2^-22 of that.
// near_limit (in units of log 2) keeps the weights' relative error below what
// rounding them to the operands' type costs (at worst 7e-4 of 4e-3 in bfloat16,
// 2.5e-4 of 5e-4 in float16; the outputs' errors are the same to three digits with it
// and without), and tiles with a bird farther away take the differences themselves.
// So do a forward pass that writes lse, which is exact to 32 bits, and the queries'
// gradients, whose sums of dS show what delta is off by.
template <typename T> constexpr float near_limit() { return 4096.0f; }
template <> constexpr float near_limit<half_t>() { return 1536.0f; }
constexpr int kNearReach = 1 << 15;

struct NearSlots {
    i16x8 half[2];  // of the lanes' halves
};

__device__ __forceinline__ void split3(float v, bf16_t (&p)[3]) {
    p[0] = static_cast<bf16_t>(v);
    v -= static_cast<float>(p[0]);
    p[1] = static_cast<bf16_t>(v);
    p[2] = static_cast<bf16_t>(v - static_cast<float>(p[1]));
}

// The key's 16 factors; n is |b|^2 in (1/16 px)^2.
__device__ __forceinline__ NearSlots near_key(int bx, int by, float n) {
    const bf16_t xh = static_cast<bf16_t>((float)bx), yh = static_cast<bf16_t>((float)by);
    const bf16_t xl = static_cast<bf16_t>((float)bx - static_cast<float>(xh));
    const bf16_t yl = static_cast<bf16_t>((float)by - static_cast<float>(yh));
    bf16_t p[3];
    split3(n, p);
    const bf16x8 lo = {xh, yh, p[0], xl, xh, yl, yh, p[1]}, hi = {p[0], xh, yh, xl, yl, p[0], p[1], p[2]};
    return {__builtin_bit_cast(i16x8, lo), __builtin_bit_cast(i16x8, hi)};
}

// The row's 16 factors; weight is the slope in the products' units and (1/16 px)^-2.
__device__ __forceinline__ NearSlots near_row(int ax, int ay, float weight) {
    bf16_t x[3], y[3], n[3];
    split3(2.0f * weight * (float)ax, x);
    split3(2.0f * weight * (float)ay, y);
    split3(-weight, n);
    const bf16x8 lo = {x[0], y[0], n[0], x[0], x[1], y[0], y[1], n[0]};
    const bf16x8 hi = {n[1], x[2], y[2], x[1], y[1], n[2], n[1], n[0]};
    return {__builtin_bit_cast(i16x8, lo), __builtin_bit_cast(i16x8, hi)};
}

__device__ __forceinline__ float square_quanta(int x, int y) {
    return __builtin_fmaf((float)x, (float)x, (float)y * (float)y);
}

// Origin of a workgroup's distances: the middle of 32 birds (a lane each, both halves alike).
__device__ __forceinline__ int2 near_origin(int2 p) {
    int x0 = p.x, x1 = p.x, y0 = p.y, y1 = p.y;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        x0 = min(x0, __shfl_xor(x0, d));
        x1 = max(x1, __shfl_xor(x1, d));
        y0 = min(y0, __shfl_xor(y0, d));
        y1 = max(y1, __shfl_xor(y1, d));
    }
    return make_int2(__builtin_amdgcn_readfirstlane((x0 + x1) / 2), __builtin_amdgcn_readfirstlane((y0 + y1) / 2));
}

// The largest |b|^2 that the heads of kv head `head` allow.  Without caps distances
// are added in the products' units, which scales below 2^-40 leave no room for.
template <typename T, int CAP>
__device__ __forceinline__ float near_largest(const AttentionArgs &a, int head, float scale) {
    float steepest = 0.0f;
    for (int e = 0; e < a.group; ++e) steepest = fmaxf(steepest, fabsf(a.slopes[head * a.group + e]) * kLog2e);
    return !CAP && scale < 0x1p-40f ? -1.0f : near_limit<T>() * 256.0f / steepest;
}

__device__ __forceinline__ bool near_enough(int x, int y, float n, float largest) {
    return abs(x) < kNearReach && abs(y) < kNearReach && n <= largest;
}

// A tile of 64 keys (or KEYS) and its values on its way from memory to LDS: load() starts
// the loads into registers, so that they run under the products of the tile
// before, store() puts them into an LDS buffer.  Hidden and absent keys become
// zeros there and get a penalty of -infinity on their scores, so that nothing
// else need tell them apart; `seen` has a bit for each key that takes part, 64 a word.
//
// Each part of a tile (kPartKeys keys, or all of them) is one buffer resource
// whose end is the end of its last key, so that loads beyond it (absent keys,
// dimensions beyond the head's and hidden keys, which are sent there) return zeros
// without a test; parts begin at 64-bit addresses.  However far rows lie apart, a
// part ends before kBeyond, and kBeyond with a thread's later rows is below 2^32.
constexpr int kTileKeys = 64, kPartKeys = 64;
constexpr int kBeyond = 0x7ffffff0;
static_assert((kPartKeys - 1) * 2 * kAttentionMaxStride + 2 * kAttentionMaxDim <= kBeyond &&
                  kBeyond + (kPartKeys - 1) * 2 * kAttentionMaxStride + 2 * kAttentionMaxDim < 1ll << 32,
              "offsets within a part of a tile fit the resource's 32 bits");

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_resource(const void *base, int64_t first_element, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(
        const_cast<short *>(static_cast<const short *>(base) + first_element), 0, bytes, 0x00027000);
}

template <int DP, int KEYS, int K_PITCH, int V_PITCH, bool NEAR>
struct KeyTile {
    static constexpr int kChunks = DP / 8;                       // of 16 bytes in a row
    static constexpr int kLoads = KEYS * kChunks / kThreads;
    static_assert(kLoads * kThreads == KEYS * kChunks, "every thread loads whole chunks");
    static constexpr int kBytes = KEYS * (K_PITCH + V_PITCH) * 16 + (NEAR ? 2 * KEYS * 16 : 0) + 3 * KEYS * 4 + 32;

    struct Lds {
        i16x8 *k, *v, *near;  // near: [half][key]
        float *x, *y, *penalty;
        uint64_t *seen;
        int *all_near;
        __device__ __forceinline__ explicit Lds(char *base) {
            k = reinterpret_cast<i16x8 *>(base);
            v = k + KEYS * K_PITCH;
            near = v + KEYS * V_PITCH;
            x = reinterpret_cast<float *>(near + (NEAR ? 2 * KEYS : 0));
            y = x + KEYS;
            penalty = y + KEYS;
            seen = reinterpret_cast<uint64_t *>(penalty + KEYS);
            all_near = reinterpret_cast<int *>(seen + 2);
        }
    };

    i32x4 k[kLoads], v[kLoads];
    int k_at, v_at;  // this thread's place in a tile
    // as loaded: what is made of them waits for the loads, so it is made in store(),
    // and a tile's hidden keys are looked up a tile ahead, so that load() can send
    // them beyond the resource
    uint8_t kept[kLoads], key_kept;
    i32x2 place;
    int present;  // keys of the tile

    // A thread's loads are of one column, rows kStep apart, unless rows have 12 chunks.
    static constexpr bool kEven = kThreads % kChunks == 0;
    static constexpr int kStep = kThreads / kChunks;

    __device__ __forceinline__ explicit KeyTile(const AttentionArgs &a) {
        const int r = threadIdx.x / kChunks, c = threadIdx.x % kChunks;
        k_at = c * 8 < a.dim ? r * (int)a.k_stride * 2 + c * 16 : kBeyond;
        v_at = c * 8 < a.dim ? r * (int)a.v_stride * 2 + c * 16 : kBeyond;
    }

    // Whether the keys of the tile from `first` are kept (absent ones are not).
    __device__ __forceinline__ void look_up(const AttentionArgs &a, const Span &sp, int first, int end) {
        if (!a.keep || first >= end) return;
        const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.keep) + sp.k0 + first, 0, end - first,
                                                         0x00027000);
#pragma unroll
        for (int n = 0; n < kLoads; ++n)
            kept[n] = __builtin_amdgcn_raw_buffer_load_b8(r, (threadIdx.x + n * kThreads) / kChunks, 0, 0);
    }

    template <bool DIST>
    __device__ __forceinline__ void load(const AttentionArgs &a, const Span &sp, int head, int first, int end) {
        const int rows = present = min(end - first, KEYS);
        const int64_t row0 = sp.k0 + first;
        const int k_step = (int)a.k_stride * 2, v_step = (int)a.v_stride * 2;
        // (wide heads in large tiles: half parts leave a thread fewer offsets to keep)
        constexpr int kPart = KEYS > kPartKeys && DP == 128 ? kPartKeys / 2 : KEYS < kPartKeys ? KEYS : kPartKeys;
        constexpr int kParts = KEYS / kPart, kEach = kLoads / kParts;
        static_assert(kEach * kThreads == kPart * kChunks, "a load of a thread is of one part");
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            const int64_t from = row0 + kPart * part;
            // without rows: a resource of no bytes, never looked at beyond its base
            const int left = min(rows - kPart * part, kPart);
            const auto kr = tile_resource(a.k, left > 0 ? from * a.k_stride + head * a.dim : 0,
                                          left > 0 ? (left - 1) * k_step + a.dim * 2 : 0);
            const auto vr = tile_resource(a.v, left > 0 ? from * a.v_stride + head * a.dim : 0,
                                          left > 0 ? (left - 1) * v_step + a.dim * 2 : 0);
#pragma unroll
            for (int m = 0; m < kEach; ++m) {
                const int n = part * kEach + m;
                // all of the offset is in the operand that is checked against the resource's end
                // (kBeyond plus a tile's rows stays below 2^32)
                uint32_t k_from = (uint32_t)k_at + (uint32_t)(m * kStep * k_step);
                uint32_t v_from = (uint32_t)v_at + (uint32_t)(m * kStep * v_step);
                if (!kEven) {
                    const int e = threadIdx.x + m * kThreads, r = e / kChunks, c = e % kChunks;  // within the part
                    k_from = c * 8 < a.dim ? r * k_step + c * 16 : kBeyond;
                    v_from = c * 8 < a.dim ? r * v_step + c * 16 : kBeyond;
                }
                if (a.keep && kept[n] == 0) k_from = v_from = kBeyond;
                k[n] = __builtin_amdgcn_raw_buffer_load_b128(kr, (int)k_from, 0, 0);
                v[n] = __builtin_amdgcn_raw_buffer_load_b128(vr, (int)v_from, 0, 0);
            }
        }
        if (threadIdx.x < KEYS) {
            key_kept = (int)threadIdx.x < rows;
            if (a.keep) {
                const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.keep) + row0, 0, rows, 0x00027000);
                key_kept = __builtin_amdgcn_raw_buffer_load_b8(r, threadIdx.x, 0, 0);
            }
            if (DIST) {
                const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t *>(a.k_xy) + 2 * row0, 0, rows * 8, 0x00027000);
                place = __builtin_amdgcn_raw_buffer_load_b64(r, threadIdx.x * 8, 0, 0);
            }
        }
    }

    // NEAR: keys' factors about origin, and whether all of them are within `largest`
    template <bool DIST>
    __device__ __forceinline__ void store(const AttentionArgs &a, const Lds &lds, int2 origin = make_int2(0, 0),
                                          float largest = 0.0f) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int e = threadIdx.x + n * kThreads;
            lds.k[e / kChunks * K_PITCH + e % kChunks] = __builtin_bit_cast(i16x8, k[n]);
            lds.v[e / kChunks * V_PITCH + e % kChunks] = __builtin_bit_cast(i16x8, v[n]);
        }
        if (threadIdx.x < KEYS) {  // whole waves
            if (DIST) {
                lds.x[threadIdx.x] = (float)place.x * kPxPerQuantum;
                lds.y[threadIdx.x] = (float)place.y * kPxPerQuantum;
            }
            if (NEAR) {
                // absent keys are as near as can be
                const bool here = (int)threadIdx.x < present;
                const int bx = here ? place.x - origin.x : 0, by = here ? place.y - origin.y : 0;
                const float n = square_quanta(bx, by);
                const NearSlots s = near_key(bx, by, n);
                lds.near[threadIdx.x] = s.half[0];
                lds.near[KEYS + threadIdx.x] = s.half[1];
                const bool all = __all(near_enough(bx, by, n, largest));
                if (threadIdx.x == 0) *lds.all_near = all;
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
// where all of a query's keys are far and its scores are large.  With a cap, qk is
// the product's cap_parts().
__device__ __forceinline__ float distance2(float dx, float dy) { return __builtin_fmaf(dx, dx, dy * dy); }

template <bool DIST, int CAP>
__device__ __forceinline__ float score(float qk, float scale, float cap2, float d2, float slope2) {
    float s = CAP ? capped<CAP>(qk, cap2, cap_constant<CAP>(cap2)) : qk * scale;
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
        auto caps = [&](auto dist) {
            if (a.cap == 0.0f || a.cap >= kLargestCap) return fn(t, dp, dist, std::integral_constant<int, kNoCap>{});
            if (a.cap <= kLowCap) return fn(t, dp, dist, std::integral_constant<int, kLow>{});
            return fn(t, dp, dist, std::integral_constant<int, kHigh>{});
        };
        return a.slopes != nullptr ? caps(std::true_type{}) : caps(std::false_type{});
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
