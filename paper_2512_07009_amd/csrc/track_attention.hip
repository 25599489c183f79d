// track_attention.hip - attention of the newest detections of each track over its
// pages of keys and values in 8 bits.
//
// For query i of n (the track's last n of `length` tokens), head h, token j:
//   t = scale k_scale q_i.k_j, capped: t = cap tanh(t / cap)
//   seen: j <= p_i = length - n + i, and with a window j > p_i - window
//   out_i = sum over the tokens seen of softmax_j(t) v_scale v_j, 0 where there are none
//
// The heads that share a kv head are packed with the queries as rows r = (i, g), 16 a
// workgroup.  Its four waves take every fourth page and join what they have in LDS (many
// short tracks are one wave's each); where there are few rows, several workgroups share a
// row's pages and a second kernel joins them.  A page is read once, from memory to
// registers, a page ahead of the products.
//
// A query a track is bound by memory: 24 tracks of 27000 tokens, heads of 128, 67 us and 6
// for the join (326 MB, 4.9 TB/s), 2000 of 1800 173 (5.3); 500 of 0 to 5400 83 (337 MB,
// 4.1), where the longest tracks' workgroups end last.  96 tracks of 0 to 9000 with some
// 15 queries each and a cap 87 us: vector instructions, 75% of the time.  Tried: keys to
// float16, four tiles of rows a wave (96 clips 95 -> 232, registers), eight waves (500
// tracks 81 -> 75, but 24 long 67 -> 89 and 2000 ragged ones 94 -> 103), values shared
// by the waves in LDS (no faster).
//
// Scores are products of whole numbers on the matrix cores (16 x 16 x 64, 8 bits, exact
// sums): keys as they lie in pages, and queries as 256 a + b with a, b in 8 bits, in steps
// of 1 / 32512 of their head's largest dimension.  A dimension is off by half a step, some
// 2^-16 of the largest: below half a step of its own type from 2^-4 (float16) or 2^-7
// (bfloat16) of the largest on, while smaller ones lose digits, so that a score is off by the
// largest dimension times the sum of |k| / 65024 at most.  That spares a lane 80 instructions
// a page to convert keys to float16 (of some 350).  Scores are transposed, S^T = K Q^T: a lane
// holds 16 tokens of one row, four of each 16, which is the order in which the product with
// the values takes its weights.  Values lie in pages so that a lane's 16 bytes are the factors
// of two such products (16 x 16 x 32); they go to float16, which holds them exactly.
//
// Weights are rounded to float16 after they were summed in 32 bits, and carry the page's scale
// relative to the largest so far while that is within 2^-4 of it: those from 2^-17 of the row's
// largest on keep float16's 11 bits, others are off by 2^-28 of it at most.  Pages of smaller
// scales are multiplied without them and join the sums in 32 bits, so that a page of large
// values takes no digits of others, whether or not a row gives it any weight (500 tracks 82.8
// -> 83.5 us; with a first page of 10^6 times the others' values 84.5, 96 clips 86.8 -> 89.7).

#include "attention_common.h"
#include "tracks_common.h"

namespace flock {
namespace {

using namespace tracks;
using attention::f16x8;
using attention::kHigh;
using attention::kLow;
using attention::kNoCap;
using attention::kLog2e;
using attention::f32x16;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef half_t f16x2 __attribute__((ext_vector_type(2)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kRows = 16, kManyRows = 128;  // of a workgroup, 2^4 and 2^7
constexpr float kSlack = 8.0f;    // scores above the shift by less are left there
// From shifts of this size on scores are taken from them before anything is added: 32 bits hold a
// smaller one's difference from its shift, the level and the lift to 2^-3, which float16 has room for.
constexpr float kLarge = 0x1p20f;
// Weights are kept 2^7 times as large, 2^15 at most, so that float16's digits go that much further
// down; what leaves a workgroup is kUnlift of it.
constexpr float kLift = 7.0f, kUnlift = 0x1p-7f;
constexpr float kNear = 0x1p-4f;  // scales of values this near to the largest so far go with the weights
constexpr float kQuery = 32512.0f;  // a query's largest dimension as 256 a + b

// Eight whole numbers in float16: 1024 + u, u = x + 128, is 0x6400 | u, and 1152 is taken off.
__device__ __forceinline__ f16x8 to_half(int lo, int hi) {
    const uint32_t a = (uint32_t)lo ^ 0x80808080u, b = (uint32_t)hi ^ 0x80808080u;
    const f16x2 off = {(half_t)1152.0f, (half_t)1152.0f};
    f16x8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = __builtin_amdgcn_perm(0x64646464u, i < 2 ? a : b, i & 1 ? 0x04030402u : 0x04010400u);
        const f16x2 x = __builtin_bit_cast(f16x2, w) - off;
        r[2 * i] = x[0];
        r[2 * i + 1] = x[1];
    }
    return r;
}

// f over the four lanes that share a row.
template <typename V, typename F>
__device__ __forceinline__ V over_parts(V x, F &&f) {
    const auto bits = [](V v) { return __builtin_bit_cast(uint32_t, v); };
    const auto value = [](uint32_t v) { return __builtin_bit_cast(V, v); };
    const auto p = __builtin_amdgcn_permlane16_swap(bits(x), bits(x), false, false);
    x = f(value(p[0]), value(p[1]));
    const auto q = __builtin_amdgcn_permlane32_swap(bits(x), bits(x), false, false);
    return f(value(q[0]), value(q[1]));
}

// A score's distance from the shift.  The product is rounded by itself, as the one that the
// shift was made of, so that the largest score's distance is 0; one above it stays within what
// is left there (and NaN stays).
__device__ __forceinline__ float distance(float product, float factor, float shift) {
#pragma clang fp contract(off)
    const float score = product * factor, x = score - shift;
    return x > kSlack ? kSlack : x;
}

// What a workgroup, or the one that joins, works on.
struct Item {
    int head, row0, rows;          // rows row0 .. row0 + rows of the track's queries and shared heads
    int first_page, pages;         // that any of them sees
    Track at;
    bool ok;
};

__device__ __forceinline__ Item item_of(const TrackAttentionArgs &a, int64_t slot, int head) {
    Item s;
    int64_t tile;
    const int group = a.group, shift = a.tile_shift;
    s.at = find_track(a.tracks, slot, ((int64_t)a.tracks.total * group >> shift) + a.tracks.n_tracks,
                      [=](int offset, int t) { return ((int64_t)offset * group >> shift) + t; }, &tile);
    s.head = head;
    const int64_t all = (int64_t)s.at.n * group;
    s.ok = s.at.ok && tile >= 0 && tile << shift < all;
    s.row0 = (int)(tile << shift);
    s.rows = (int)min((int64_t)1 << shift, all - s.row0);
    const int before = s.at.length - s.at.n;  // tokens before the first query's own (may be negative)
    const int last = before + (s.row0 + s.rows - 1) / group, first = before + s.row0 / group;
    const int lo = a.window && first >= a.window ? first - a.window + 1 : 0;
    s.first_page = lo / kPage;
    s.pages = last < 0 || last < lo ? 0 : last / kPage + 1 - s.first_page;
    return s;
}

// How a query whose largest dimension has these bits goes to whole numbers.  One below
// 2^-100 is zeros, one that is not finite NaN.
struct Whole {
    float most, per;
    bool finite;
    __device__ __forceinline__ explicit Whole(uint32_t largest) {
        most = __uint_as_float(largest);
        finite = largest < 0x7f800000u;
        per = finite && most >= 0x1p-100f ? kQuery / most : 0.0f;
    }
    __device__ __forceinline__ void split(const float (&x)[16], i32x4 &high, i32x4 &low) const {
        high = low = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int n = per > 0.0f ? (int)rintf(x[e] * per) : 0;
            high[e >> 2] |= ((n + 128) >> 8 & 0xff) << (8 * (e & 3));
            low[e >> 2] |= (n & 0xff) << (8 * (e & 3));
        }
    }
    // What products of whole numbers are multiplied by, beside the page's scale (finite, so
    // that a zero times it stays one).
    template <int CAP>
    __device__ __forceinline__ float factor(const TrackAttentionArgs &a) const {
        const float scale = CAP == kHigh ? a.scale / a.cap : CAP == kLow ? 2.0f * kLog2e * a.scale / a.cap : a.scale * kLog2e;
        return finite ? fminf(scale * (per > 0.0f ? most / kQuery : 1.0f), 0x1p127f) : NAN;
    }
};

// How a page's values, of this scale, are added to rows that count in `unit`, the largest
// scale of values so far.  Near to it the weights take the quotient (level: its logarithm and
// the lift; the total takes the quotient back).  Where it would cost weights digits of
// float16, or there is none, the page's products are made by themselves and multiplied by
// `times` in 32 bits.
struct Level {
    bool near;
    float level, back, times;
    __device__ __forceinline__ Level(float v_scale, float unit) {
        near = v_scale > 0.0f && v_scale >= unit * kNear;
        level = near ? __log2f(v_scale / unit) + kLift : kLift;
        back = near ? unit / v_scale : 1.0f;
        times = v_scale > 0.0f ? v_scale / unit : 0.0f;
    }
};

// What a lane holds of a row: its dimensions as right factors, the tokens that it sees
// (lo, own], and the softmax so far.
template <int DI>
struct Row {
    i32x4 high[DI], low[DI];
    float factor;          // of products of whole numbers and the page's scale
    int lo, own;
    float shift, total;
    f32x4 acc[4 * DI];
};

template <typename T, int DI, int CAP>
__device__ __forceinline__ void begin(Row<DI> &w, const TrackAttentionArgs &a, const Item &it, int r) {
    const int part = (threadIdx.x & 63) >> 4, dim = a.cache.dim;
    const bool valid = r < it.rows;
    const int row = it.row0 + (valid ? r : 0), query = row / a.group, head = it.head * a.group + row % a.group;
    w.own = it.at.length - it.at.n + query;
    w.lo = a.window ? max(w.own, 0) - a.window : -1;
    w.shift = -INFINITY;
    w.total = 0.0f;
#pragma unroll
    for (int b = 0; b < 4 * DI; ++b) w.acc[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const T *q = static_cast<const T *>(a.q) + (int64_t)(it.at.row0 + query) * a.q_stride + head * dim;
    float x[DI][16];
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < DI; ++i) {
        const int d = 16 * (part + 4 * i);
        load_some<T, 16>(q + min(d, dim - 16), valid && d < dim ? 16 : 0, x[i]);
#pragma unroll
        for (int e = 0; e < 16; ++e) bits = max(bits, __float_as_uint(x[i][e]) & 0x7fffffffu);
    }
    bits = over_parts(bits, [](uint32_t u, uint32_t v) { return max(u, v); });
    const Whole whole(bits);
#pragma unroll
    for (int i = 0; i < DI; ++i) whole.split(x[i], w.high[i], w.low[i]);
    w.factor = whole.factor<CAP>(a);
}

template <typename T, int DI, int CAP, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, DI > 1 ? 2 : CAP == kNoCap ? 4 : 3) track_attention_kernel(TrackAttentionArgs a) {
    constexpr int kBlocks = 4 * DI;   // 16 dimensions each, at most
    __shared__ float sums[WAVES][kRows][64 * DI + 1];
    __shared__ float stats[2][WAVES][kRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane >> 4, r = lane & 15;
    const int dim = a.cache.dim, blocks = dim / 16;
    const uint32_t block_id = a.gathered ? (uint32_t)attention::xcd_order(blockIdx.x, gridDim.x) : blockIdx.x;
    const uint32_t id = block_id / a.splits, heads = a.cache.kv_heads;
    const int split = (int)(block_id - id * a.splits);
    const Item it = item_of(a, id / heads, (int)(id % heads));
    if (!it.ok) return;
    const int active = max((it.pages + a.split_pages - 1) / a.split_pages, 1);
    if (split >= active) return;
    const int p0 = it.first_page + split * a.split_pages + wave;
    const int p1 = min(it.first_page + (split + 1) * a.split_pages, it.first_page + it.pages);
    const int count = p1 > p0 ? (p1 - p0 + WAVES - 1) / WAVES : 0;  // of this wave: p0, p0 + 4, ...

    Row<DI> w;
    begin<T, DI, CAP>(w, a, it, r);
    const float cap2 = a.cap * kLog2e, constant = attention::cap_constant<CAP>(cap2);

    // the wave's pages, 64 at a time, a lane each
    int my_page = -1;
    float my_k = 0.0f, my_v = 0.0f;
    const int32_t *table = a.tracks.table + (int64_t)it.at.index * a.tracks.table_stride;
    // the next page from the n-th on that is one of the pool (tokens of others are not seen), and its number
    const auto next = [&](int &n) {
        for (; n < count; ++n) {
            if ((n & 63) == 0) {
                const int mine = n + lane;
                my_page = mine < count ? table[p0 + WAVES * mine] : -1;
                if (my_page >= a.cache.pages) my_page = -1;
                const int64_t block = (int64_t)max(my_page, 0) * a.cache.kv_heads + it.head;
                my_k = my_page >= 0 ? a.cache.k_scale[block] : 0.0f;
                my_v = my_page >= 0 ? a.cache.v_scale[block] : 0.0f;
                asm volatile("" ::"v"(my_k), "v"(my_v));  // (waited for here, not where pages' loads are on their way)
            }
            const int page = __builtin_amdgcn_readlane(my_page, n & 63);
            if (page >= 0) return page;
        }
        return -1;
    };
    const auto scale_of = [&](float mine, int n) {
        return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), n & 63));
    };
    i32x4 kr[4][DI], vr[kBlocks];
    const auto load_k = [&](int page) {
        const int8_t *p = a.cache.k + ((int64_t)page * a.cache.kv_heads + it.head) * (kPage * dim) + r * dim + 16 * part;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < DI; ++i) {
                kr[b][i] = i32x4{0, 0, 0, 0};
                if (part + 4 * i < blocks) kr[b][i] = *reinterpret_cast<const i32x4 *>(p + 16 * b * dim + 64 * i);
            }
    };
    const auto load_v = [&](int page) {
        const int8_t *p = a.cache.v + ((int64_t)page * a.cache.kv_heads + it.head) * (kPage * dim) + r * kPage + 16 * part;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
            if (b < blocks) vr[b] = *reinterpret_cast<const i32x4 *>(p + 16 * b * kPage);
    };

    float unit = 0.0f;  // largest scale of values so far
    bool large = false;  // some row's shift is
    // tokens that every row sees, of pages that lie within
    const int all_lo = a.window ? max(it.at.length - it.at.n + (it.row0 + it.rows - 1) / a.group, 0) - a.window : -1;
    const int all_own = it.at.length - it.at.n + it.row0 / a.group;
    int n = 0, page = next(n);
    if (page >= 0) {
        load_k(page);
        load_v(page);
    }
    while (page >= 0) {
        const int token0 = (p0 + WAVES * n) * kPage;
        const float k_scale = scale_of(my_k, n), v_scale = scale_of(my_v, n);
        ++n;
        const int after = next(n);
        float keep_v = 1.0f;
        if (v_scale > unit) {
            keep_v = unit / v_scale;
            unit = v_scale;
        }
        const Level values(v_scale, unit);
        const bool inside = token0 + kPage - 1 <= all_own && token0 > all_lo;
        f16x8 weights[2];
        f32x16 s;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            i32x4 high = {0, 0, 0, 0}, low = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < DI; ++i) {
                high = __builtin_amdgcn_mfma_i32_16x16x64_i8(kr[b][i], w.high[i], high, 0, 0, 0);
                low = __builtin_amdgcn_mfma_i32_16x16x64_i8(kr[b][i], w.low[i], low, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * b + e] = (float)(256 * high[e] + low[e]);
        }
        if (after >= 0) load_k(after);
        float f = w.factor * k_scale;
        if (f > 0x1p127f) f = 0x1p127f;  // (NaN stays)
        if (CAP != kNoCap) {
            attention::cap_parts<CAP>(s, f);
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = attention::capped<CAP>(s[e], cap2, constant);
            f = 1.0f;
        }
        if (!inside) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int token = token0 + 16 * (e >> 2) + 4 * part + (e & 3);
                s[e] = token > w.own || token <= w.lo ? -INFINITY : s[e] * f;
            }
            f = 1.0f;
        }
        float most = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) most = fmaxf(most, s[e]);
        most = over_parts(most, [](float u, float v) { return fmaxf(u, v); }) * f;
        float keep = keep_v;
        if (__any(most > w.shift + kSlack || (w.shift == -INFINITY && most > w.shift))) {
            const float now = fmaxf(w.shift, most);
            const float less = w.shift == -INFINITY ? 0.0f : attention::exp2_fast(w.shift - now);
            w.total *= less;
            keep *= less;
            w.shift = now;
            large = __any(fabsf(now) > kLarge && now != -INFINITY);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) w.acc[b] *= keep;
        } else if (keep_v != 1.0f) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) w.acc[b] *= keep;
        }
        float from = w.shift == -INFINITY ? 0.0f : w.shift;
        if (large) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = distance(s[e], f, from);
            f = 1.0f;
            from = 0.0f;
        }
        const float base = from - values.level;
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float x = attention::exp2_fast(__builtin_fmaf(s[e], f, -base));
            sum += x;
            weights[e >> 3][e & 7] = (half_t)x;
        }
        w.total += sum * values.back;
        if (v_scale != v_scale) {  // values that are not finite: none for rows that see the page, whatever its weight
            // (a branch, which keeps the values' registers apart from the scores' where those are fewest)
            if (CAP == kNoCap) asm volatile("" ::: "memory");
            if (most != -INFINITY) w.total = NAN;
        }
        const auto product = [&](int b, f32x4 to) {
            const f16x8 v0 = to_half(vr[b][0], vr[b][1]), v1 = to_half(vr[b][2], vr[b][3]);
            to = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, weights[0], to, 0, 0, 0);
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, weights[1], to, 0, 0, 0);
        };
        if (values.near) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
                if (b < blocks) w.acc[b] = product(b, w.acc[b]);
        } else {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
                if (b < blocks) w.acc[b] += product(b, f32x4{0.0f, 0.0f, 0.0f, 0.0f}) * values.times;
        }
        if (after >= 0) load_v(after);
        page = after;
    }

    // the waves' parts, joined
    w.total = over_parts(w.total, [](float u, float v) { return u + v; }) * kUnlift;
    unit *= kUnlift;
    if (part == 0) stats[0][wave][r] = w.shift;
    __syncthreads();
    float now = stats[0][0][r];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) now = fmaxf(now, stats[0][v][r]);
    // (a shift that nothing has moved: no token, or none but NaN)
    const float keep = w.shift == -INFINITY ? (w.total == w.total ? 0.0f : w.total) : attention::exp2_fast(w.shift - now);
    if (part == 0) stats[1][wave][r] = w.total * keep;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[wave][r][16 * b + 4 * part + e] = w.acc[b][e] * (keep * unit);
    __syncthreads();
    // a wave a row, a lane a dimension
#pragma unroll 1
    for (int rr = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); rr < it.rows; rr += WAVES) {
        float l = 0.0f, m = -INFINITY;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            l += stats[1][v][rr];
            m = fmaxf(m, stats[0][v][rr]);
        }
        const uint32_t row = it.row0 + rr, query = row / (uint32_t)a.group;
        const int64_t bird = it.at.row0 + query;
        const int head = it.head * a.group + (int)(row - query * a.group);
        const int64_t to = ((int64_t)split * a.tracks.total + bird) * a.q_heads + head;
        for (int d = threadIdx.x & 63; d < dim; d += 64) {
            float o = 0.0f;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) o += sums[v][rr][d];
            if (active == 1) static_cast<T *>(a.out)[bird * a.out_stride + head * dim + d] = static_cast<T>(l == 0.0f ? 0.0f : o / l);
            else a.part_out[to * dim + d] = o;
        }
        if (active > 1 && (threadIdx.x & 63) == 0) reinterpret_cast<float2 *>(a.part_stat)[to] = make_float2(m, l);
    }
}

// ---------------------------------------------------------------------------
// Many rows: 128 a workgroup, 32 a wave, all waves over the same pages.
//
// Pages go to LDS as they are, without registers in between, kAhead pages ahead of the
// products: a page waits for its own loads alone (they come back in order), with one
// barrier a page.  Chunks of 16 bytes of a key or of a dimension are stored in an order
// that turns with it, so that the 32 that a wave reads a chunk of lie in different banks.
// Products are 32 x 32 x 32 (8 bits) and 32 x 32 x 16: a lane holds 32 tokens of one row, and
// of a dimension it takes the two parts that hold the same tokens.  Bound by vector
// instructions, some seven a score and 80 a page to convert its values: 64 tracks of 1000
// with 1000 queries, 4 heads on each of 2, 167 us (392 TFLOP/s), with 16 rows a workgroup 359.
// ---------------------------------------------------------------------------

constexpr int kAhead = 3, kBuffers = kAhead + 1;

template <int DP>
struct ManyShared {
    int8_t k[kBuffers][kPage * DP], v[kBuffers][DP * kPage];
};

// Where chunk `chunk` (16 bytes) of a row of WIDTH bytes lies in LDS.
template <int WIDTH>
__device__ __forceinline__ int turned(int row, int chunk) {
    return WIDTH == 64 ? chunk ^ ((row >> 2) & 3) : chunk ^ ((row >> 1) & 7);
}

// Waits for LDS, and for all but the last N loads.
template <int N>
__device__ __forceinline__ void wait_but() {
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x070);
}

// The compiler moves no access to memory over this.
__device__ __forceinline__ void stand() { asm volatile("" ::: "memory"); }

template <typename T, int DP, int CAP>
__global__ void __launch_bounds__(kThreads, DP == 64 ? 3 : 2) track_rows_kernel(TrackAttentionArgs a) {
    constexpr int kChunks = DP / 16, kSteps = DP / 32, kBlocks = DP / 32;
    constexpr int kLoads = kPage * DP / 16 / kThreads;  // of 16 bytes a thread, for keys and for values
    __shared__ ManyShared<DP> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, r = lane & 31;
    const int dim = a.cache.dim;
    const uint32_t block_id = a.gathered ? (uint32_t)attention::xcd_order(blockIdx.x, gridDim.x) : blockIdx.x;
    const uint32_t id = block_id / a.splits, heads = a.cache.kv_heads;
    const int split = (int)(block_id - id * a.splits);
    const Item it = item_of(a, id / heads, (int)(id % heads));
    if (!it.ok) return;
    const int active = max((it.pages + a.split_pages - 1) / a.split_pages, 1);
    if (split >= active) return;
    const int p0 = it.first_page + split * a.split_pages;
    const int count = min(a.split_pages, it.first_page + it.pages - p0);

    // this lane's row: its dimensions as right factors, and the tokens that it sees
    const int at = 32 * wave + r;
    const bool valid = at < it.rows;
    const int row = it.row0 + (valid ? at : 0), query = row / a.group, head = it.head * a.group + row % a.group;
    const int before = it.at.length - it.at.n, own = before + query;
    const int lo = a.window ? max(own, 0) - a.window : -1;  // tokens in (lo, own]
    i32x4 high[kSteps], low[kSteps];
    float factor;
    {
        const T *q = static_cast<const T *>(a.q) + (int64_t)(it.at.row0 + query) * a.q_stride + head * dim;
        float x[kSteps][16];
        uint32_t bits = 0;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int d = 32 * i + 16 * h;
            load_some<T, 16>(q + min(d, dim - 16), valid && d < dim ? 16 : 0, x[i]);
#pragma unroll
            for (int e = 0; e < 16; ++e) bits = max(bits, __float_as_uint(x[i][e]) & 0x7fffffffu);
        }
        bits = max(bits, (uint32_t)__shfl_xor((int)bits, 32));
        const Whole whole(bits);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) whole.split(x[i], high[i], low[i]);
        factor = whole.factor<CAP>(a);
    }
    const float cap2 = a.cap * kLog2e, constant = attention::cap_constant<CAP>(cap2);
    // tokens that some and that every row of the wave sees
    const bool some_rows = 32 * wave < it.rows;
    const int wave_first = before + (it.row0 + 32 * wave) / a.group;
    const int wave_last = before + (it.row0 + min(32 * wave + 31, it.rows - 1)) / a.group;
    const int all_lo = a.window ? max(wave_last, 0) - a.window : -1, some_lo = a.window ? max(wave_first, 0) - a.window : -1;

    int my_page = -1;
    float my_k = 0.0f, my_v = 0.0f;
    const int32_t *table = a.tracks.table + (int64_t)it.at.index * a.tracks.table_stride;
    const auto next = [&](int &n) {
        for (; n < count; ++n) {
            if ((n & 63) == 0) {
                const int mine = n + lane;
                my_page = mine < count ? table[p0 + mine] : -1;
                if (my_page >= a.cache.pages) my_page = -1;
                const int64_t block = (int64_t)max(my_page, 0) * a.cache.kv_heads + it.head;
                my_k = my_page >= 0 ? a.cache.k_scale[block] : 0.0f;
                my_v = my_page >= 0 ? a.cache.v_scale[block] : 0.0f;
                asm volatile("" ::"v"(my_k), "v"(my_v));  // (waited for here, not where pages' loads are on their way)
            }
            const int page = __builtin_amdgcn_readlane(my_page, n & 63);
            if (page >= 0) return page;
        }
        return -1;
    };
    const auto scale_of = [&](float mine, int n) {
        return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), n & 63));
    };
    // the stream of pages: number, scales, and loads into the buffers in turn
    struct Ahead {
        int n;  // -1: none
        float k, v;
    };
    int n_next = 0, buffer_next = 0;
    const auto load = [&]() -> Ahead {
        const int page = next(n_next);
        if (page < 0) return {-1, 0.0f, 0.0f};
        const Ahead one = {n_next, scale_of(my_k, n_next), scale_of(my_v, n_next)};
        ++n_next;
        const int64_t block = ((int64_t)page * a.cache.kv_heads + it.head) * (kPage * dim);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int slot = i * kThreads + threadIdx.x, token = slot / kChunks, chunk = turned<DP>(token, slot % kChunks);
            // (dimensions beyond the head's: queries have zeros there)
            const int8_t *from = a.cache.k + block + token * dim + 16 * (16 * chunk < dim ? chunk : 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                             (__attribute__((address_space(3))) void *)(shared.k[buffer_next] + 16 * (i * kThreads + 64 * wave)),
                                             16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int slot = i * kThreads + threadIdx.x, d = slot >> 2, part = turned<kPage>(d, slot & 3);
            // (... and nothing is stored of them)
            const int8_t *from = a.cache.v + block + (d < dim ? d : 0) * kPage + 16 * part;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                             (__attribute__((address_space(3))) void *)(shared.v[buffer_next] + 16 * (i * kThreads + 64 * wave)),
                                             16, 0, 0);
        }
        buffer_next = (buffer_next + 1) & (kBuffers - 1);
        return one;
    };

    f32x16 acc[kBlocks] = {};
    float shift = -INFINITY, total = 0.0f, unit = 0.0f;
    bool large = false;
    static_assert(kAhead == 3, "the pages ahead have a name each");
    Ahead now = load(), second = load(), third = load();
    int buffer = 0;
    while (now.n >= 0) {
        const int token0 = (p0 + now.n) * kPage;
        const float k_scale = now.k, v_scale = now.v;
        stand();
        if (third.n >= 0) wait_but<(kAhead - 1) * 2 * kLoads>();
        else wait_but<0>();
        stand();
        __builtin_amdgcn_s_barrier();  // this page is there, and the one before has been read by all
        stand();
        now = second;
        second = third;
        third = load();
        if (some_rows && token0 <= wave_last && token0 + kPage - 1 > some_lo) {
            float keep_v = 1.0f;
            if (v_scale > unit) {
                keep_v = unit / v_scale;
                unit = v_scale;
            }
            const Level values(v_scale, unit);
            f32x16 s[2];
            float f = factor * k_scale;
            if (f > 0x1p127f) f = 0x1p127f;  // (NaN stays)
            float g = f;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int token = 32 * t + r;
                i32x16 hi = {}, lw = {};
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const i32x4 k = *reinterpret_cast<const i32x4 *>(shared.k[buffer] + token * DP + 16 * turned<DP>(token, 2 * i + h));
                    hi = __builtin_amdgcn_mfma_i32_32x32x32_i8(k, high[i], hi, 0, 0, 0);
                    lw = __builtin_amdgcn_mfma_i32_32x32x32_i8(k, low[i], lw, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) s[t][e] = (float)(256 * hi[e] + lw[e]);
                if (CAP != kNoCap) {
                    attention::cap_parts<CAP>(s[t], f);
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[t][e] = attention::capped<CAP>(s[t][e], cap2, constant);
                    g = 1.0f;
                }
            }
            if (token0 + kPage - 1 > wave_first || token0 <= all_lo) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int token = token0 + 32 * t + attention::out_row(e, h);
                        s[t][e] = token > own || token <= lo ? -INFINITY : s[t][e] * g;
                    }
                g = 1.0f;
            }
            float most = s[0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) most = fmaxf(most, s[t][e]);
            most = attention::across(most, [](float u, float v) { return fmaxf(u, v); }) * g;
            float keep = keep_v;
            if (__any(most > shift + kSlack || (shift == -INFINITY && most > shift))) {
                const float now = fmaxf(shift, most);
                const float less = shift == -INFINITY ? 0.0f : attention::exp2_fast(shift - now);
                total *= less;
                keep *= less;
                shift = now;
                large = __any(fabsf(now) > kLarge && now != -INFINITY);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) acc[b] *= keep;
            } else if (keep_v != 1.0f) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) acc[b] *= keep;
            }
            float from = shift == -INFINITY ? 0.0f : shift;
            if (large) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[t][e] = distance(s[t][e], g, from);
                g = 1.0f;
                from = 0.0f;
            }
            const float base = from - values.level;
            float sum = 0.0f;
            f16x8 weights[4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float x = attention::exp2_fast(__builtin_fmaf(s[t][e], g, -base));
                    sum += x;
                    weights[2 * t + (e >> 3)][e & 7] = (half_t)x;
                }
            total += sum * values.back;
            if (v_scale != v_scale) {  // values that are not finite: none for rows that see the page, whatever its weight
                stand();               // (a branch, which keeps the values' registers apart from the scores')
                if (most != -INFINITY) total = NAN;
            }
            const auto product = [&](int b, f32x16 to) {
                const int d = 32 * b + r;
                const int8_t *v = shared.v[buffer] + d * kPage;
                const i32x4 x = *reinterpret_cast<const i32x4 *>(v + 16 * turned<kPage>(d, h));
                const i32x4 y = *reinterpret_cast<const i32x4 *>(v + 16 * turned<kPage>(d, h + 2));
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    to = __builtin_amdgcn_mfma_f32_32x32x16_f16(to_half(x[i], y[i]), weights[i], to, 0, 0, 0);
                return to;
            };
            if (values.near) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) acc[b] = product(b, acc[b]);
            } else {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    acc[b] += product(b, f32x16{}) * values.times;
                    __builtin_amdgcn_sched_barrier(0);  // (one product's registers at a time)
                }
            }
        }
        buffer = (buffer + 1) & (kBuffers - 1);
    }
    total = attention::across(total, [](float u, float v) { return u + v; }) * kUnlift;
    unit *= kUnlift;
    if (!valid) return;
    const int64_t bird = it.at.row0 + query;
    // (a shift that nothing has moved: no token, or none but NaN)
    const bool none = shift == -INFINITY && total == total;
    if (active == 1) {
        T *out = static_cast<T *>(a.out) + bird * a.out_stride + head * dim;
        const float per = none || total == 0.0f ? 0.0f : unit / total;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int d = 32 * b + 8 * q + 4 * h;
                const float o[4] = {acc[b][4 * q] * per, acc[b][4 * q + 1] * per, acc[b][4 * q + 2] * per, acc[b][4 * q + 3] * per};
                if (d < dim) store_pack<T, 4>(out + d, o);
            }
        return;
    }
    const int64_t to = ((int64_t)split * a.tracks.total + bird) * a.q_heads + head;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int d = 32 * b + 8 * q + 4 * h;
            const float o[4] = {acc[b][4 * q] * unit, acc[b][4 * q + 1] * unit, acc[b][4 * q + 2] * unit, acc[b][4 * q + 3] * unit};
            if (d < dim) store_pack<float, 4>(a.part_out + to * dim + d, o);
        }
    if (h == 0) {
        a.part_stat[2 * to] = shift;
        a.part_stat[2 * to + 1] = total;
    }
}

// Rows whose pages several workgroups shared: a wave a row, a lane a dimension (or two)
// of all shares, whose weights are found first, a lane a share.
template <typename T>
__global__ void __launch_bounds__(kThreads) track_join_kernel(TrackAttentionArgs a) {
    const uint32_t id = blockIdx.x, heads = a.cache.kv_heads;
    const Item it = item_of(a, id / heads, (int)(id % heads));
    const int rr = kWaves * blockIdx.y + (threadIdx.x >> 6);
    if (!it.ok || rr >= it.rows) return;
    const int active = (it.pages + a.split_pages - 1) / a.split_pages;
    if (active <= 1) return;
    const int dim = a.cache.dim, lane = threadIdx.x & 63, d0 = min(lane, dim - 1), d1 = min(lane + 64, dim - 1);
    const int row = it.row0 + rr, head = it.head * a.group + row % a.group;
    const int64_t bird = it.at.row0 + row / a.group;
    const int64_t pitch = (int64_t)a.tracks.total * a.q_heads, at = bird * a.q_heads + head;
    float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int first = 0; first < active; first += 64) {
        const int s = first + lane, here = min(active - first, 64);
        float2 stat = make_float2(-INFINITY, 0.0f);
        if (s < active) stat = reinterpret_cast<const float2 *>(a.part_stat)[s * pitch + at];
        float now = stat.x;
        now = over_lanes<64>(now, [](float u, float v) { return fmaxf(u, v); });
        now = fmaxf(now, m);
        if (now > m) {
            if (m != -INFINITY) {
                const float less = attention::exp2_fast(m - now);
                l *= less;
                o0 *= less;
                o1 *= less;
            }
            m = now;
        }
        const float keep = stat.y == 0.0f ? 0.0f : stat.x == -INFINITY ? stat.y : attention::exp2_fast(stat.x - m);
        float sum = stat.y * keep;
        sum = over_lanes<64>(sum, [](float u, float v) { return u + v; });
        l += sum;
        const float *p = a.part_out + (first * pitch + at) * dim;
#pragma unroll 8
        for (int i = 0; i < here; ++i, p += pitch * dim) {
            const float k = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(keep), i));
            o0 += p[d0] * k;
            o1 += p[d1] * k;
        }
    }
    T *out = static_cast<T *>(a.out) + bird * a.out_stride + head * dim;
    if (lane < dim) out[lane] = static_cast<T>(l == 0.0f ? 0.0f : o0 / l);
    if (lane + 64 < dim) out[lane + 64] = static_cast<T>(l == 0.0f ? 0.0f : o1 / l);
}

template <typename T, int DI, int WAVES>
void launch_few(const TrackAttentionArgs &a, dim3 grid, hipStream_t stream) {
    const dim3 block(64 * WAVES);
    if (a.cap == 0.0f) hipLaunchKernelGGL((track_attention_kernel<T, DI, kNoCap, WAVES>), grid, block, 0, stream, a);
    else if (a.cap <= attention::kLowCap) hipLaunchKernelGGL((track_attention_kernel<T, DI, kLow, WAVES>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((track_attention_kernel<T, DI, kHigh, WAVES>), grid, block, 0, stream, a);
}

template <typename T, int DP>
void launch_many(const TrackAttentionArgs &a, dim3 grid, hipStream_t stream) {
    if (a.cap == 0.0f) hipLaunchKernelGGL((track_rows_kernel<T, DP, kNoCap>), grid, dim3(kThreads), 0, stream, a);
    else if (a.cap <= attention::kLowCap) hipLaunchKernelGGL((track_rows_kernel<T, DP, kLow>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((track_rows_kernel<T, DP, kHigh>), grid, dim3(kThreads), 0, stream, a);
}

template <typename T>
hipError_t launch_type(const TrackAttentionArgs &a, const TrackPlan &p, hipStream_t stream) {
    const int64_t items = p.slots * a.cache.kv_heads;
    const dim3 grid((uint32_t)(items * p.splits));
    if (p.tile_rows == kRows) {
        if (a.cache.dim <= 64) p.waves == 1 ? launch_few<T, 1, 1>(a, grid, stream) : launch_few<T, 1, kWaves>(a, grid, stream);
        else p.waves == 1 ? launch_few<T, 2, 1>(a, grid, stream) : launch_few<T, 2, kWaves>(a, grid, stream);
    } else {
        if (a.cache.dim <= 64) launch_many<T, 64>(a, grid, stream);
        else launch_many<T, 128>(a, grid, stream);
    }
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || p.splits == 1) return err;
    hipLaunchKernelGGL((track_join_kernel<T>), dim3((uint32_t)items, p.tile_rows / kWaves), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

TrackPlan plan_track_attention(int32_t n_tracks, int32_t total, int32_t max_pages, int32_t q_heads, int32_t kv_heads,
                               int n_cus) {
    TrackPlan p;
    const int group = q_heads / kv_heads;
    // 128 rows a workgroup where tracks have more on average and those fill the card: 64 tracks
    // of 1000 queries of 4 heads 359 -> 182 us, but 16 tracks of 100 of 2000 tokens 33 -> 43
    const int64_t rows = (int64_t)total * group;
    const bool many = rows > kManyRows * (int64_t)n_tracks && rows / kManyRows * kv_heads >= n_cus;
    p.tile_rows = many ? kManyRows : kRows;
    p.slots = (int64_t)total * group / p.tile_rows + n_tracks;
    // as many workgroups as the card holds at a time, of at least two pages a wave: with
    // more of them some begin when others end (24 tracks of 27000, heads of 128: two a
    // compute unit 68 us, four 77, eight 88); three where a tile's rows are at least half there
    // and instructions are what takes the time (256 tracks of 4000, 16 heads of 128 that share
    // one: two 68 us, three 52, four 83; 96 of 0 to 9000 with 5 queries of 4 heads 50, 45, 50)
    const int64_t items = std::max<int64_t>(n_tracks, (int64_t)total * group / p.tile_rows) * kv_heads;
    const int resident = many || rows >= kRows / 2 * (int64_t)n_tracks ? 3 : 2;
    // one wave a workgroup where short tracks fill the card so (4096 of 64 tokens 48 -> 22 us, of 256
    // 68 -> 49; of 1024 196 -> 204, 2000 of up to 1800 94 -> 110)
    p.waves = !many && max_pages <= 8 && items >= 12 * (int64_t)n_cus ? 1 : kWaves;
    int64_t splits = resident * (int64_t)n_cus / items;
    splits = std::max<int64_t>(std::min<int64_t>(splits, (max_pages + 2 * kWaves - 1) / (2 * kWaves)), 1);
    p.split_pages = std::max((int32_t)((max_pages + splits - 1) / splits), 1);
    p.splits = std::max((max_pages + p.split_pages - 1) / p.split_pages, 1);
    return p;
}

size_t track_attention_workspace_bytes(const TrackPlan &p, int32_t total, int32_t q_heads, int32_t dim) {
    return p.splits == 1 ? 0 : (size_t)p.splits * total * q_heads * (dim + 2) * sizeof(float);
}

hipError_t launch_track_attention(TrackAttentionArgs a, int32_t dtype, const TrackPlan &p, void *workspace,
                                  hipStream_t stream) {
    a.group = a.q_heads / a.cache.kv_heads;
    a.tile_shift = p.tile_rows == kManyRows ? 7 : 4;
    // workgroups of a track that read the same pages meet in one XCD's L2 (96 clips: 102 -> 94 us);
    // with one tile a track they would only be spread less evenly (24 long tracks: 67 -> 84)
    a.gathered = (int64_t)a.tracks.total * a.group > kRows * (int64_t)a.tracks.n_tracks;
    a.splits = p.splits;
    a.split_pages = p.split_pages;
    a.part_stat = static_cast<float *>(workspace);
    a.part_out = a.part_stat + (size_t)2 * p.splits * a.tracks.total * a.q_heads;
    if (a.cap >= attention::kLargestCap) a.cap = 0.0f;
    return dtype == FLOCK_F16 ? launch_type<half_t>(a, p, stream) : launch_type<bf16_t>(a, p, stream);
}

}  // namespace flock
