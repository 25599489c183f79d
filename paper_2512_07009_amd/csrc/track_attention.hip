// track_attention.hip - attention of the newest detections of each track over its
// pages of keys and values in 8 bits.
//
// For query i of n (the track's last n of `length` tokens), head h, token j:
//   t = scale k_scale q_i.k_j, capped: t = cap tanh(t / cap)
//   seen: j <= p_i = length - n + i, and with a window j > p_i - window
//   out_i = sum over the tokens seen of softmax_j(t) v_scale v_j, 0 where there are none
//
// The heads that share a kv head are packed with the queries as rows r = (i, g), 16 a
// workgroup.  Its four waves take every fourth page and join what they have in LDS;
// where there are few rows, several workgroups share a row's pages and a second kernel
// joins them.  Bound by the bytes of the pages for single tokens.
//
// Whole numbers of 8 bits are exact in float16, so products run on the matrix cores in
// float16 (16 x 16 x 32) with no rounding of keys and values.  Queries in bfloat16 are
// scaled by a power of two that brings their largest dimension near 1: exact above 2^-14
// of it, and below off by 2^-25 of it at most.  Scores are transposed, S^T = K Q^T: a
// lane holds 16 tokens of one row, four of each 16, which is the order in which the
// product with the values takes its weights; the values lie in pages so that a lane's 16
// bytes are the factors of two such products.  Weights carry the page's scale relative to
// the largest so far and are rounded to float16 (2^-11), after they were summed in 32 bits.

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

constexpr int kThreads = 256, kWaves = 4, kRows = 16;
constexpr float kSlack = 8.0f;  // scores above the shift by less are left there

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

template <typename F>
__device__ __forceinline__ float over_parts(float x, F &&f) {
    x = f(x, __shfl_xor(x, 16));
    return f(x, __shfl_xor(x, 32));
}

// What a workgroup, or the one that joins, works on.
struct Item {
    int track, head, row0, rows;   // rows row0 .. row0 + rows of the track's queries and shared heads
    int first_page, pages;         // that any of them sees
    Track at;
    bool ok;
};

__device__ __forceinline__ Item item_of(const TrackAttentionArgs &a, int64_t slot, int head) {
    Item s;
    int64_t tile;
    const int group = a.group;
    s.track = find_track(a.tracks.n_tracks, slot,
                         [&](int i) { return (int64_t)a.tracks.offsets[i] * group / kRows + i; }, &tile);
    s.at = track_of(a.tracks, s.track);
    s.head = head;
    const int64_t all = (int64_t)s.at.n * group;
    s.ok = s.at.ok && tile >= 0 && tile * kRows < all;
    s.row0 = (int)(tile * kRows);
    s.rows = (int)min((int64_t)kRows, all - s.row0);
    const int before = s.at.length - s.at.n;  // tokens before the first query's own (may be negative)
    const int last = before + (s.row0 + s.rows - 1) / group, first = before + s.row0 / group;
    const int lo = a.window && first >= a.window ? first - a.window + 1 : 0;
    s.first_page = lo / kPage;
    s.pages = last < 0 || last < lo ? 0 : last / kPage + 1 - s.first_page;
    return s;
}

template <typename T, int DI, int CAP>
__global__ void __launch_bounds__(kThreads) track_attention_kernel(TrackAttentionArgs a) {
    constexpr int kBlocks = 4 * DI;   // 16 dimensions each, at most
    __shared__ float sums[kWaves][kRows][64 * DI + 1];
    __shared__ float stats[2][kWaves][kRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane >> 4, r = lane & 15;
    const int dim = a.cache.dim, blocks = dim / 16;
    const int split = (int)(blockIdx.x % a.splits);
    const int64_t id = blockIdx.x / a.splits;
    const Item it = item_of(a, id / a.cache.kv_heads, (int)(id % a.cache.kv_heads));
    if (!it.ok) return;
    const int active = max((it.pages + a.split_pages - 1) / a.split_pages, 1);
    if (split >= active) return;
    const int p0 = it.first_page + split * a.split_pages;
    const int p1 = min(p0 + a.split_pages, it.first_page + it.pages);

    // this lane's row: its dimensions as right factors, and the tokens that it sees
    const bool valid = r < it.rows;
    const int row = it.row0 + (valid ? r : 0), query = row / a.group, head = it.head * a.group + row % a.group;
    const int own = it.at.length - it.at.n + query;
    const int lo = a.window ? max(own, 0) - a.window : -1;  // tokens in (lo, own]
    const T *qp = static_cast<const T *>(a.q) + (int64_t)(it.at.row0 + query) * a.q_stride + head * dim;
    f16x8 q[DI][2];
    float q_scale = 1.0f;
    {
        float x[DI][2][8], most = 0.0f;
#pragma unroll
        for (int i = 0; i < DI; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int d = 16 * (part + 4 * i) + 8 * h;
                load_some<T, 8>(qp + min(d, dim - 8), valid && d < dim ? 8 : 0, x[i][h]);
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[i][h][e]));
            }
        most = over_parts(most, [](float u, float v) { return fmaxf(u, v); });
        int exponent = 0;
        if (sizeof(T) == 2 && !__is_same(T, half_t) && most > 0.0f && most < INFINITY) exponent = ilogbf(most);
        q_scale = ldexpf(1.0f, max(exponent, -126));
#pragma unroll
        for (int i = 0; i < DI; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 8; ++e) q[i][h][e] = (half_t)ldexpf(x[i][h][e], -max(exponent, -126));
    }
    // (finite, so that a zero times it stays one)
    const float factor = fminf((CAP == kHigh ? a.scale / a.cap : CAP == kLow ? 2.0f * kLog2e * a.scale / a.cap : a.scale * kLog2e) * q_scale, 0x1p127f);
    const float cap2 = a.cap * kLog2e, constant = attention::cap_constant<CAP>(cap2);

    f32x4 acc[kBlocks] = {};
    float shift = -INFINITY, total = 0.0f, unit = 0.0f;
    // tokens that every row sees, of pages that lie within
    const int all_lo = a.window ? max(it.at.length - it.at.n + (it.row0 + it.rows - 1) / a.group, 0) - a.window : -1;
    const int all_own = it.at.length - it.at.n + it.row0 / a.group;
    int batch = 0, my_page = -1;
    float my_k = 0.0f, my_v = 0.0f;
    for (int n = 0, p = p0 + wave; p < p1; ++n, p += kWaves) {
        if ((n & 63) == 0) {  // the next 64 pages of this wave, a lane each
            batch = n;
            const int mine = p + kWaves * lane;
            my_page = mine < p1 ? a.tracks.table[(int64_t)it.track * a.tracks.table_stride + mine] : -1;
            if (my_page >= a.cache.pages) my_page = -1;
            const int64_t block = (int64_t)max(my_page, 0) * a.cache.kv_heads + it.head;
            my_k = my_page >= 0 ? a.cache.k_scale[block] : 0.0f;
            my_v = my_page >= 0 ? a.cache.v_scale[block] : 0.0f;
        }
        const int page = __builtin_amdgcn_readlane(my_page, n - batch);
        if (page < 0) continue;  // no page of the pool: its tokens are not seen
        const float k_scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_k), n - batch));
        const float v_scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_v), n - batch));
        const int64_t block = ((int64_t)page * a.cache.kv_heads + it.head) * (kPage * dim);
        const int8_t *kp = a.cache.k + block + r * dim + 16 * part, *vp = a.cache.v + block + r * kPage + 16 * part;
        i32x4 kr[4][DI], vr[kBlocks];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < DI; ++i) {
                kr[b][i] = i32x4{0, 0, 0, 0};
                if (part + 4 * i < blocks) kr[b][i] = *reinterpret_cast<const i32x4 *>(kp + 16 * b * dim + 64 * i);
            }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
            if (b < blocks) vr[b] = *reinterpret_cast<const i32x4 *>(vp + 16 * b * kPage);
        f32x16 s;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            f32x4 c = {};
#pragma unroll
            for (int i = 0; i < DI; ++i) {
                c = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_half(kr[b][i][0], kr[b][i][1]), q[i][0], c, 0, 0, 0);
                c = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_half(kr[b][i][2], kr[b][i][3]), q[i][1], c, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * b + e] = c[e];
        }
        float f = factor * k_scale;
        if (f > 0x1p127f) f = 0x1p127f;  // (NaN stays)
        if (CAP == kNoCap) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] *= f;
        } else {
            attention::cap_parts<CAP>(s, f);
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = attention::capped<CAP>(s[e], cap2, constant);
        }
        const int token0 = p * kPage;
        if (token0 + kPage - 1 > all_own || token0 <= all_lo) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int token = token0 + 16 * (e >> 2) + 4 * part + (e & 3);
                if (token > own || token <= lo) s[e] = -INFINITY;
            }
        }
        float most = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) most = fmaxf(most, s[e]);
        most = over_parts(most, [](float u, float v) { return fmaxf(u, v); });
        if (__any(most > shift + kSlack || (shift == -INFINITY && most > shift))) {
            const float now = fmaxf(shift, most);
            const float keep = shift == -INFINITY ? 0.0f : attention::exp2_fast(shift - now);
            total *= keep;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) acc[b] *= keep;
            shift = now;
        }
        const float base = shift == -INFINITY ? 0.0f : shift;
        if (v_scale > unit) {
            const float keep = unit / v_scale;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) acc[b] *= keep;
            unit = v_scale;
        }
        const float ratio = unit > 0.0f ? v_scale / unit : v_scale;
        f16x8 weights[2];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float w = attention::exp2_fast(s[e] - base);
            total += w;
            weights[e >> 3][e & 7] = (half_t)(w == 0.0f ? 0.0f : w * ratio);
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
            if (b < blocks) {
                acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_half(vr[b][0], vr[b][1]), weights[0], acc[b], 0, 0, 0);
                acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_half(vr[b][2], vr[b][3]), weights[1], acc[b], 0, 0, 0);
            }
    }
    total = over_parts(total, [](float u, float v) { return u + v; });

    // the waves' parts, joined
    if (part == 0) stats[0][wave][r] = shift;
    __syncthreads();
    float now = stats[0][0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) now = fmaxf(now, stats[0][w][r]);
    const float keep = shift == -INFINITY ? (total == total ? 0.0f : total) : attention::exp2_fast(shift - now);
    if (part == 0) stats[1][wave][r] = keep == 0.0f ? 0.0f : total * keep;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[wave][r][16 * b + 4 * part + e] = keep == 0.0f ? 0.0f : acc[b][e] * (keep * unit);
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * dim; i += kThreads) {
        const int rr = i / dim, d = i % dim;
        if (rr >= it.rows) break;
        const float l = (stats[1][0][rr] + stats[1][1][rr]) + (stats[1][2][rr] + stats[1][3][rr]);
        const float o = (sums[0][rr][d] + sums[1][rr][d]) + (sums[2][rr][d] + sums[3][rr][d]);
        const int rw = it.row0 + rr;
        const int64_t bird = it.at.row0 + rw / a.group;
        const int hd = it.head * a.group + rw % a.group;
        if (active == 1) {
            static_cast<T *>(a.out)[bird * a.out_stride + hd * dim + d] = static_cast<T>(l == 0.0f ? 0.0f : o / l);
        } else {
            const int64_t to = ((int64_t)split * a.tracks.total + bird) * a.q_heads + hd;
            a.part_out[to * dim + d] = o;
            if (d == 0) {
                float m = stats[0][0][rr];
                for (int w = 1; w < kWaves; ++w) m = fmaxf(m, stats[0][w][rr]);
                a.part_stat[2 * to] = m;
                a.part_stat[2 * to + 1] = l;
            }
        }
    }
}

// Rows whose pages several workgroups shared.
template <typename T>
__global__ void __launch_bounds__(kThreads) track_join_kernel(TrackAttentionArgs a) {
    const int64_t id = blockIdx.x;
    const Item it = item_of(a, id / a.cache.kv_heads, (int)(id % a.cache.kv_heads));
    if (!it.ok) return;
    const int active = (it.pages + a.split_pages - 1) / a.split_pages;
    if (active <= 1) return;
    const int dim = a.cache.dim;
    for (int i = threadIdx.x; i < it.rows * dim; i += kThreads) {
        const int rw = it.row0 + i / dim, d = i % dim;
        const int64_t bird = it.at.row0 + rw / a.group;
        const int hd = it.head * a.group + rw % a.group;
        const int64_t pitch = (int64_t)a.tracks.total * a.q_heads, at = bird * a.q_heads + hd;
        float m = -INFINITY;
        for (int s = 0; s < active; ++s) m = fmaxf(m, a.part_stat[2 * (s * pitch + at)]);
        float o = 0.0f, l = 0.0f;
        for (int s = 0; s < active; ++s) {
            const int64_t from = s * pitch + at;
            const float shift = a.part_stat[2 * from], total = a.part_stat[2 * from + 1];
            if (total == 0.0f) continue;
            const float keep = shift == -INFINITY ? total : attention::exp2_fast(shift - m);
            l += total * keep;
            o += a.part_out[from * dim + d] * keep;
        }
        static_cast<T *>(a.out)[bird * a.out_stride + hd * dim + d] = static_cast<T>(l == 0.0f ? 0.0f : o / l);
    }
}

template <typename T, int DI>
void launch_cap(const TrackAttentionArgs &a, dim3 grid, hipStream_t stream) {
    if (a.cap == 0.0f) hipLaunchKernelGGL((track_attention_kernel<T, DI, kNoCap>), grid, dim3(kThreads), 0, stream, a);
    else if (a.cap <= attention::kLowCap) hipLaunchKernelGGL((track_attention_kernel<T, DI, kLow>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((track_attention_kernel<T, DI, kHigh>), grid, dim3(kThreads), 0, stream, a);
}

template <typename T>
hipError_t launch_type(TrackAttentionArgs a, const TrackPlan &p, hipStream_t stream) {
    const int64_t items = p.slots * a.cache.kv_heads;
    if (a.cache.dim <= 64) launch_cap<T, 1>(a, dim3((uint32_t)(items * p.splits)), stream);
    else launch_cap<T, 2>(a, dim3((uint32_t)(items * p.splits)), stream);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || p.splits == 1) return err;
    hipLaunchKernelGGL((track_join_kernel<T>), dim3((uint32_t)items), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

TrackPlan plan_track_attention(int32_t n_tracks, int32_t total, int32_t max_pages, int32_t q_heads, int32_t kv_heads,
                               int n_cus) {
    TrackPlan p;
    const int group = q_heads / kv_heads;
    p.slots = (int64_t)total * group / kRows + n_tracks;
    const int64_t items = std::max<int64_t>(p.slots * kv_heads, 1);
    // enough workgroups for the card, of at least a page a wave
    int64_t splits = (8 * (int64_t)n_cus + items - 1) / items;
    splits = std::max<int64_t>(std::min<int64_t>(splits, (max_pages + kWaves - 1) / kWaves), 1);
    p.split_pages = (int32_t)((max_pages + splits - 1) / std::max<int64_t>(splits, 1));
    p.split_pages = std::max(p.split_pages, 1);
    p.splits = (int32_t)std::max<int64_t>((max_pages + p.split_pages - 1) / p.split_pages, 1);
    return p;
}

size_t track_attention_workspace_bytes(const TrackPlan &p, int32_t total, int32_t q_heads, int32_t dim) {
    return p.splits == 1 ? 0 : (size_t)p.splits * total * q_heads * (dim + 2) * sizeof(float);
}

hipError_t launch_track_attention(TrackAttentionArgs a, int32_t dtype, const TrackPlan &p, void *workspace,
                                  hipStream_t stream) {
    a.group = a.q_heads / a.cache.kv_heads;
    a.splits = p.splits;
    a.split_pages = p.split_pages;
    a.part_stat = static_cast<float *>(workspace);
    a.part_out = a.part_stat + (size_t)2 * p.splits * a.tracks.total * a.q_heads;
    if (a.cap >= attention::kLargestCap) a.cap = 0.0f;
    return dtype == FLOCK_F16 ? launch_type<half_t>(a, p, stream) : launch_type<bf16_t>(a, p, stream);
}

}  // namespace flock
