// attention_backward.hip - gradients of attention (the formulas stand in
// attention.hip): two kernels, each summing its own outputs in a fixed order,
// at the price of computing scores and dP twice, and P K beside dS K (eight
// products for five).

#include "attention_common.h"

namespace flock {
namespace {

using namespace attention;

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------

// dS and P as factors of float16 need a scale: dS is about |grad_out| / keys, below
// the type's normal numbers for ordinary gradients, and may pass its largest.  They
// are carried times 2^14, which holds P and dS to their last digit down to 2^-28, and
// each output's sum of dS has a power of two of its own, lowered as for a running
// maximum: what passes 2^15 is brought to 2^8 (gradients of 1e-4 over 2000 keys: error of
// dq 2.6e-2 -> 4.6e-3 of its norm, what rounding dq alone costs; a training step on
// tracks takes 4% longer for it).
template <typename T> constexpr bool kScaled = std::is_same_v<T, half_t>;
template <typename T> constexpr float kFactorBits = kScaled<T> ? 14.0f : 0.0f;
template <typename T> constexpr float kFactorScale = kScaled<T> ? 0x1p14f : 1.0f;
constexpr float kLargestFactor = 0x1p15f;
constexpr int kScaleTo = 8;

// The most of 16 factors, of both halves' lanes.
__device__ __forceinline__ float most_of(const f32x16 &s) {
    float most = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(s[r]));
    return across(most, [](float x, float y) { return fmaxf(x, y); });
}

// What brings `most` to 2^kScaleTo if it is too large, or 1.
__device__ __forceinline__ float scale_step(float most) {
    return most > kLargestFactor ? __builtin_ldexpf(1.0f, kScaleTo - __builtin_amdgcn_frexp_expf(most)) : 1.0f;
}

// Heads of 128 leave registers for half as many keys in flight.
template <int DP>
using DqTile = KeyTile<DP, DP <= 96 ? 64 : 32, Pitch<DP>::kBoth, Pitch<DP>::kRows, false>;

// Gradients of the queries: 128 rows a workgroup, 32 a wave, over the tiles of
// keys that they see.  Also delta = dout.out of every row, which the keys'
// gradients take from here, and each workgroup's share of its heads' slope
// gradients (zeros from one without rows, so that every share is written).
// Bound by vector instructions: 64 frames of 2000, 8 heads of 64 with distances
// 1550 us, 0.68 PFLOP/s of its four products (VALU 74% of the time, matrix cores
// 32%); 96 tracks in order 1611 us, 0.76 (56%, 38%: two waves a SIMD).
// dS is rounded to the operands' type as a factor of the product with K: that
// makes dq's error 2.4e-3 of its norm in bfloat16 where rounding dq alone costs
// 1.7e-3.
template <typename T, int DP, bool DIST, int CAP>
__global__ void __launch_bounds__(kThreads, (DP >= 96 && DIST) || (DP == 128 && CAP) ? 1 : 2) attention_dq_kernel(AttentionBackwardArgs b) {
    using F = typename Frag<T>::type;
    using Tile = DqTile<DP>;
    constexpr int kRows = 128, kKeys = DP <= 96 ? 64 : 32;
    const AttentionArgs &a = b.fwd;
    extern __shared__ char shared[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, col = lane & 31;
    const int64_t id = xcd_order(blockIdx.x, gridDim.x);
    const int head = (int)(id / a.slots);
    int64_t tile;
    const int f = find_frame(a.q_offsets, a.n_frames, a.group, kRows, id % a.slots, &tile);
    const Span sp = frame_span(a, f);
    const int n_rows = sp.ok ? sp.nq * a.group : 0;
    float *const shares = DIST && b.slope_shares ? b.slope_shares + id % a.slots * a.q_heads + head * a.group : nullptr;
    if (tile < 0 || tile * kRows >= n_rows) {
        if (shares)
            for (int g = threadIdx.x; g < a.group; g += kThreads) shares[g] = 0.0f;
        return;
    }
    const int row0 = (int)tile * kRows;
    const RowRun run(a, row0);
    const bool valid = row0 + 32 * wave + col < n_rows;
    int qi = 0, g = 0;
    if (valid) run.find(a, 32 * wave + col, qi, g);
    const int qh = head * a.group + g;
    const int64_t qrow = sp.q0 + qi;
    const short *q_row = valid ? static_cast<const short *>(a.q) + qrow * a.q_stride + qh * a.dim : nullptr;
    const short *g_row = valid ? static_cast<const short *>(b.grad_out) + qrow * b.grad_out_stride + qh * a.dim : nullptr;
    const short *o_row = valid ? static_cast<const short *>(a.out) + qrow * a.out_stride + qh * a.dim : nullptr;
    F q[DP / 16], go[DP / 16];
    float delta = 0.0f;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        q[s] = load_frag<T>(q_row, s, h, a.dim);
        go[s] = load_frag<T>(g_row, s, h, a.dim);
        const F o = load_frag<T>(o_row, s, h, a.dim);
#pragma unroll
        for (int e = 0; e < 8; ++e) delta = __builtin_fmaf(static_cast<float>(go[s][e]), static_cast<float>(o[e]), delta);
    }
    delta = across(delta, [](float x, float y) { return x + y; });
    const int prefix = a.causal && a.prefix ? min(max(a.prefix[f], 0), sp.nk) : 0;
    const int limit = valid ? seen_limit(a, sp, prefix, qi) : sp.nk;
    float qx = 0.0f, qy = 0.0f, slope2 = 0.0f;
    if (DIST && valid) {
        const int2 place = reinterpret_cast<const int2 *>(a.q_xy)[qrow];
        qx = (float)place.x * kPxPerQuantum;
        qy = (float)place.y * kPxPerQuantum;
        slope2 = a.slopes[qh] * kLog2e;
    }
    const float scale = score_scale<CAP>(a), cap2 = a.cap * kLog2e;
    float shift, rest;
    split_lse(valid ? a.lse[qrow * a.q_heads + qh] : -INFINITY, shift, rest);
    // (dS carries its scale from here, and so do its sums)
    float ds_scale = kFactorScale<T>;
    int wave_end = sp.nk, wave_all = sp.nk, end = sp.nk;
    if (a.causal) {
        wave_end = wave_max(limit);
        wave_all = -wave_max(-limit);
        end = seen_limit(a, sp, prefix, run.query(a, min(kRows, n_rows - row0) - 1));
    }

    // delta comes from the rounded output, and where the weights are sharp, dP - delta
    // is small for the keys that have them: with scores eight times normal ones dq's
    // error is 5.0e-3 of its norm in bfloat16, and 2.4e-3 with the right delta.  The sum
    // of dS, which should be zero, is what delta is off by: the keys' gradients take
    // the right one, and dq gets that much of P K taken off.  P K is summed on the way,
    // beside dq (training steps 2 to 8%), but for wide heads that it would leave one wave
    // a SIMD (without distances or caps; heads of 128: 1.47 -> 2.03 ms).  Their keys are
    // gone over again, in workgroups that have a row where it matters: delta's error
    // above a quarter of a factor's rounding (1.49 ms where none has).
    constexpr bool SUMMED = DP <= 64 || DIST || (DP == 128 && CAP);
    constexpr float kTolerated = kScaled<T> ? 0x1p-13f : 0x1p-10f;
    f32x16 dq[DP / 32] = {}, pk[SUMMED ? DP / 32 : 1] = {};
    float off = 0.0f;  // what delta is off by, times rest
    // sums of P, dS, its size, P d2 and dS d2.  P sums to one but for the rounding of
    // lse; the slope's gradient is rid of that and of delta's error.
    float sum_p = 0.0f, sum_ds = 0.0f, size_ds = 0.0f, sum_p_d2 = 0.0f, sum_ds_d2 = 0.0f;
    // (AGAIN: the keys once more, for P K alone)
    auto sub_tile = [&](auto again, const typename Tile::Lds &t, int kt, int first, bool hidden, bool limited) {
        constexpr bool AGAIN = decltype(again)::value;
        const float rest_scale = rest * ds_scale, rest_delta = delta * rest_scale;
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int st = 0; st < DP / 16; ++st) {
            s = mfma(read_rows<T, Pitch<DP>::kBoth>(t.k, first + col, st, h), q[st], s);
            if (!AGAIN) dp = mfma(read_rows<T, Pitch<DP>::kRows>(t.v, first + col, st, h), go[st], dp);
        }
        if (CAP) cap_parts<CAP>(s, scale);
        float d2[DIST ? 16 : 1], of_cap[CAP ? 16 : 1];
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            float kx[4], ky[4];
            if (DIST) {
                *reinterpret_cast<float4 *>(kx) = read4(t.x, first, r, h);
                *reinterpret_cast<float4 *>(ky) = read4(t.y, first, r, h);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (DIST) d2[r + e] = distance2(qx - kx[e], qy - ky[e]);
                if (CAP) of_cap[r + e] = s[r + e];
                s[r + e] = score<DIST, CAP>(s[r + e], scale, cap2, DIST ? d2[r + e] : 0.0f, slope2);
            }
        }
        if (hidden) {
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const float4 pen = read4(t.penalty, first, r, h);
                s[r] += pen.x;
                s[r + 1] += pen.y;
                s[r + 2] += pen.z;
                s[r + 3] += pen.w;
            }
        }
        if (limited) {
            const uint32_t seen = seen_bits(0xffffffffu, limit, kt + first, h);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = (seen >> out_row(r, 0)) & 1 ? s[r] : -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float p = exp2_fast(s[r] - shift);  // P / rest; rest is in the other factors
            const float slope = CAP ? cap_slope<CAP>(of_cap[r]) : 1.0f;
            if (AGAIN) {
                s[r] = -off * (CAP ? p * slope : p);
                continue;
            }
            const float ds = p * __builtin_fmaf(dp[r], rest_scale, -rest_delta);
            sum_ds += ds;
            if (!SUMMED) size_ds += fabsf(ds);
            if (DIST) {
                sum_p += p;
                sum_p_d2 = __builtin_fmaf(p, d2[r], sum_p_d2);
                sum_ds_d2 = __builtin_fmaf(ds, d2[r], sum_ds_d2);
            }
            s[r] = CAP ? ds * slope : ds;
            if (SUMMED) dp[r] = CAP ? p * slope : p;
        }
        if (kScaled<T> && !AGAIN) {
            const float most = most_of(s);
            if (__any(most > kLargestFactor)) {
                const float step = scale_step(most);
                ds_scale *= step;
                sum_ds *= step;
                size_ds *= step;
                sum_ds_d2 *= step;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] *= step;
#pragma unroll
                for (int blk = 0; blk < DP / 32; ++blk)
#pragma unroll
                    for (int r = 0; r < 16; ++r) dq[blk][r] *= step;
            }
        }
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const F d = round_frag<T>(s, part);
            F p;
            if (SUMMED) p = round_frag<T>(dp, part);
#pragma unroll
            for (int blk = 0; blk < DP / 32; ++blk) {
                const F k = read_columns<T, Pitch<DP>::kBoth>(t.k, first + 16 * part, blk, lane);
                dq[blk] = mfma(k, d, dq[blk]);
                if (SUMMED) pk[blk] = mfma(k, p, pk[blk]);
            }
        }
    };

    auto over_keys = [&](auto again) {
        Tile next(a);
        if (end > 0) {
            next.look_up(a, sp, 0, end);
            next.template load<DIST>(a, sp, head, 0, end);
            next.look_up(a, sp, kKeys, end);
            next.template store<DIST>(a, typename Tile::Lds(shared));
        }
        wait_for_loads();
        __syncthreads();
        int buffer = 0;
        for (int kt = 0; kt < end; kt += kKeys) {
            const bool more = kt + kKeys < end;
            if (more) {
                next.template load<DIST>(a, sp, head, kt + kKeys, end);
                next.look_up(a, sp, kt + 2 * kKeys, end);
            }
            const typename Tile::Lds t(shared + buffer * Tile::kBytes);
            const uint64_t seen = *t.seen;
            if (kt < wave_end) {
#pragma unroll(DP <= 64 ? 2 : 1)
                for (int sub = 0; sub < kKeys / 32; ++sub) {
                    const uint32_t bits = __builtin_amdgcn_readfirstlane((uint32_t)(seen >> (32 * sub)));
                    if (bits != 0) sub_tile(again, t, kt, 32 * sub, bits != 0xffffffffu, kt + 32 * sub + 32 > wave_all);
                }
            }
            buffer ^= 1;
            if (more) next.template store<DIST>(a, typename Tile::Lds(shared + buffer * Tile::kBytes));
            __syncthreads();
        }
    };
    over_keys(std::false_type{});
    const float unscale = 1.0f / ds_scale;  // (a power of two)
    auto add = [](float x, float y) { return x + y; };
    sum_ds = across(sum_ds, add) * unscale;
    off = sum_ds * rest;
    if (DIST) {
        sum_p = across(sum_p, add);
        sum_p_d2 = across(sum_p_d2, add);
        sum_ds_d2 = across(sum_ds_d2, add) * unscale;
        float share = 0.0f;
        if (sum_p > 0.0f) {
            off = sum_ds / sum_p;
            share = (off * sum_p_d2 - sum_ds_d2) / (sum_p * rest);
        }
        if (shares) {
            // the tiles in LDS are done with; rows of a head are added in their order
            float *const rows = reinterpret_cast<float *>(shared);
            if (h == 0) rows[32 * wave + col] = valid ? share : 0.0f;
            __syncthreads();
            for (int g = threadIdx.x; g < a.group; g += kThreads) {
                float sum = 0.0f;
                for (int r = g >= run.first_g ? g - run.first_g : g - run.first_g + a.group; r < kRows; r += a.group)
                    sum += rows[r];
                shares[g] = sum;
            }
            __syncthreads();
        }
    }
    if (valid && h == 0) b.delta[qrow * a.q_heads + qh] = rest > 0.0f ? delta + off / rest : delta;
    if (!SUMMED) {
        size_ds = across(size_ds, add) * unscale;
        if (__syncthreads_or(fabsf(sum_ds) > kTolerated * size_ds)) {
            off *= ds_scale;
            if (kScaled<T>) {
                const float step = scale_step(fabsf(off));
                off *= step;
                ds_scale *= step;
#pragma unroll
                for (int blk = 0; blk < DP / 32; ++blk)
#pragma unroll
                    for (int r = 0; r < 16; ++r) dq[blk][r] *= step;
            }
            over_keys(std::true_type{});
        }
    }
    if (!valid) return;
    T *out = static_cast<T *>(b.grad_q) + qrow * b.grad_q_stride + qh * a.dim;
    const float out_scale = a.scale / ds_scale, off_scale = a.scale * off;
#pragma unroll
    for (int blk = 0; blk < DP / 32; ++blk)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * blk + out_row(r, h);
            if (d < a.dim) {
                float z[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z[e] = dq[blk][r + e] * out_scale;
                    if (SUMMED) z[e] -= pk[blk][r + e] * off_scale;
                }
                store_pack<T, 4>(out + d, z);
            }
        }
}

// A tile of 64 rows (queries of the heads that share a kv head), their output
// gradients and what their scores need, on its way to LDS as KeyTile is.
constexpr int kTileRows = 64;

template <typename T, int DP, bool NEAR>
struct RowTile {
    static constexpr int kChunks = DP / 8;
    static constexpr int kLoads = kTileRows * kChunks / kThreads;
    static constexpr int kPitch = Pitch<DP>::kBoth;
    static constexpr int kRowChunks = kTileRows * kPitch;
    static constexpr int kBytes = 2 * kRowChunks * 16 + (NEAR ? 2 * kTileRows * 16 : 0) + 8 * kTileRows * 4 + 16;

    struct Lds {
        i16x8 *q, *g, *near;  // near: [half][row]
        float *x, *y, *slope, *shift, *near_shift, *delta, *rest;
        int *limit, *exact, *all_near;
        __device__ __forceinline__ explicit Lds(char *base) {
            q = reinterpret_cast<i16x8 *>(base);
            g = q + kRowChunks;
            near = g + kRowChunks;
            x = reinterpret_cast<float *>(near + (NEAR ? 2 * kTileRows : 0));
            y = x + kTileRows;
            slope = y + kTileRows;
            shift = slope + kTileRows;
            near_shift = shift + kTileRows;
            delta = near_shift + kTileRows;
            rest = delta + kTileRows;
            limit = reinterpret_cast<int *>(rest + kTileRows);
            exact = limit + kTileRows;
            all_near = exact + 1;
        }
    };

    i32x4 q[kLoads], g[kLoads];
    // as loaded: what is made of them waits for the loads, so it is made in store()
    double lse;
    int2 place;
    float slope, delta;
    int limit;

    template <bool DIST>
    __device__ __forceinline__ void load(const AttentionBackwardArgs &b, const Span &sp, int head, int prefix,
                                         const RowRun &run, int rows) {
        const AttentionArgs &a = b.fwd;
        const int64_t first = sp.q0 + run.first_query;
        const int q_step = (int)a.q_stride * 2, g_step = (int)b.grad_out_stride * 2;
        // absent rows and dimensions go beyond the resource, everything else is within the tile
        const auto qr = tile_resource(a.q, first * a.q_stride + head * a.group * a.dim, kBeyond);
        const auto gr = tile_resource(b.grad_out, first * b.grad_out_stride + head * a.group * a.dim, kBeyond);
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int e = threadIdx.x + n * kThreads;
            const int r = e / kChunks, c = e % kChunks;
            const uint32_t u = run.first_g + r, i = group_quotient(u, a.group_reciprocal);
            const int at = (int)__umul24(u - __umul24(i, a.group), a.dim * 2) + c * 16;
            const bool in = c * 8 < a.dim && r < rows;
            const int q_at = (int)i * q_step + at, g_at = (int)i * g_step + at;
            q[n] = __builtin_amdgcn_raw_buffer_load_b128(qr, in ? q_at : kBeyond, 0, 0);
            g[n] = __builtin_amdgcn_raw_buffer_load_b128(gr, in ? g_at : kBeyond, 0, 0);
        }
        if (threadIdx.x < kTileRows) {
            // absent rows read the last one's values and have no weights
            int i, gg;
            run.find(a, min((int)threadIdx.x, rows - 1), i, gg);
            const int qh = head * a.group + gg;
            const int64_t row = sp.q0 + i;
            lse = a.lse[row * a.q_heads + qh];
            delta = b.delta[row * a.q_heads + qh];
            if (DIST) {
                place = reinterpret_cast<const int2 *>(a.q_xy)[row];
                slope = a.slopes[qh];
            }
            limit = seen_limit(a, sp, prefix, i);
            if ((int)threadIdx.x >= rows) limit = -1;
        }
    }

    // units: of the products, to which the distances are added
    template <bool DIST>
    __device__ __forceinline__ void store(const Lds &lds, int2 origin, float largest, float units, float constant) const {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int e = threadIdx.x + n * kThreads;
            const int at = e / kChunks * kPitch + e % kChunks;
            lds.q[at] = __builtin_bit_cast(i16x8, q[n]);
            lds.g[at] = __builtin_bit_cast(i16x8, g[n]);
        }
        if (threadIdx.x < kTileRows) {  // the first wave
            const bool absent = limit < 0;
            if (DIST) {
                lds.x[threadIdx.x] = (float)place.x * kPxPerQuantum;
                lds.y[threadIdx.x] = (float)place.y * kPxPerQuantum;
                lds.slope[threadIdx.x] = slope * kLog2e;
            }
            float shift, rest;
            split_lse(absent ? -INFINITY : lse, shift, rest);
            shift -= kFactorBits<T>;  // the weights' scale
            lds.shift[threadIdx.x] = shift;
            if (NEAR) {
                // the row's term of the distances goes with the shift
                const int ax = place.x - origin.x, ay = place.y - origin.y;
                const float n = square_quanta(ax, ay), weight = slope * kLog2e / 256.0f;
                const NearSlots s = near_row(ax, ay, weight * units);
                lds.near[threadIdx.x] = s.half[0];
                lds.near[kTileRows + threadIdx.x] = s.half[1];
                lds.near_shift[threadIdx.x] = __builtin_fmaf(weight, n, shift - constant);
                const bool all = __all(near_enough(ax, ay, n, largest));
                if (threadIdx.x == 0) *lds.all_near = all;
            }
            lds.delta[threadIdx.x] = delta;
            lds.rest[threadIdx.x] = rest;
            lds.limit[threadIdx.x] = limit;
            // rest is 1 to a rounding of the weights, but for large scores (rows without keys have P = 0)
            const bool one = __all(fabsf(rest - 1.0f) < 0x1p-16f || shift == INFINITY);
            if (threadIdx.x == 0) *lds.exact = one ? 1 : 0;
        }
    }
};

// Gradients of keys and values: 32 keys a wave, over the rows that see them.  The
// products are S = Q K^T and dP = dO V^T here, so that a lane holds one key.  64 keys
// a wave would halve what is read of LDS for each, but leave one wave a SIMD (4.37 ms
// against 3.67 for a training step on 64 frames of 2000, 8 heads of 64 with
// distances).  Same frames, 1451 us, 0.72 PFLOP/s of four products (VALU 42%, matrix
// cores 35%, LDS 40% of the time, a fifth of that bank conflicts of rows that are
// read both ways); the phases of the two waves a SIMD overlap only in part.
template <typename T, int DP, bool DIST, int CAP>
__global__ void __launch_bounds__(kThreads, DP <= 64 ? 2 : 1) attention_dkv_kernel(AttentionBackwardArgs b) {
    using F = typename Frag<T>::type;
    using Tile = RowTile<T, DP, DIST>;
    constexpr int kKeys = 128;
    const AttentionArgs &a = b.fwd;
    extern __shared__ char shared[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, col = lane & 31;
    const int64_t id = xcd_order(blockIdx.x, gridDim.x);
    const int head = (int)(id / b.key_slots);
    int64_t tile;
    const int f = find_frame(a.k_offsets, a.n_frames, 1, kKeys, id % b.key_slots, &tile);
    const Span sp = frame_span(a, f);
    if (!sp.ok || tile < 0) return;
    const int64_t key0 = tile * kKeys;
    if (key0 >= sp.nk) return;
    const int n_rows = sp.nq * a.group;
    F k[DP / 16], v[DP / 16];
    const int wave_key = (int)key0 + 32 * wave;  // the wave's first key
    const int key = wave_key + col;
    const bool valid = key < sp.nk;
    const int64_t krow = sp.k0 + (valid ? key : 0);
    const bool kept = valid && (!a.keep || a.keep[krow]);
    const short *k_row = kept ? static_cast<const short *>(a.k) + krow * a.k_stride + head * a.dim : nullptr;
    const short *v_row = kept ? static_cast<const short *>(a.v) + krow * a.v_stride + head * a.dim : nullptr;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        k[s] = load_frag<T>(k_row, s, h, a.dim);
        v[s] = load_frag<T>(v_row, s, h, a.dim);
    }
    float kx = 0.0f, ky = 0.0f;
    if (DIST && valid) {
        const int2 place = reinterpret_cast<const int2 *>(a.k_xy)[krow];
        kx = (float)place.x * kPxPerQuantum;
        ky = (float)place.y * kPxPerQuantum;
    }
    const float scale = score_scale<CAP>(a), cap2 = a.cap * kLog2e;
    float largest = 0.0f;
    int2 origin = make_int2(0, 0);
    bool keys_near = false;
    bf16x8 key_slots = {};
    if (DIST) {
        origin = near_origin(reinterpret_cast<const int2 *>(a.k_xy)[sp.k0 + min((int)key0 + col, sp.nk - 1)]);
        largest = near_largest<T, CAP>(a, head, scale);
        const int bx = (int)(kx * 16.0f) - origin.x, by = (int)(ky * 16.0f) - origin.y;
        const float n2 = square_quanta(bx, by);
        const NearSlots s = near_key(bx, by, n2);
        key_slots = __builtin_bit_cast(bf16x8, h ? s.half[1] : s.half[0]);
        keys_near = __all(!valid || near_enough(bx, by, n2, largest));
    }
    const int prefix = a.causal && a.prefix ? min(max(a.prefix[f], 0), sp.nk) : 0;
    // the first query that sees the workgroup's first key
    int begin = 0;
    if (a.causal && key0 >= prefix)
        begin = (int)(max((int64_t)0, key0 - sp.nk + sp.nq) * a.group / kTileRows * kTileRows);

    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    float ds_scale = 1.0f;  // beside that of the weights
    bool lowered = false;   // any lane's
    auto sub_tile = [&](const typename Tile::Lds &t, int first, bool limited, bool exact, bool near) {
        F qf[DP / 16], gf[DP / 16];
#pragma unroll
        for (int st = 0; st < DP / 16; ++st) {
            qf[st] = read_rows<T, Tile::kPitch>(t.q, first + col, st, h);
            gf[st] = read_rows<T, Tile::kPitch>(t.g, first + col, st, h);
        }
        // the columns are read here where registers allow it, to be there when the weights are
        // (halves of the 32 rows; with distances a fourth of them more would spill)
        constexpr int G_EARLY = DP <= 64 && !(DIST && (CAP || kScaled<T>)) ? 2 : 0;
        constexpr int Q_EARLY = DIST && G_EARLY ? 1 : G_EARLY;
        F gc[2][DP / 32], qc[2][DP / 32];
        auto columns = [&](int part, int blk, bool g, bool q) {
            if (g) gc[part][blk] = read_columns<T, Tile::kPitch>(t.g, first + 16 * part, blk, lane);
            if (q) qc[part][blk] = read_columns<T, Tile::kPitch>(t.q, first + 16 * part, blk, lane);
        };
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int blk = 0; blk < DP / 32; ++blk) columns(part, blk, part < G_EARLY, part < Q_EARLY);
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int st = 0; st < DP / 16; ++st) {
            s = mfma(qf[st], k[st], s);
            dp = mfma(gf[st], v[st], dp);
        }
        if (CAP) cap_parts<CAP>(s, scale);
        if (near) {
            const bf16x8 row = __builtin_bit_cast(bf16x8, t.near[h * kTileRows + first + col]);
            f32x16 bias;
            if (CAP) bias = mfma(row, key_slots, f32x16{});
            else s = mfma(row, key_slots, s);
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                float shift[4], delta[4];
                *reinterpret_cast<float4 *>(shift) = read4(t.near_shift, first, r, h);
                *reinterpret_cast<float4 *>(delta) = read4(t.delta, first, r, h);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float d = dp[r + e] - delta[e];
                    if (CAP) {
                        d *= cap_slope<CAP>(s[r + e]);
                        s[r + e] = exp2_fast(capped<CAP>(s[r + e], cap2, bias[r + e]) - shift[e]);
                    } else {
                        s[r + e] = exp2_fast(__builtin_fmaf(s[r + e], scale, -shift[e]));
                    }
                    dp[r + e] = s[r + e] * d;
                }
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                float x[4], y[4], slope[4] = {}, shift[4], delta[4];
                if (DIST) {
                    *reinterpret_cast<float4 *>(x) = read4(t.x, first, r, h);
                    *reinterpret_cast<float4 *>(y) = read4(t.y, first, r, h);
                    *reinterpret_cast<float4 *>(slope) = read4(t.slope, first, r, h);
                }
                *reinterpret_cast<float4 *>(shift) = read4(t.shift, first, r, h);
                *reinterpret_cast<float4 *>(delta) = read4(t.delta, first, r, h);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float d2 = DIST ? distance2(x[e] - kx, y[e] - ky) : 0.0f;
                    const float z = score<DIST, CAP>(s[r + e], scale, cap2, d2, slope[e]);
                    const float p = exp2_fast(z - shift[e]);
                    float d = p * (dp[r + e] - delta[e]);
                    if (CAP) d *= cap_slope<CAP>(s[r + e]);
                    s[r + e] = p;
                    dp[r + e] = d;
                }
            }
        }
        if (limited) {
            const int key = wave_key + col;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (key >= t.limit[first + out_row(r, h)]) s[r] = dp[r] = 0.0f;
        }
        if (!exact) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float rest = t.rest[first + out_row(r, h)];
                s[r] *= rest;
                dp[r] *= rest;
            }
        }
        if (kScaled<T>) {
            if (lowered) {
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] *= ds_scale;
            }
            const float most = most_of(dp);
            if (__any(most > kLargestFactor)) {
                lowered = true;
                const float step = scale_step(most);
                ds_scale *= step;
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] *= step;
#pragma unroll
                for (int blk = 0; blk < DP / 32; ++blk)
#pragma unroll
                    for (int r = 0; r < 16; ++r) dk[blk][r] *= step;
            }
        }
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const F p = round_frag<T>(s, part), ds = round_frag<T>(dp, part);
#pragma unroll
            for (int blk = 0; blk < DP / 32; ++blk) {
                columns(part, blk, part >= G_EARLY, part >= Q_EARLY);
                dv[blk] = mfma(gc[part][blk], p, dv[blk]);
                dk[blk] = mfma(qc[part][blk], ds, dk[blk]);
            }
        }
    };

    const float units = CAP ? 1.0f : 1.0f / scale, constant = CAP ? cap_constant<CAP>(cap2) : 0.0f;
    Tile next;
    RowRun run(a, begin);
    if (begin < n_rows) {
        next.template load<DIST>(b, sp, head, prefix, run, min(kTileRows, n_rows - begin));
        next.template store<DIST>(typename Tile::Lds(shared), origin, largest, units, constant);
    }
    wait_for_loads();
    __syncthreads();
    int buffer = 0;
    for (int rt = begin; rt < n_rows; rt += kTileRows) {
        const bool more = rt + kTileRows < n_rows;
        run.advance(a, kTileRows);
        if (more) next.template load<DIST>(b, sp, head, prefix, run, min(kTileRows, n_rows - rt - kTileRows));
        const typename Tile::Lds t(shared + buffer * Tile::kBytes);
        const bool exact = __builtin_amdgcn_readfirstlane(*t.exact) != 0;
        const bool near = DIST && keys_near && __builtin_amdgcn_readfirstlane(*t.all_near) != 0;
        // limits grow with the rows: those of the first and of the last row say which keys all and some rows see
        const int some = a.causal ? __builtin_amdgcn_readfirstlane(t.limit[min(kTileRows, n_rows - rt) - 1]) : sp.nk;
        const int all = a.causal ? __builtin_amdgcn_readfirstlane(t.limit[0]) : sp.nk;
        if (wave_key < some) {
#pragma unroll 1
            for (int sub = 0; sub < kTileRows / 32; ++sub)
                sub_tile(t, 32 * sub, min(wave_key + 32, sp.nk) > all, exact, near);
        }
        buffer ^= 1;
        if (more) next.template store<DIST>(typename Tile::Lds(shared + buffer * Tile::kBytes), origin, largest, units, constant);
        __syncthreads();
    }
    if (wave_key + col >= sp.nk) return;
    const int64_t row = sp.k0 + wave_key + col;
    T *dk_out = static_cast<T *>(b.grad_k) + row * b.grad_k_stride + head * a.dim;
    T *dv_out = static_cast<T *>(b.grad_v) + row * b.grad_v_stride + head * a.dim;
    constexpr float kUnscale = 1.0f / kFactorScale<T>;
    const float dk_scale = a.scale * kUnscale / ds_scale;
#pragma unroll
    for (int blk = 0; blk < DP / 32; ++blk)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * blk + out_row(r, h);
            if (d < a.dim) {
                // a hidden key's scores are not masked above: its gradients are zero
                float x[4], y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = kept ? dk[blk][r + e] * dk_scale : 0.0f;
                    y[e] = kept ? dv[blk][r + e] * kUnscale : 0.0f;
                }
                store_pack<T, 4>(dk_out + d, x);
                store_pack<T, 4>(dv_out + d, y);
            }
        }
}

// Gradient of a head's slope: the workgroups' shares, in 64 bits and a fixed
// order, a block a head.
__global__ void __launch_bounds__(1024) slope_total_kernel(const float *shares, int64_t n, int q_heads,
                                                           float *grad_slopes) {
    __shared__ double sums[1024];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) s += shares[i * q_heads + blockIdx.x];
    sums[threadIdx.x] = s;
    for (int d = 512; d > 0; d >>= 1) {
        __syncthreads();
        if (threadIdx.x < d) sums[threadIdx.x] += sums[threadIdx.x + d];
    }
    if (threadIdx.x == 0) grad_slopes[blockIdx.x] = (float)sums[0];
}

// Numbers of row tiles of the queries' gradients, of key tiles of the keys'.
int64_t backward_slots(int32_t n_frames, int32_t total_q, int group) { return (int64_t)total_q * group / 128 + n_frames; }
int64_t backward_key_slots(int32_t n_frames, int32_t total_k) { return (int64_t)total_k / 128 + n_frames; }

}  // namespace

int64_t attention_backward_workgroups(int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads, int32_t kv_heads) {
    return std::max(backward_slots(n_frames, total_q, q_heads / kv_heads), backward_key_slots(n_frames, total_k)) * kv_heads;
}

size_t attention_backward_workspace_bytes(int32_t n_frames, int32_t total_q, int32_t q_heads, int32_t kv_heads) {
    if (n_frames <= 0 || total_q < 0 || q_heads <= 0 || kv_heads <= 0) return 0;
    const size_t slots = (size_t)backward_slots(n_frames, total_q, q_heads / kv_heads);
    return align256((size_t)total_q * (size_t)q_heads * sizeof(float)) + align256(slots * (size_t)q_heads * sizeof(float));
}

hipError_t launch_attention_backward(AttentionBackwardArgs b, int32_t dtype, void *workspace, float *grad_slopes,
                                     hipStream_t stream) {
    AttentionArgs &a = b.fwd;
    b.delta = static_cast<float *>(workspace);
    b.slope_shares = nullptr;
    if (grad_slopes)
        b.slope_shares = reinterpret_cast<float *>(static_cast<char *>(workspace) +
                                                   align256((size_t)a.total_q * (size_t)a.q_heads * sizeof(float)));
    a.slots = backward_slots(a.n_frames, a.total_q, a.group);
    a.group_reciprocal = group_reciprocal(a.group);
    hipError_t err = a.n_frames == 0 ? hipSuccess : with_kernel(a, dtype, [&](auto t, auto dp, auto dist, auto cap) {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool DIST = decltype(dist)::value;
        constexpr int CAP = decltype(cap)::value;
        hipError_t e = hipSuccess;
        if (a.total_q > 0) {
            constexpr size_t bytes = 2 * DqTile<DP>::kBytes;
            auto kernel = attention_dq_kernel<T, DP, DIST, CAP>;
            hipLaunchKernelGGL(kernel, dim3((uint32_t)(a.slots * a.kv_heads)), dim3(kThreads), bytes, stream, b);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (a.total_k > 0) {
            constexpr size_t bytes = 2 * RowTile<T, DP, DIST>::kBytes;
            b.key_slots = backward_key_slots(a.n_frames, a.total_k);
            auto kernel = attention_dkv_kernel<T, DP, DIST, CAP>;
            hipLaunchKernelGGL(kernel, dim3((uint32_t)(b.key_slots * a.kv_heads)), dim3(kThreads), bytes, stream, b);
            e = hipGetLastError();
        }
        return e;
    });
    if (err != hipSuccess || !grad_slopes) return err;
    // without frames or queries there are no shares, and the gradients are zeros
    hipLaunchKernelGGL(slope_total_kernel, dim3(a.q_heads), dim3(1024), 0, stream, b.slope_shares,
                       a.n_frames > 0 && a.total_q > 0 ? a.slots : 0, a.q_heads, grad_slopes);
    return hipGetLastError();
}

}  // namespace flock
