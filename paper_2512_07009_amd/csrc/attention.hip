// attention.hip - attention of the birds of a frame (or of a track) among
// themselves, or of a few queries over them.
//
// For query i and key j of a frame, head h, d2 their squared distance in px^2:
//   t = scale q_i.k_j, capped: t = cap tanh(t / cap);   s = t - slope_h d2
//   key j is seen by query i: keep[j], and in ordered frames j < limit_i with
//   limit_i = max(prefix, i + n_k - n_q + 1)
//   out_i = sum_j softmax_j(s) v_j over the keys seen, 0 where there are none
//   backward: P = exp(s - lse), delta_i = dout_i.out_i, dP = dout_i.v_j
//   dS = P (dP - delta), dT = dS (1 - (t / cap)^2)
//   dq = scale dT k, dk = scale dT^T q, dv = P^T dout, dslope_h = -sum dS d2
// (out is rounded, and with it delta; what that leaves in sum_j dS is taken off)
//
// Queries of the heads that share a kv head are packed as rows r = (i, g) of
// one problem per frame and kv head, so that shared keys are read once and
// their gradients are summed where they are computed.  Every product runs on
// the matrix cores (32 x 32 x 16, 16-bit factors, 32-bit sums); the softmax, its
// statistics and dS are in 32 bits, and P and dS are rounded to the operands'
// type only as factors of the next product.
//
// Scores are computed transposed, S^T = K Q^T: a lane then holds scores of one
// query, in the order in which the next product wants them as its right
// factor, so that they never leave the registers.  The left factor's rows
// follow the same order of keys: lane half h holds keys 4h .. 4h + 3 and
// 8 + 4h .. 8 + 4h + 3 of each 16, which the transposing LDS read returns for
// 16 columns a group of lanes.

#include "attention_common.h"

namespace flock {
namespace {

using namespace attention;

// ---------------------------------------------------------------------------
// Forward, many rows: 128 rows a workgroup, 32 a wave, all waves over the same
// tiles of keys.  A tile's loads are in flight while the tile before is worked
// on, between two LDS buffers with one barrier a tile.
//
// Bound by vector instructions, not by the matrix cores: of 32 x 32 scores with
// heads of 64 the products take 8 x 32 cycles, the softmax at least 320 (a multiply
// and add, half a maximum, an exponential at half the rate, a sum and half a rounding
// to 16 bits each), and distances, caps and masks add to that.  8 heads of 64: 96
// tracks in order 875 us, 0.70 PFLOP/s (VALU 69% of the time, matrix cores 38%); 64
// frames of 2000 with distances and lse 999 us, 0.52 (91%, 23%), with distances and
// cap 1065 us, 0.49 (84%, 24%).  24 frames of 8000, 8 heads of 128 over 2: 8.9 ms, 0.71
// PFLOP/s (50%, 32%); registers leave two waves a SIMD there, which do not cover
// each other's waits, and a third would spill.
// ---------------------------------------------------------------------------

// Scores above the shift by less than this are left there (their weights reach
// 2^8, well within 32 bits and float16), so that sums and outputs are rescaled
// only now and then.
constexpr float kSlack = 8.0f;

template <int DP, bool DIST>
using RowsTile = KeyTile<DP, kTileKeys, Pitch<DP>::kRows, Pitch<DP>::kColumns, DIST>;

template <typename T, int DP, bool DIST, int CAP>
__global__ void __launch_bounds__(kThreads, DP <= 64 ? 3 : 2) attention_rows_kernel(AttentionArgs a) {
    using F = typename Frag<T>::type;
    using Tile = RowsTile<DP, DIST>;
    constexpr int kRows = 128;
    extern __shared__ char shared[];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, col = lane & 31;
    const int64_t id = xcd_order(blockIdx.x, gridDim.x);
    const int head = (int)(id / a.slots);
    int64_t tile;
    const int f = find_frame(a.q_offsets, a.n_frames, a.group, kRows, id % a.slots, &tile);
    const Span sp = frame_span(a, f);
    if (!sp.ok || tile < 0) return;
    const int n_rows = sp.nq * a.group;
    if (tile * kRows >= n_rows) return;
    const int row0 = (int)tile * kRows;
    const RowRun run(a, row0);

    // this lane's query
    const bool valid = row0 + 32 * wave + col < n_rows;
    int qi = 0, g = 0;
    if (valid) run.find(a, 32 * wave + col, qi, g);
    const int qh = head * a.group + g;
    const short *q_row = valid ? static_cast<const short *>(a.q) + (int64_t)(sp.q0 + qi) * a.q_stride + qh * a.dim
                               : nullptr;
    F q[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) q[s] = load_frag<T>(q_row, s, h, a.dim);
    const int prefix = a.causal && a.prefix ? min(max(a.prefix[f], 0), sp.nk) : 0;
    const int limit = valid ? seen_limit(a, sp, prefix, qi) : sp.nk;
    float qx = 0.0f, qy = 0.0f, slope2 = 0.0f;
    if (DIST && valid) {
        const int2 place = reinterpret_cast<const int2 *>(a.q_xy)[sp.q0 + qi];
        qx = (float)place.x * kPxPerQuantum;
        qy = (float)place.y * kPxPerQuantum;
        slope2 = a.slopes[qh] * kLog2e;
    }
    const float scale = score_scale<CAP>(a), cap2 = a.cap * kLog2e;
    // distances on the matrix cores: the row's factors, what they leave for the
    // row, and the largest |b|^2 that any slope of the rows' heads allows
    int2 origin = make_int2(0, 0);
    float largest = 0.0f, row_term = 0.0f;
    bool row_near = false;
    bf16x8 row_slots = {};
    if (DIST) {
        int i, gg;
        run.find(a, min(col, n_rows - 1 - row0), i, gg);
        origin = near_origin(reinterpret_cast<const int2 *>(a.q_xy)[sp.q0 + i]);
        largest = near_largest<T, CAP>(a, head, scale);
        const int ax = (int)(qx * 16.0f) - origin.x, ay = (int)(qy * 16.0f) - origin.y;
        const float n = square_quanta(ax, ay), weight = slope2 / 256.0f;
        row_near = !a.lse && __all(!valid || near_enough(ax, ay, n, largest));
        const float units = CAP ? weight : weight / scale;
        row_term = -units * n + (CAP ? cap_constant<CAP>(cap2) : 0.0f);  // with the constant of tanh = 1 - 2 r
        const NearSlots s = near_row(ax, ay, units);
        row_slots = __builtin_bit_cast(bf16x8, h ? s.half[1] : s.half[0]);
    }
    // the keys that any of the wave's rows sees, that all of them see, and that
    // any of the workgroup's sees
    int wave_end = sp.nk, wave_all = sp.nk, end = sp.nk;
    if (a.causal) {
        wave_end = wave_max(limit);
        wave_all = -wave_max(-limit);
        end = seen_limit(a, sp, prefix, run.query(a, min(kRows, n_rows - row0) - 1));
    }

    f32x16 o[DP / 32] = {};
    float m = -INFINITY, shift = 0.0f, l = 0.0f;

    // A tile is worked on at once where registers allow it for the waves there are
    // (no distances), else by halves.  A weight is
    // 2^(s * unit - shift): scores without caps (and with distances on the matrix
    // cores) stay products until then.
    constexpr bool PLAIN = !DIST && !CAP;
    constexpr int SUBS = DIST ? 1 : 2;
    auto near_term = [&](const typename Tile::Lds &t, int first) {
        // the sum begins at the row's term, so that it is small again before the products come in
        const bf16x8 k = __builtin_bit_cast(bf16x8, t.near[h * kTileKeys + first + col]);
        f32x16 start;
#pragma unroll
        for (int r = 0; r < 16; ++r) start[r] = row_term;
        return mfma(k, row_slots, start);
    };
    auto work = [&](const typename Tile::Lds &t, int first, int first_key, bool near, bool hidden, bool limited) {
        f32x16 s[SUBS];
#pragma unroll
        for (int u = 0; u < SUBS; ++u) {
            s[u] = f32x16{};
            if (near && !CAP) s[u] = near_term(t, first + 32 * u);
#pragma unroll
            for (int st = 0; st < DP / 16; ++st)
                s[u] = mfma(read_rows<T, Pitch<DP>::kRows>(t.k, first + 32 * u + col, st, h), q[st], s[u]);
        }
        if (CAP) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u) cap_parts<CAP>(s[u], scale);
        }
        const float unit = PLAIN || (near && !CAP) ? scale : 1.0f;
        if (near && CAP) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
                const f32x16 term = near_term(t, first + 32 * u);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = capped<CAP>(s[u][r], cap2, term[r]);
            }
        } else if (!PLAIN && !near) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    float kx[4], ky[4];
                    if (DIST) {
                        *reinterpret_cast<float4 *>(kx) = read4(t.x, first + 32 * u, r, h);
                        *reinterpret_cast<float4 *>(ky) = read4(t.y, first + 32 * u, r, h);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float d2 = DIST ? distance2(qx - kx[e], qy - ky[e]) : 0.0f;
                        s[u][r + e] = score<DIST, CAP>(s[u][r + e], scale, cap2, d2, slope2);
                    }
                }
        }
        if (hidden) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const float4 pen = read4(t.penalty, first + 32 * u, r, h);
                    s[u][r] += pen.x;
                    s[u][r + 1] += pen.y;
                    s[u][r + 2] += pen.z;
                    s[u][r + 3] += pen.w;
                }
        }
        if (limited) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
                const uint32_t seen = seen_bits(0xffffffffu, limit, first_key + 32 * u, h);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = (seen >> out_row(r, 0)) & 1 ? s[u][r] : -INFINITY;
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int u = 0; u < SUBS; ++u) top = fmaxf(top, s[u][r]);
        top = unit * across(top, [](float x, float y) { return fmaxf(x, y); });
        if (__any(top > m + kSlack)) {
            // 2^(old shift - new shift); the first scores seen find nothing to rescale
            m = fmaxf(m, top);
            const float to = m == -INFINITY ? 0.0f : m;
            const float fade = exp2_fast(fminf(shift - to, 0.0f));
            shift = to;
            l *= fade;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= fade;
        }
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < SUBS; ++u) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[u][r] = exp2_fast(__builtin_fmaf(s[u][r], unit, -shift));
                sum[r & 1] += s[u][r];
            }
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const F p = round_frag<T>(s[u], part);
#pragma unroll
                for (int b = 0; b < DP / 32; ++b)
                    o[b] = mfma(read_columns<T, Pitch<DP>::kColumns>(t.v, first + 32 * u + 16 * part, b, lane), p, o[b]);
            }
        }
        l += sum[0] + sum[1];
    };

    Tile next(a);
    if (end > 0) {
        next.look_up(a, sp, 0, end);
        next.template load<DIST>(a, sp, head, 0, end);
        next.look_up(a, sp, kTileKeys, end);
        next.template store<DIST>(a, typename Tile::Lds(shared), origin, largest);
    }
    wait_for_loads();
    __syncthreads();
    int buffer = 0;
    for (int kt = 0; kt < end; kt += kTileKeys) {
        const bool more = kt + kTileKeys < end;
        if (more) {
            next.template load<DIST>(a, sp, head, kt + kTileKeys, end);
            next.look_up(a, sp, kt + 2 * kTileKeys, end);
        }
        const typename Tile::Lds t(shared + buffer * Tile::kBytes);
        const uint64_t seen = *t.seen;
        if (kt < wave_end) {
            const bool near = DIST && row_near && __builtin_amdgcn_readfirstlane(*t.all_near);
#pragma unroll
            for (int sub = 0; sub < 2; sub += SUBS) {
                constexpr uint64_t kAll = SUBS == 2 ? ~0ull : 0xffffffffull;
                const uint64_t bits = (seen >> (32 * sub)) & kAll;
                const uint32_t some = __builtin_amdgcn_readfirstlane((uint32_t)(bits | (bits >> 32)));
                const bool hidden = __builtin_amdgcn_readfirstlane(bits == kAll) == 0;
                if (some != 0) work(t, 32 * sub, kt + 32 * sub, near, hidden, kt + 32 * (sub + SUBS) > wave_all);
            }
        }
        buffer ^= 1;
        if (more) next.template store<DIST>(a, typename Tile::Lds(shared + buffer * Tile::kBytes), origin, largest);
        __syncthreads();
    }
    l = across(l, [](float x, float y) { return x + y; });
    if (!valid) return;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    T *out = static_cast<T *>(a.out) + (int64_t)(sp.q0 + qi) * a.out_stride + qh * a.dim;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * b + out_row(r, h);
            if (d < a.dim) {
                const float z[4] = {o[b][r] * inv, o[b][r + 1] * inv, o[b][r + 2] * inv, o[b][r + 3] * inv};
                store_pack<T, 4>(out + d, z);
            }
        }
    if (a.lse && h == 0) a.lse[(int64_t)(sp.q0 + qi) * a.q_heads + qh] = row_lse(shift, l);
}

// ---------------------------------------------------------------------------
// Forward, few rows: 32 rows a workgroup, its waves over a quarter of the keys
// each, joined in LDS, and where a.splits > 1 each workgroup over a share of the
// keys, joined by attention_join_kernel: for launches that would leave the card
// idle otherwise, and for rows too few to fill a tile.  Bound by memory over a
// long history: 256 frames of one query and 8000 keys, 8 heads over 2 of 128,
// 352 us, 6.0 TB/s of keys and values (the first form, a tile at a time without
// loads ahead, took 724); one frame of 500 birds 11.3 us, the chain of loads,
// four tiles and the joint.
// ---------------------------------------------------------------------------

// (two workgroups of a compute unit have LDS for rows of 17 chunks with heads of 128, not of 20)
template <int DP>
using SplitTile = KeyTile<DP, 128, Pitch<DP>::kRows, DP == 128 ? 17 : Pitch<DP>::kColumns, false>;

template <int DP>
constexpr int split_lds_bytes() {
    const int join = 4 * 32 * (DP + 2) * 4;
    const int tiles = SplitTile<DP>::kBytes + 32 * Pitch<DP>::kRows * 16;
    return join > tiles ? join : tiles;
}

template <typename T, int DP, bool DIST, int CAP>
__global__ void __launch_bounds__(kThreads, DP == 128 && DIST && CAP ? 1 : 2) attention_split_kernel(AttentionArgs a) {
    using F = typename Frag<T>::type;
    constexpr int kRows = 32, kKeys = 128;
    using Tile = SplitTile<DP>;
    constexpr int kVPitch = DP == 128 ? 17 : Pitch<DP>::kColumns;
    extern __shared__ char shared[];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, col = lane & 31;
    const int64_t id = xcd_order(blockIdx.x, gridDim.x);
    const int head = (int)(id / a.slots);
    const int split = blockIdx.y;
    int64_t tile;
    const int f = find_frame(a.q_offsets, a.n_frames, a.group, kRows, id % a.slots, &tile);
    const Span sp = frame_span(a, f);
    if (!sp.ok || tile < 0) return;
    const int n_rows = sp.nq * a.group;
    if (tile * kRows >= n_rows) return;
    const int row0 = (int)tile * kRows;
    const RowRun run(a, row0);

    // keys that any of the workgroup's rows sees
    const int prefix = a.causal && a.prefix ? min(max(a.prefix[f], 0), sp.nk) : 0;
    int end = seen_limit(a, sp, prefix, run.query(a, min(kRows, n_rows - row0) - 1));
    int begin = 0;
    if (a.splits > 1) {
        const int per = ((sp.nk + a.splits - 1) / a.splits + kKeys - 1) / kKeys * kKeys;
        begin = (int)min((int64_t)split * per, (int64_t)end);
        end = (int)min(begin + (int64_t)per, (int64_t)end);
    }
    Tile next(a);
    if (begin < end) {
        next.look_up(a, sp, begin, end);
        next.template load<DIST>(a, sp, head, begin, end);
        next.look_up(a, sp, begin + kKeys, end);
    }

    // this lane's query
    const bool valid = row0 + col < n_rows;
    int qi = 0, g = 0;
    if (valid) run.find(a, col, qi, g);
    const int qh = head * a.group + g;
    // the rows stay in LDS: the loads in flight take the registers
    i16x8 *const q_lds = reinterpret_cast<i16x8 *>(shared + Tile::kBytes);
    for (int e = threadIdx.x; e < kRows * Tile::kChunks; e += kThreads) {
        const int r = e / Tile::kChunks, c = e % Tile::kChunks;
        i16x8 z = {};
        if (row0 + r < n_rows && c * 8 < a.dim) {
            int i, gg;
            run.find(a, r, i, gg);
            z = *reinterpret_cast<const i16x8 *>(static_cast<const short *>(a.q) + (int64_t)(sp.q0 + i) * a.q_stride +
                                                 (head * a.group + gg) * a.dim + c * 8);
        }
        q_lds[r * Pitch<DP>::kRows + c] = z;
    }
    const int limit = valid ? seen_limit(a, sp, prefix, qi) : sp.nk;
    const int all_end = a.causal ? -wave_max(-limit) : sp.nk;
    float qx = 0.0f, qy = 0.0f, slope2 = 0.0f;
    if (DIST && valid) {
        const int2 place = reinterpret_cast<const int2 *>(a.q_xy)[sp.q0 + qi];
        qx = (float)place.x * kPxPerQuantum;
        qy = (float)place.y * kPxPerQuantum;
        slope2 = a.slopes[qh] * kLog2e;
    }
    const float scale = score_scale<CAP>(a), cap2 = a.cap * kLog2e;

    f32x16 o[DP / 32] = {};
    float m = -INFINITY, shift = 0.0f, l = 0.0f;
    const typename Tile::Lds t(shared);
    const int k0 = 32 * wave;
    for (int kt = begin; kt < end; kt += kKeys) {
        if (kt > begin) __syncthreads();
        next.template store<DIST>(a, t);
        __syncthreads();
        if (kt + kKeys < end) {
            next.template load<DIST>(a, sp, head, kt + kKeys, end);
            next.look_up(a, sp, kt + 2 * kKeys, end);
        }
        const uint32_t bits = __builtin_amdgcn_readfirstlane(reinterpret_cast<const uint32_t *>(t.seen)[wave]);
        if (bits == 0) continue;
        f32x16 s = {};
#pragma unroll
        for (int st = 0; st < DP / 16; ++st) 
            s = mfma(read_rows<T, Pitch<DP>::kRows>(t.k, k0 + col, st, h), read_rows<T, Pitch<DP>::kRows>(q_lds, col, st, h), s);
        if (CAP) cap_parts<CAP>(s, scale);
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            float kx[4], ky[4], pen[4] = {};
            if (DIST) {
                *reinterpret_cast<float4 *>(kx) = read4(t.x, k0, r, h);
                *reinterpret_cast<float4 *>(ky) = read4(t.y, k0, r, h);
            }
            if (bits != 0xffffffffu) *reinterpret_cast<float4 *>(pen) = read4(t.penalty, k0, r, h);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float d2 = DIST ? distance2(qx - kx[e], qy - ky[e]) : 0.0f;
                s[r + e] = score<DIST, CAP>(s[r + e], scale, cap2, d2, slope2) + pen[e];
            }
        }
        if (kt + k0 + 32 > all_end) {
            const uint32_t seen = seen_bits(0xffffffffu, limit, kt + k0, h);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = (seen >> out_row(r, 0)) & 1 ? s[r] : -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[r]);
        top = across(top, [](float x, float y) { return fmaxf(x, y); });
        if (__any(top > m + kSlack)) {
            m = fmaxf(m, top);
            const float to = m == -INFINITY ? 0.0f : m;
            const float fade = exp2_fast(fminf(shift - to, 0.0f));
            shift = to;
            l *= fade;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= fade;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = exp2_fast(s[r] - shift);
            l += s[r];
        }
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const F p = round_frag<T>(s, part);
#pragma unroll
            for (int b = 0; b < DP / 32; ++b) o[b] = mfma(read_columns<T, kVPitch>(t.v, k0 + 16 * part, b, lane), p, o[b]);
        }
    }
    l = across(l, [](float x, float y) { return x + y; });

    // join the waves' shares of the keys
    float *const join = reinterpret_cast<float *>(shared);
    constexpr int kPitch = DP + 2;
    __syncthreads();
    {
        float *mine = join + (wave * 32 + col) * kPitch;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) mine[32 * b + out_row(r, h)] = o[b][r];
        if (h == 0) {
            mine[DP] = m == -INFINITY ? m : shift;
            mine[DP + 1] = l;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 32 * DP; e += kThreads) {
        const int c = e / DP, d = e % DP;
        if (row0 + c >= n_rows || d >= a.dim) continue;
        float top = -INFINITY;
        for (int w = 0; w < 4; ++w) top = fmaxf(top, join[(w * 32 + c) * kPitch + DP]);
        const float shift = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f, z = 0.0f;
        for (int w = 0; w < 4; ++w) {
            const float *p = join + (w * 32 + c) * kPitch;
            const float fade = exp2_fast(p[DP] - shift);
            sum += p[DP + 1] * fade;
            z += p[d] * fade;
        }
        int iq, gg;
        run.find(a, c, iq, gg);
        const int64_t i = sp.q0 + iq;
        const int hh = head * a.group + gg;
        const int64_t at = i * a.q_heads + hh;
        if (a.splits > 1) {
            const int64_t all = (int64_t)a.total_q * a.q_heads;
            a.part_out[((int64_t)split * all + at) * a.dim + d] = z;
            if (d == 0) {
                a.part_stat[2 * ((int64_t)split * all + at)] = top;
                a.part_stat[2 * ((int64_t)split * all + at) + 1] = sum;
            }
        } else {
            static_cast<T *>(a.out)[i * a.out_stride + hh * a.dim + d] = static_cast<T>(sum > 0.0f ? z / sum : 0.0f);
            if (a.lse && d == 0) a.lse[at] = row_lse(top, sum);
        }
    }
}

// Joins the shares of the keys: a wave per query and head.
template <typename T>
__global__ void __launch_bounds__(kThreads) attention_join_kernel(AttentionArgs a) {
    const int64_t all = (int64_t)a.total_q * a.q_heads;
    const int64_t at = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (at >= all) return;
    // a query of an inconsistent frame has no shares: its output is left alone
    const int64_t i = at / a.q_heads;
    int lo = 0, hi = a.n_frames - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.q_offsets[mid] <= i) lo = mid;
        else hi = mid - 1;
    }
    const Span sp = frame_span(a, lo);
    if (!sp.ok || i < sp.q0 || i >= sp.q0 + sp.nq) return;
    // a lane per share (at most 64) for the weights, a lane per dimension for the sums
    const int lane = threadIdx.x & 63;
    float m = -INFINITY, l = 0.0f;
    if (lane < a.splits) {
        const float2 stat = *reinterpret_cast<const float2 *>(a.part_stat + 2 * (lane * all + at));
        m = stat.x;
        l = stat.y;
    }
    float top = m;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float shift = top == -INFINITY ? 0.0f : top;
    const float weight = exp2_fast(m - shift);
    float sum = l * weight;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    float z[2] = {0.0f, 0.0f};  // dimensions lane and lane + 64
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) {
        const float w = __shfl(weight, s);
        const float *part = a.part_out + (s * all + at) * a.dim;
        if (lane < a.dim) z[0] += part[lane] * w;
        if (lane + 64 < a.dim) z[1] += part[lane + 64] * w;
    }
    T *out = static_cast<T *>(a.out) + i * a.out_stride + (at % a.q_heads) * a.dim;
    if (lane < a.dim) out[lane] = static_cast<T>(z[0] * inv);
    if (lane + 64 < a.dim) out[lane + 64] = static_cast<T>(z[1] * inv);
    if (a.lse && lane == 0) a.lse[at] = row_lse(top, sum);
}

constexpr int kMaxSplits = 64;

}  // namespace

AttentionPlan plan_attention(int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads, int32_t kv_heads,
                             int n_cus) {
    AttentionPlan p{};
    if (n_frames <= 0 || total_q <= 0 || q_heads <= 0 || kv_heads <= 0) return p;
    const int64_t rows = (int64_t)total_q * (q_heads / kv_heads);
    const int64_t tiles = rows / 128 + n_frames;
    // few rows a frame would fill half a 128-row tile at most; few tiles leave compute units idle
    p.split = tiles * kv_heads < 2 * (int64_t)n_cus || rows / n_frames <= 64;
    p.slots = rows / (p.split ? 32 : 128) + n_frames;
    p.splits = 1;
    if (p.split) {
        // two workgroups a compute unit, each with two tiles of 128 keys at least
        const int64_t real = std::max<int64_t>(rows / 32, n_frames) * kv_heads;
        const int64_t keys = (int64_t)total_k / n_frames;
        int64_t s = (2 * (int64_t)n_cus + real - 1) / real;
        s = std::min<int64_t>(s, keys / 256);
        p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(s, kMaxSplits));
    }
    return p;
}

int64_t attention_workgroups(const AttentionPlan &p, int32_t total_q, int32_t q_heads, int32_t kv_heads) {
    const int64_t joins = p.splits > 1 ? ((int64_t)total_q * q_heads + 3) / 4 : 0;
    return std::max(p.slots * kv_heads, joins);
}

size_t attention_workspace_bytes(const AttentionPlan &p, int32_t total_q, int32_t q_heads, int32_t dim) {
    if (p.splits <= 1) return 0;
    const size_t all = (size_t)total_q * (size_t)q_heads * (size_t)p.splits;
    return align256(all * (size_t)dim * sizeof(float)) + align256(all * 2 * sizeof(float));
}

hipError_t launch_attention(AttentionArgs a, int32_t dtype, const AttentionPlan &p, void *workspace,
                            hipStream_t stream) {
    a.slots = p.slots;
    a.splits = p.splits;
    a.group_reciprocal = group_reciprocal(a.group);
    if (p.splits > 1) {
        const size_t all = (size_t)a.total_q * (size_t)a.q_heads * (size_t)p.splits;
        a.part_out = static_cast<float *>(workspace);
        a.part_stat = reinterpret_cast<float *>(static_cast<char *>(workspace) + align256(all * (size_t)a.dim * sizeof(float)));
    }
    hipError_t err = with_kernel(a, dtype, [&](auto t, auto dp, auto dist, auto cap) {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool DIST = decltype(dist)::value;
        constexpr int CAP = decltype(cap)::value;
        constexpr size_t rows_bytes = 2 * RowsTile<DP, DIST>::kBytes;
        const dim3 grid((uint32_t)(p.slots * a.kv_heads), (uint32_t)p.splits);
        if (p.split)
            hipLaunchKernelGGL((attention_split_kernel<T, DP, DIST, CAP>), grid, dim3(kThreads), split_lds_bytes<DP>(),
                               stream, a);
        else
            hipLaunchKernelGGL((attention_rows_kernel<T, DP, DIST, CAP>), grid, dim3(kThreads), rows_bytes,
                               stream, a);
        return hipGetLastError();
    });
    if (err != hipSuccess || p.splits <= 1) return err;
    const int64_t all = (int64_t)a.total_q * a.q_heads;
    const dim3 grid((uint32_t)((all + 3) / 4));
    if (dtype == FLOCK_F16) hipLaunchKernelGGL(attention_join_kernel<half_t>, grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL(attention_join_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace flock
