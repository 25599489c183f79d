// attention.hip - attention of the birds of a frame (or of a track) among
// themselves, or of a few queries over them, and its backward pass.
//
// For query i and key j of a frame, head h, d2 their squared distance in px^2:
//   t = scale q_i.k_j, capped: t = cap tanh(t / cap);   s = t - slope_h d2
//   key j is seen by query i: keep[j], and in ordered frames j < limit_i with
//   limit_i = max(prefix, i + n_k - n_q + 1)
//   out_i = sum_j softmax_j(s) v_j over the keys seen, 0 where there are none
//   backward: P = exp(s - lse), delta_i = dout_i.out_i, dP = dout_i.v_j
//   dS = P (dP - delta), dT = dS (1 - (t / cap)^2)
//   dq = scale dT k, dk = scale dT^T q, dv = P^T dout, dslope_h = -sum dS d2
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

#include "encoder_common.h"

namespace flock {
namespace {

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

// ---------------------------------------------------------------------------
// Forward.  SPLIT = false: 128 rows a workgroup, 32 a wave, all waves over the
// same keys.  SPLIT = true: 32 rows a workgroup, its waves over a quarter of
// the keys each, joined in LDS, and where a.splits > 1 each workgroup over a
// share of the keys, joined by attention_join_kernel: for launches that would
// leave the card idle otherwise, and for rows too few to fill a tile.
// ---------------------------------------------------------------------------

template <int DP, bool SPLIT>
constexpr int forward_lds_bytes() {
    constexpr int kKeys = SPLIT ? 128 : 64;
    int bytes = 2 * kKeys * (DP + 8) * 2 + 2 * kKeys * 4;
    if (SPLIT) {
        const int join = 4 * 32 * (DP + 2) * 4;
        if (join > bytes) bytes = join;
    }
    return bytes;
}

template <typename T, int DP, bool SPLIT, bool DIST, bool CAP>
__global__ void __launch_bounds__(kThreads) attention_kernel(AttentionArgs a) {
    using F = typename Frag<T>::type;
    constexpr int kRows = SPLIT ? 32 : 128;
    constexpr int kKeys = SPLIT ? 128 : 64;
    constexpr int kSubs = SPLIT ? 1 : kKeys / 32;
    extern __shared__ i16x8 lds[];
    i16x8 *const k_lds = lds;
    i16x8 *const v_lds = lds + kKeys * (DP / 8 + 1);
    float *const kx = reinterpret_cast<float *>(v_lds + kKeys * (DP / 8 + 1));
    float *const ky = kx + kKeys;

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, col = lane & 31;
    const int64_t id = xcd_order(blockIdx.x, gridDim.x);
    const int head = (int)(id / a.slots);
    const int split = SPLIT ? blockIdx.y : 0;
    int64_t tile;
    const int f = find_frame(a.q_offsets, a.n_frames, a.group, kRows, id % a.slots, &tile);
    const Span sp = frame_span(a, f);
    if (!sp.ok || tile < 0) return;
    const int64_t n_rows = (int64_t)sp.nq * a.group;
    const int64_t row0 = tile * kRows;
    if (row0 >= n_rows) return;

    // this lane's query
    const int64_t row = row0 + (SPLIT ? 0 : 32 * wave) + col;
    const bool valid = row < n_rows;
    const int qi = valid ? (int)(row / a.group) : 0, g = valid ? (int)(row % a.group) : 0;
    const int qh = head * a.group + g;
    const short *q_row = valid ? static_cast<const short *>(a.q) + (int64_t)(sp.q0 + qi) * a.q_stride + qh * a.dim
                               : nullptr;
    F q[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) q[s] = load_frag<T>(q_row, s, h, a.dim);
    const int prefix = a.causal && a.prefix ? min(max(a.prefix[f], 0), sp.nk) : 0;
    const int limit = !valid ? 0 : a.causal ? min(max((int64_t)prefix, (int64_t)qi + sp.nk - sp.nq + 1), (int64_t)sp.nk) : sp.nk;
    float qx = 0.0f, qy = 0.0f, slope2 = 0.0f;
    if (DIST && valid) {
        qx = (float)a.q_xy[2 * (int64_t)(sp.q0 + qi)] * kPxPerQuantum;
        qy = (float)a.q_xy[2 * (int64_t)(sp.q0 + qi) + 1] * kPxPerQuantum;
        slope2 = a.slopes[qh] * kLog2e;
    }
    const float scale = CAP ? a.scale / a.cap : a.scale * kLog2e, cap2 = a.cap * kLog2e;

    // keys that any of the workgroup's rows sees
    const int last = (int)((min(row0 + kRows, n_rows) - 1) / a.group);
    int end = a.causal ? (int)min(max((int64_t)prefix, (int64_t)last + sp.nk - sp.nq + 1), (int64_t)sp.nk) : sp.nk;
    int begin = 0;
    if (SPLIT && a.splits > 1) {
        const int per = ((sp.nk + a.splits - 1) / a.splits + kKeys - 1) / kKeys * kKeys;
        begin = min((int64_t)split * per, (int64_t)end);
        end = min(begin + (int64_t)per, (int64_t)end);
    }

    f32x16 o[DP / 32] = {};
    float m = -INFINITY, l = 0.0f;
    for (int kt = begin; kt < end; kt += kKeys) {
        __syncthreads();
        auto key_row = [&](const void *base, int64_t stride, int r) -> const short * {
            const int j = kt + r;
            if (j >= end || (a.keep && !a.keep[sp.k0 + j])) return nullptr;
            return static_cast<const short *>(base) + (int64_t)(sp.k0 + j) * stride + head * a.dim;
        };
        stage_rows<DP, kKeys>(k_lds, a.dim, [&](int r) { return key_row(a.k, a.k_stride, r); });
        stage_rows<DP, kKeys>(v_lds, a.dim, [&](int r) { return key_row(a.v, a.v_stride, r); });
        if (DIST && threadIdx.x < kKeys) {
            const int j = kt + (int)threadIdx.x;
            kx[threadIdx.x] = j < end ? (float)a.k_xy[2 * (int64_t)(sp.k0 + j)] * kPxPerQuantum : 0.0f;
            ky[threadIdx.x] = j < end ? (float)a.k_xy[2 * (int64_t)(sp.k0 + j) + 1] * kPxPerQuantum : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int sub = 0; sub < kSubs; ++sub) {
            const int k0 = SPLIT ? 32 * wave : 32 * sub;
            const int j = kt + k0 + col;
            const uint32_t bits = (uint32_t)__ballot(h == 0 && j < end && (!a.keep || a.keep[sp.k0 + j]));
            if (bits == 0) continue;
            f32x16 s = {};
#pragma unroll
            for (int st = 0; st < DP / 16; ++st) s = mfma(read_rows<T, DP>(k_lds, k0 + col, st, h), q[st], s);
            const uint32_t seen = seen_bits(bits, limit, kt + k0, h);
            float top = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int kr = k0 + out_row(r, h);
                float d2 = 0.0f;
                if (DIST) {
                    d2 = distance2(qx - kx[kr], qy - ky[kr]);
                }
                float th;
                const float v = score<DIST, CAP>(s[r], scale, cap2, d2, slope2, th);
                s[r] = (seen >> out_row(r, 0)) & 1 ? v : -INFINITY;
                top = fmaxf(top, s[r]);
            }
            top = across(top, [](float x, float y) { return fmaxf(x, y); });
            const float m_new = fmaxf(m, top);
            const float shift = m_new == -INFINITY ? 0.0f : m_new;
            const float fade = exp2_fast(m - shift);
            m = m_new;
            l *= fade;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = exp2_fast(s[r] - shift);
                l += s[r];
            }
#pragma unroll
            for (int b = 0; b < DP / 32; ++b) {
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= fade;
#pragma unroll
                for (int part = 0; part < 2; ++part)
                    o[b] = mfma(read_columns<T, DP>(v_lds, k0 + 16 * part, b, lane), round_frag<T>(s, part), o[b]);
            }
        }
    }
    l = across(l, [](float x, float y) { return x + y; });

    if (!SPLIT) {
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
        if (a.lse && h == 0)
            a.lse[(int64_t)(sp.q0 + qi) * a.q_heads + qh] = row_lse(m, l);
        return;
    }

    // join the waves' shares of the keys
    float *const join = reinterpret_cast<float *>(lds);
    constexpr int kPitch = DP + 2;
    __syncthreads();
    {
        float *mine = join + (wave * 32 + col) * kPitch;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) mine[32 * b + out_row(r, h)] = o[b][r];
        if (h == 0) {
            mine[DP] = m;
            mine[DP + 1] = l;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 32 * DP; e += kThreads) {
        const int c = e / DP, d = e % DP;
        const int64_t r = row0 + c;
        if (r >= n_rows || d >= a.dim) continue;
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
        const int64_t i = sp.q0 + r / a.group;
        const int hh = head * a.group + (int)(r % a.group);
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
    float top = -INFINITY;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, a.part_stat[2 * (s * all + at)]);
    const float shift = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
    for (int s = 0; s < a.splits; ++s)
        sum += a.part_stat[2 * (s * all + at) + 1] * exp2_fast(a.part_stat[2 * (s * all + at)] - shift);
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    T *out = static_cast<T *>(a.out) + i * a.out_stride + (at % a.q_heads) * a.dim;
    for (int d = threadIdx.x & 63; d < a.dim; d += 64) {
        float z = 0.0f;
        for (int s = 0; s < a.splits; ++s)
            z += a.part_out[(s * all + at) * a.dim + d] * exp2_fast(a.part_stat[2 * (s * all + at)] - shift);
        out[d] = static_cast<T>(z * inv);
    }
    if (a.lse && (threadIdx.x & 63) == 0) a.lse[at] = row_lse(top, sum);
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------

// delta = dout.out of every query and head: 16 lanes each.
template <typename T>
__global__ void __launch_bounds__(kThreads) attention_delta_kernel(AttentionBackwardArgs b) {
    const AttentionArgs &a = b.fwd;
    const int64_t all = (int64_t)a.total_q * a.q_heads;
    const int64_t at = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    if (at >= all) return;
    const int64_t i = at / a.q_heads;
    const int hd = (int)(at % a.q_heads);
    const T *o = static_cast<const T *>(a.out) + i * a.out_stride + hd * a.dim;
    const T *g = static_cast<const T *>(b.grad_out) + i * b.grad_out_stride + hd * a.dim;
    float s = 0.0f;
    for (int d = (threadIdx.x & 15) * 8; d < a.dim; d += 128) {
        float x[8], y[8];
        load_pack<T, 8>(o + d, x);
        load_pack<T, 8>(g + d, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += x[e] * y[e];
    }
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 15) == 0) {
        b.delta[at] = s;
        if (b.row_slopes) b.row_slopes[at] = 0.0f;  // queries of inconsistent frames add nothing
    }
}

// Gradients of the queries: 128 rows a workgroup, over the keys they see.
template <typename T, int DP, bool DIST, bool CAP>
__global__ void __launch_bounds__(kThreads) attention_dq_kernel(AttentionBackwardArgs b) {
    using F = typename Frag<T>::type;
    constexpr int kRows = 128, kKeys = 64;
    const AttentionArgs &a = b.fwd;
    extern __shared__ i16x8 lds[];
    i16x8 *const k_lds = lds;
    i16x8 *const v_lds = lds + kKeys * (DP / 8 + 1);
    float *const kx = reinterpret_cast<float *>(v_lds + kKeys * (DP / 8 + 1));
    float *const ky = kx + kKeys;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, col = lane & 31;
    const int64_t id = xcd_order(blockIdx.x, gridDim.x);
    const int head = (int)(id / a.slots);
    int64_t tile;
    const int f = find_frame(a.q_offsets, a.n_frames, a.group, kRows, id % a.slots, &tile);
    const Span sp = frame_span(a, f);
    if (!sp.ok || tile < 0) return;
    const int64_t n_rows = (int64_t)sp.nq * a.group;
    const int64_t row0 = tile * kRows;
    if (row0 >= n_rows) return;
    const int64_t row = row0 + 32 * wave + col;
    const bool valid = row < n_rows;
    const int qi = valid ? (int)(row / a.group) : 0, g = valid ? (int)(row % a.group) : 0;
    const int qh = head * a.group + g;
    const int64_t qrow = sp.q0 + qi;
    const short *q_row = valid ? static_cast<const short *>(a.q) + qrow * a.q_stride + qh * a.dim : nullptr;
    const short *g_row = valid ? static_cast<const short *>(b.grad_out) + qrow * b.grad_out_stride + qh * a.dim : nullptr;
    F q[DP / 16], go[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        q[s] = load_frag<T>(q_row, s, h, a.dim);
        go[s] = load_frag<T>(g_row, s, h, a.dim);
    }
    const int prefix = a.causal && a.prefix ? min(max(a.prefix[f], 0), sp.nk) : 0;
    const int limit = !valid ? 0 : a.causal ? min(max((int64_t)prefix, (int64_t)qi + sp.nk - sp.nq + 1), (int64_t)sp.nk) : sp.nk;
    float qx = 0.0f, qy = 0.0f, slope2 = 0.0f;
    if (DIST && valid) {
        qx = (float)a.q_xy[2 * qrow] * kPxPerQuantum;
        qy = (float)a.q_xy[2 * qrow + 1] * kPxPerQuantum;
        slope2 = a.slopes[qh] * kLog2e;
    }
    const float scale = CAP ? a.scale / a.cap : a.scale * kLog2e, cap2 = a.cap * kLog2e;
    float shift, rest;
    split_lse(valid ? a.lse[qrow * a.q_heads + qh] : -INFINITY, shift, rest);
    const float delta = valid ? b.delta[qrow * a.q_heads + qh] * rest : 0.0f;
    const int last = (int)((min(row0 + kRows, n_rows) - 1) / a.group);
    const int end = a.causal ? (int)min(max((int64_t)prefix, (int64_t)last + sp.nk - sp.nq + 1), (int64_t)sp.nk) : sp.nk;

    f32x16 dq[DP / 32] = {};
    // sums of P dP, P d2 and P dP d2: the slope's gradient takes delta from the
    // same P, since dS = P (dP - delta) sums to zero only then to 32 bits
    float pdp = 0.0f, pd2 = 0.0f, pdpd2 = 0.0f;
    for (int kt = 0; kt < end; kt += kKeys) {
        __syncthreads();
        auto key_row = [&](const void *base, int64_t stride, int r) -> const short * {
            const int j = kt + r;
            if (j >= end || (a.keep && !a.keep[sp.k0 + j])) return nullptr;
            return static_cast<const short *>(base) + (int64_t)(sp.k0 + j) * stride + head * a.dim;
        };
        stage_rows<DP, kKeys>(k_lds, a.dim, [&](int r) { return key_row(a.k, a.k_stride, r); });
        stage_rows<DP, kKeys>(v_lds, a.dim, [&](int r) { return key_row(a.v, a.v_stride, r); });
        if (DIST && threadIdx.x < kKeys) {
            const int j = kt + (int)threadIdx.x;
            kx[threadIdx.x] = j < end ? (float)a.k_xy[2 * (int64_t)(sp.k0 + j)] * kPxPerQuantum : 0.0f;
            ky[threadIdx.x] = j < end ? (float)a.k_xy[2 * (int64_t)(sp.k0 + j) + 1] * kPxPerQuantum : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int sub = 0; sub < kKeys / 32; ++sub) {
            const int k0 = 32 * sub;
            const int j = kt + k0 + col;
            const uint32_t bits = (uint32_t)__ballot(h == 0 && j < end && (!a.keep || a.keep[sp.k0 + j]));
            if (bits == 0) continue;
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int st = 0; st < DP / 16; ++st) {
                s = mfma(read_rows<T, DP>(k_lds, k0 + col, st, h), q[st], s);
                dp = mfma(read_rows<T, DP>(v_lds, k0 + col, st, h), go[st], dp);
            }
            const uint32_t seen = seen_bits(bits, limit, kt + k0, h);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int kr = k0 + out_row(r, h);
                float d2 = 0.0f;
                if (DIST) {
                    d2 = distance2(qx - kx[kr], qy - ky[kr]);
                }
                float th;
                const float v = score<DIST, CAP>(s[r], scale, cap2, d2, slope2, th);
                // P / rest; rest is in the other factors
                const float p = (seen >> out_row(r, 0)) & 1 ? exp2_fast(v - shift) : 0.0f;
                if (DIST) {
                    const float pd = p * dp[r];
                    pdp += pd;
                    pd2 += p * d2;
                    pdpd2 += pd * d2;
                }
                float ds = p * __builtin_fmaf(dp[r], rest, -delta);
                if (CAP) ds *= 1.0f - th * th;
                s[r] = ds;
            }
#pragma unroll
            for (int blk = 0; blk < DP / 32; ++blk)
#pragma unroll
                for (int part = 0; part < 2; ++part)
                    dq[blk] = mfma(read_columns<T, DP>(k_lds, k0 + 16 * part, blk, lane), round_frag<T>(s, part), dq[blk]);
        }
    }
    if (DIST && b.row_slopes) {
        auto add = [](float x, float y) { return x + y; };
        pdp = across(pdp, add);
        pd2 = across(pd2, add);
        pdpd2 = across(pdpd2, add);
        if (valid && h == 0) b.row_slopes[qrow * a.q_heads + qh] = rest * (rest * pdp * pd2 - pdpd2);
    }
    if (!valid) return;
    T *out = static_cast<T *>(b.grad_q) + qrow * b.grad_q_stride + qh * a.dim;
#pragma unroll
    for (int blk = 0; blk < DP / 32; ++blk)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * blk + out_row(r, h);
            if (d < a.dim) {
                const float z[4] = {dq[blk][r] * a.scale, dq[blk][r + 1] * a.scale, dq[blk][r + 2] * a.scale,
                                    dq[blk][r + 3] * a.scale};
                store_pack<T, 4>(out + d, z);
            }
        }
}

// Gradients of keys and values: 128 keys a workgroup, 32 a wave, over the rows
// that see them.  The products are S = Q K^T and dP = dO V^T here, so that a lane
// holds one key.
template <typename T, int DP, bool DIST, bool CAP>
__global__ void __launch_bounds__(kThreads) attention_dkv_kernel(AttentionBackwardArgs b) {
    using F = typename Frag<T>::type;
    constexpr int kKeys = 128, kRows = 64;
    const AttentionArgs &a = b.fwd;
    extern __shared__ i16x8 lds[];
    i16x8 *const q_lds = lds;
    i16x8 *const g_lds = lds + kRows * (DP / 8 + 1);
    float *const r_shift = reinterpret_cast<float *>(g_lds + kRows * (DP / 8 + 1));
    float *const r_rest = r_shift + kRows;
    float *const r_delta = r_rest + kRows;
    float *const r_x = r_delta + kRows;
    float *const r_y = r_x + kRows;
    float *const r_slope = r_y + kRows;
    int *const r_limit = reinterpret_cast<int *>(r_slope + kRows);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, col = lane & 31;
    const int64_t id = xcd_order(blockIdx.x, gridDim.x);
    const int head = (int)(id / b.key_slots);
    int64_t tile;
    const int f = find_frame(a.k_offsets, a.n_frames, 1, kKeys, id % b.key_slots, &tile);
    const Span sp = frame_span(a, f);
    if (!sp.ok || tile < 0) return;
    const int64_t key0 = tile * kKeys;
    if (key0 >= sp.nk) return;
    const int64_t n_rows = (int64_t)sp.nq * a.group;
    const int64_t key = key0 + 32 * wave + col;
    const bool valid = key < sp.nk;
    const int64_t krow = sp.k0 + (valid ? key : 0);
    const bool kept = valid && (!a.keep || a.keep[krow]);
    const short *k_row = kept ? static_cast<const short *>(a.k) + krow * a.k_stride + head * a.dim : nullptr;
    const short *v_row = kept ? static_cast<const short *>(a.v) + krow * a.v_stride + head * a.dim : nullptr;
    F k[DP / 16], v[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        k[s] = load_frag<T>(k_row, s, h, a.dim);
        v[s] = load_frag<T>(v_row, s, h, a.dim);
    }
    float kx = 0.0f, ky = 0.0f;
    if (DIST && valid) {
        kx = (float)a.k_xy[2 * krow] * kPxPerQuantum;
        ky = (float)a.k_xy[2 * krow + 1] * kPxPerQuantum;
    }
    const float scale = CAP ? a.scale / a.cap : a.scale * kLog2e, cap2 = a.cap * kLog2e;
    const int prefix = a.causal && a.prefix ? min(max(a.prefix[f], 0), sp.nk) : 0;
    // the first query that sees the workgroup's first key
    int64_t begin = 0;
    if (a.causal && key0 >= prefix) begin = max((int64_t)0, key0 - sp.nk + sp.nq) * a.group / kRows * kRows;

    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    for (int64_t rt = begin; rt < n_rows; rt += kRows) {
        __syncthreads();
        auto row_of = [&](const void *base, int64_t stride, int r) -> const short * {
            const int64_t row = rt + r;
            if (row >= n_rows) return nullptr;
            return static_cast<const short *>(base) + (sp.q0 + row / a.group) * stride +
                   (head * a.group + (int)(row % a.group)) * a.dim;
        };
        stage_rows<DP, kRows>(q_lds, a.dim, [&](int r) { return row_of(a.q, a.q_stride, r); });
        stage_rows<DP, kRows>(g_lds, a.dim, [&](int r) { return row_of(b.grad_out, b.grad_out_stride, r); });
        if (threadIdx.x < kRows) {
            const int64_t row = rt + threadIdx.x;
            float shift = INFINITY, rest = 0.0f, delta = 0.0f, x = 0.0f, y = 0.0f, slope2 = 0.0f;
            int limit = 0;
            if (row < n_rows) {
                const int64_t i = row / a.group;
                const int qh = head * a.group + (int)(row % a.group);
                split_lse(a.lse[(sp.q0 + i) * a.q_heads + qh], shift, rest);
                delta = b.delta[(sp.q0 + i) * a.q_heads + qh];
                if (DIST) {
                    x = (float)a.q_xy[2 * (sp.q0 + i)] * kPxPerQuantum;
                    y = (float)a.q_xy[2 * (sp.q0 + i) + 1] * kPxPerQuantum;
                    slope2 = a.slopes[qh] * kLog2e;
                }
                limit = a.causal ? (int)min(max((int64_t)prefix, i + sp.nk - sp.nq + 1), (int64_t)sp.nk) : sp.nk;
            }
            r_shift[threadIdx.x] = shift;
            r_rest[threadIdx.x] = rest;
            r_delta[threadIdx.x] = delta;
            r_x[threadIdx.x] = x;
            r_y[threadIdx.x] = y;
            r_slope[threadIdx.x] = slope2;
            r_limit[threadIdx.x] = limit;
        }
        __syncthreads();
#pragma unroll
        for (int sub = 0; sub < kRows / 32; ++sub) {
            const int r0 = 32 * sub;
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int st = 0; st < DP / 16; ++st) {
                s = mfma(read_rows<T, DP>(q_lds, r0 + col, st, h), k[st], s);
                dp = mfma(read_rows<T, DP>(g_lds, r0 + col, st, h), v[st], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int rr = r0 + out_row(r, h);
                float th, d2 = 0.0f;
                if (DIST) d2 = distance2(r_x[rr] - kx, r_y[rr] - ky);
                const float z = score<DIST, CAP>(s[r], scale, cap2, d2, DIST ? r_slope[rr] : 0.0f, th);
                float p = exp2_fast(z - r_shift[rr]) * r_rest[rr];
                if (a.causal && key >= r_limit[rr]) p = 0.0f;
                float ds = p * (dp[r] - r_delta[rr]);
                if (CAP) ds *= 1.0f - th * th;
                s[r] = p;
                dp[r] = ds;
            }
#pragma unroll
            for (int blk = 0; blk < DP / 32; ++blk)
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    dv[blk] = mfma(read_columns<T, DP>(g_lds, r0 + 16 * part, blk, lane), round_frag<T>(s, part), dv[blk]);
                    dk[blk] = mfma(read_columns<T, DP>(q_lds, r0 + 16 * part, blk, lane), round_frag<T>(dp, part), dk[blk]);
                }
        }
    }
    if (!valid) return;
    // a hidden key's scores are not masked above: its gradients are zero
    T *dk_out = static_cast<T *>(b.grad_k) + krow * b.grad_k_stride + head * a.dim;
    T *dv_out = static_cast<T *>(b.grad_v) + krow * b.grad_v_stride + head * a.dim;
#pragma unroll
    for (int blk = 0; blk < DP / 32; ++blk)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * blk + out_row(r, h);
            if (d < a.dim) {
                float x[4], y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = kept ? dk[blk][r + e] * a.scale : 0.0f;
                    y[e] = kept ? dv[blk][r + e] : 0.0f;
                }
                store_pack<T, 4>(dk_out + d, x);
                store_pack<T, 4>(dv_out + d, y);
            }
        }
}

// Gradient of a head's slope: the queries' shares, a block per head and part
// of the queries, then the parts, in 64 bits and a fixed order.
constexpr int kSlopeParts = 64;

__global__ void __launch_bounds__(kThreads) slope_parts_kernel(const float *rows, int64_t total_q, int q_heads,
                                                               double *parts) {
    __shared__ double sums[kThreads];
    const int head = blockIdx.x, part = blockIdx.y;
    double s = 0.0;
    for (int64_t i = (int64_t)part * kThreads + threadIdx.x; i < total_q; i += (int64_t)kSlopeParts * kThreads)
        s += rows[i * q_heads + head];
    sums[threadIdx.x] = s;
    for (int d = kThreads / 2; d > 0; d >>= 1) {
        __syncthreads();
        if (threadIdx.x < d) sums[threadIdx.x] += sums[threadIdx.x + d];
    }
    if (threadIdx.x == 0) parts[head * kSlopeParts + part] = sums[0];
}

__global__ void __launch_bounds__(64) slope_total_kernel(const double *parts, float *grad_slopes) {
    double s = parts[blockIdx.x * kSlopeParts + threadIdx.x];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if (threadIdx.x == 0) grad_slopes[blockIdx.x] = (float)s;
}

// fn<T, DP, DIST, CAP>() of the call.
template <typename F>
hipError_t with_kernel(const AttentionArgs &a, int32_t dtype, F &&fn) {
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

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

constexpr int kMaxSplits = 64;

}  // namespace

AttentionPlan plan_attention(int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads, int32_t kv_heads,
                             int n_cus) {
    AttentionPlan p{};
    if (n_frames <= 0 || total_q <= 0 || q_heads <= 0 || kv_heads <= 0) return p;
    const int64_t rows = (int64_t)total_q * (q_heads / kv_heads);
    const int64_t tiles = rows / 128 + n_frames;
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

size_t attention_workspace_bytes(const AttentionPlan &p, int32_t total_q, int32_t q_heads, int32_t dim) {
    if (p.splits <= 1) return 0;
    const size_t all = (size_t)total_q * (size_t)q_heads * (size_t)p.splits;
    return align256(all * (size_t)dim * sizeof(float)) + align256(all * 2 * sizeof(float));
}

hipError_t launch_attention(AttentionArgs a, int32_t dtype, const AttentionPlan &p, void *workspace,
                            hipStream_t stream) {
    a.slots = p.slots;
    a.splits = p.splits;
    if (p.splits > 1) {
        const size_t all = (size_t)a.total_q * (size_t)a.q_heads * (size_t)p.splits;
        a.part_out = static_cast<float *>(workspace);
        a.part_stat = reinterpret_cast<float *>(static_cast<char *>(workspace) + align256(all * (size_t)a.dim * sizeof(float)));
    }
    hipError_t err = with_kernel(a, dtype, [&](auto t, auto dp, auto dist, auto cap) {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        auto go = [&](auto split) {
            constexpr bool SPLIT = decltype(split)::value;
            constexpr size_t bytes = forward_lds_bytes<DP, SPLIT>();
            auto kernel = attention_kernel<T, DP, SPLIT, decltype(dist)::value, decltype(cap)::value>;
            hipLaunchKernelGGL(kernel, dim3((uint32_t)(p.slots * a.kv_heads), (uint32_t)p.splits), dim3(kThreads), bytes,
                               stream, a);
            return hipGetLastError();
        };
        return p.split ? go(std::true_type{}) : go(std::false_type{});
    });
    if (err != hipSuccess || p.splits <= 1) return err;
    const int64_t all = (int64_t)a.total_q * a.q_heads;
    const dim3 grid((uint32_t)((all + 3) / 4));
    if (dtype == FLOCK_F16) hipLaunchKernelGGL(attention_join_kernel<half_t>, grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL(attention_join_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

size_t attention_backward_workspace_bytes(int32_t total_q, int32_t q_heads) {
    const size_t all = (size_t)std::max(total_q, 0) * (size_t)std::max(q_heads, 0);
    return 2 * align256(all * sizeof(float)) + align256((size_t)std::max(q_heads, 0) * kSlopeParts * sizeof(double));
}

hipError_t launch_attention_backward(AttentionBackwardArgs b, int32_t dtype, void *workspace, float *grad_slopes,
                                     hipStream_t stream) {
    AttentionArgs &a = b.fwd;
    const size_t all = (size_t)a.total_q * (size_t)a.q_heads;
    char *ws = static_cast<char *>(workspace);
    b.delta = reinterpret_cast<float *>(ws);
    b.row_slopes = grad_slopes ? reinterpret_cast<float *>(ws + align256(all * sizeof(float))) : nullptr;
    double *parts = reinterpret_cast<double *>(ws + 2 * align256(all * sizeof(float)));
    a.slots = (int64_t)a.total_q * a.group / 128 + a.n_frames;
    b.key_slots = (int64_t)a.total_k / 128 + a.n_frames;
    hipError_t err = hipSuccess;
    if (a.total_q > 0) {
        const dim3 grid((uint32_t)((all + 15) / 16));
        if (dtype == FLOCK_F16) hipLaunchKernelGGL(attention_delta_kernel<half_t>, grid, dim3(kThreads), 0, stream, b);
        else hipLaunchKernelGGL(attention_delta_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, b);
        err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    err = with_kernel(a, dtype, [&](auto t, auto dp, auto dist, auto cap) {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool DIST = decltype(dist)::value, CAP = decltype(cap)::value;
        hipError_t e = hipSuccess;
        if (a.total_q > 0) {
            constexpr size_t bytes = 2 * 64 * (DP + 8) * 2 + 2 * 64 * 4;
            auto kernel = attention_dq_kernel<T, DP, DIST, CAP>;
            hipLaunchKernelGGL(kernel, dim3((uint32_t)(a.slots * a.kv_heads)), dim3(kThreads), bytes, stream, b);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (a.total_k > 0) {
            constexpr size_t bytes = 2 * 64 * (DP + 8) * 2 + 7 * 64 * 4;
            auto kernel = attention_dkv_kernel<T, DP, DIST, CAP>;
            hipLaunchKernelGGL(kernel, dim3((uint32_t)(b.key_slots * a.kv_heads)), dim3(kThreads), bytes, stream, b);
            e = hipGetLastError();
        }
        return e;
    });
    if (err != hipSuccess || !grad_slopes) return err;
    hipLaunchKernelGGL(slope_parts_kernel, dim3(a.q_heads, kSlopeParts), dim3(kThreads), 0, stream, b.row_slopes,
                       (int64_t)a.total_q, a.q_heads, parts);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(slope_total_kernel, dim3(a.q_heads), dim3(64), 0, stream, parts, grad_slopes);
    return hipGetLastError();
}

}  // namespace flock
