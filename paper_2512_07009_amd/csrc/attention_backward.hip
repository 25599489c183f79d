// attention_backward.hip - gradients of attention (the formulas stand in
// attention.hip): two kernels, each summing its own outputs in a fixed order,
// at the price of computing scores and dP twice (seven products for five).

#include "attention_common.h"

namespace flock {
namespace {

using namespace attention;

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
__global__ void __launch_bounds__(kThreads, 2) attention_dq_kernel(AttentionBackwardArgs b) {
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
__global__ void __launch_bounds__(kThreads, DP <= 96 ? 2 : 1) attention_dkv_kernel(AttentionBackwardArgs b) {
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

}  // namespace

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
