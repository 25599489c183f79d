// linear.hip - products of rows in 8 bits with weights in 8 bits, a scale for
// each row and each output:
//
//   y[m, n] = act(x_scale[m] * w_scale[n] * sum_k x[m, k] w[n, k] + bias[n])
//
// Sums are whole numbers of 32 bits on the matrix cores, exact up to a width of
// 2^17 - 1, so they do not depend on their order; what follows is in 32 bits with
// one rounding to the output's type.

#include "encoder_common.h"
#include "linear_common.h"

namespace flock {
namespace {

using namespace linear;

constexpr int kThreads = 256;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// 16 bytes of a row from `k` on, zeros beyond its width.
__device__ __forceinline__ i32x4 load_chunk(const int8_t *row, int k, int width) {
    if (k + 16 <= width) {
        const Pack<int8_t, 16> a = *reinterpret_cast<const Pack<int8_t, 16> *>(row + k);
        return __builtin_bit_cast(i32x4, a);
    }
    i32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int b = 0; b < 16; ++b)
        if (k + b < width) v[b / 4] |= (int)(uint8_t)row[k + b] << (8 * (b % 4));
    return v;
}

// x Phi(x), Phi the normal distribution.  With z = |x| / sqrt 2 and t = 1 / (1 + c z),
// e^(z^2) erfc(z) / t is nearly a polynomial of t (fitted to erfc over z <= 10), so that the
// tail of negative x keeps its digits: 7 terms are off by 9e-7 of it, and with the roundings
// the result by 6.5e-6; 5 by 3.2e-5, and the result by 3.7e-5 against 4.9e-4 and 3.9e-3 for
// half a step of float16 and bfloat16, which get those.  The library's erfc takes some three
// times the instructions, and instructions are what bounds the products that end in it.
template <typename T>
__device__ __forceinline__ float gelu(float x) {
    constexpr bool kShort = sizeof(T) == 2;
    const float z = fminf(fabsf(x), 0x1p60f);  // (infinity times nothing)
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(kShort ? 0.3747665940288702f : 0.36062445840513924f, z, 1.0f));
    float p;
    if constexpr (kShort) {
        p = -0.09049928f;
        p = __builtin_fmaf(p, t, 0.20043353f);
        p = __builtin_fmaf(p, t, 0.08345564f);
        p = __builtin_fmaf(p, t, 0.15764168f);
        p = __builtin_fmaf(p, t, 0.14896917f);
    } else {
        p = 0.047249945f;
        p = __builtin_fmaf(p, t, -0.1795673f);
        p = __builtin_fmaf(p, t, 0.17922265f);
        p = __builtin_fmaf(p, t, 0.027526545f);
        p = __builtin_fmaf(p, t, 0.13953302f);
        p = __builtin_fmaf(p, t, 0.142076165f);
        p = __builtin_fmaf(p, t, 0.14395875f);
    }
    const float tail = p * t * __builtin_amdgcn_exp2f(x * x * -0.72134752044448170368f);  // 1 - Phi(|x|)
    return __builtin_fmaf(-z, tail, fmaxf(x, 0.0f));
}

// ---------------------------------------------------------------------------
// Many rows: BM x BN outputs a tile, a quarter of them a wave.
//
// The weights are the left factor (32 outputs), the rows the right one (32 rows),
// so that a lane holds four outputs of one row side by side; halves of a wave trade
// fours for eights, and each lane stores 16 bytes of a row.
//
// Tiles of kStep bytes of every row go to LDS without registers in between (16 bytes
// a lane).  A row's chunks of 16 bytes are stored in an order that turns with the row,
// so that the 32 rows that a wave reads a chunk of lie in different banks.
//
// A workgroup stays for many tiles, and its steps are one stream: loads run a step
// before the products, across the ends of tiles, and a step waits for its own loads
// alone (they come back in order), with one barrier a step.
//
// Two workgroups of four waves a compute unit make 128 x 128 outputs each, and one's
// outputs are made beside the other's products: 40000 rows of 2048 to 512 outputs 52 us
// (1.6 POP/s, of 2.1 of a product of 8192^3 by the library).  What bounds it are the loads
// to LDS and the outputs' stores (128000 x 512 to 1536, 172 us: without stores 143,
// without making outputs 109, loads alone 106); steps of 64 bytes take half a line of a
// row each (8192^3 609 -> 720 us).  Fewer than two tiles of 128 x 128 a compute unit are
// made as tiles of 64 x 64 by four workgroups (500 rows to 1536 5.6 us).
// ---------------------------------------------------------------------------

__device__ const __attribute__((aligned(16))) int8_t kZeros[16] = {};

__device__ __forceinline__ int turned(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

#define FLOCK_TO_LDS(FROM, TO, SIZE)                                                                  \
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(FROM),         \
                                     (__attribute__((address_space(3))) void *)(TO), SIZE, 0, 0)

// Where a tile's rows begin, for the loads or for the products.
template <int BM, int BN>
struct LinearTile {
    int64_t m0;
    int n0, rows, columns;
    __device__ __forceinline__ LinearTile(const LinearArgs &a, uint32_t tile) {
        const uint32_t row = tile / (uint32_t)a.column_tiles;
        m0 = (int64_t)row * BM;
        n0 = (int)(tile - row * a.column_tiles) * BN;
        rows = (int)min((int64_t)BM, a.rows - m0);
        columns = min(BN, a.outputs - n0);
    }
};

// The loads' side of the stream.
template <int BM, int BN, int THREADS = 256>
struct LinearLoads {
    static constexpr int kThreads = THREADS, kX = BM * kChunks / THREADS, kW = BN * kChunks / THREADS, kLoads = kX + kW;
    const int8_t *x, *w;          // the tile's first rows
    uint32_t x_at[kX], w_at[kW];  // the lane's chunks, from them
    int wave;

    __device__ __forceinline__ LinearLoads() { wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

    template <typename S>
    __device__ __forceinline__ void begin(const LinearArgs &a, uint32_t tile, int turn, S &s) {
        const LinearTile<BM, BN> t(a, tile);
        x = a.x + t.m0 * a.x_stride;
        w = a.w + t.n0 * a.w_stride;
        // (rows beyond the last are the last: what they give is not stored)
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const int slot = i * kThreads + threadIdx.x, row = slot / kChunks;
            x_at[i] = (uint32_t)min(row, t.rows - 1) * (uint32_t)a.x_stride + 16u * turned(row, slot % kChunks);
        }
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            const int slot = i * kThreads + threadIdx.x, row = slot / kChunks;
            w_at[i] = (uint32_t)min(row, t.columns - 1) * (uint32_t)a.w_stride + 16u * turned(row, slot % kChunks);
        }
        // the scales and the bias: a load of 64 of each a wave, where there are so many
        const int lane = threadIdx.x & 63, part = 64 * wave;
        if (part < BM) FLOCK_TO_LDS(a.x_scale + t.m0 + min(part + lane, t.rows - 1), s.x_scale[turn] + part, 4);
        if (part < BN) {
            const int n = t.n0 + min(part + lane, t.columns - 1);
            FLOCK_TO_LDS(a.w_scale + n, s.w_scale[turn] + part, 4);
            FLOCK_TO_LDS(a.bias ? static_cast<const void *>(a.bias + n) : kZeros, s.bias[turn] + part, 4);
        }
    }

    __device__ __forceinline__ void step(int k0, int width, int8_t *xs, int8_t *ws) const {
        if (k0 + kStep <= width) {
#pragma unroll
            for (int i = 0; i < kX; ++i) FLOCK_TO_LDS(x + k0 + x_at[i], xs + 16 * (i * kThreads + 64 * wave), 16);
#pragma unroll
            for (int i = 0; i < kW; ++i) FLOCK_TO_LDS(w + k0 + w_at[i], ws + 16 * (i * kThreads + 64 * wave), 16);
            return;
        }
        // the row's end: no chunks beyond it, of the weights zeros instead
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const int slot = i * kThreads + threadIdx.x, c = 16 * turned(slot / kChunks, slot % kChunks);
            FLOCK_TO_LDS(x + (k0 + c < width ? k0 + x_at[i] : x_at[i] - c), xs + 16 * (i * kThreads + 64 * wave), 16);
        }
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            const int slot = i * kThreads + threadIdx.x, c = 16 * turned(slot / kChunks, slot % kChunks);
            FLOCK_TO_LDS(k0 + c < width ? w + k0 + w_at[i] : kZeros, ws + 16 * (i * kThreads + 64 * wave), 16);
        }
    }

    // Zeros for the weights' bytes beyond the width in a chunk that it ends in.
    __device__ __forceinline__ void mask(int k0, int width, int8_t *ws) const {
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            const int slot = i * kThreads + threadIdx.x, left = width - k0 - 16 * turned(slot / kChunks, slot % kChunks);
            if (left > 0 && left < 16) {
                i32x4 v = *reinterpret_cast<i32x4 *>(ws + 16 * slot);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int bytes = min(max(left - 4 * e, 0), 4);
                    v[e] = bytes == 4 ? v[e] : v[e] & ((1 << (8 * bytes)) - 1);
                }
                *reinterpret_cast<i32x4 *>(ws + 16 * slot) = v;
            }
        }
    }
};

// One step of a wave: its rows' and outputs' chunks from LDS.  (Loads go to another
// stage, and the compiler is told so.)
template <int KM, int KN>
__device__ __forceinline__ void multiply(const int8_t *__restrict__ x, const int8_t *__restrict__ w, i32x16 (&acc)[KN][KM]) {
    const int lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    constexpr int kParts = kStep / 32;
    i32x4 wf[kParts][KN], xf[kParts][KM];
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
#pragma unroll
        for (int i = 0; i < KN; ++i)
            wf[k][i] = *reinterpret_cast<const i32x4 *>(w + (32 * i + col) * kStep + 16 * turned(col, 2 * k + h));
#pragma unroll
        for (int j = 0; j < KM; ++j)
            xf[k][j] = *reinterpret_cast<const i32x4 *>(x + (32 * j + col) * kStep + 16 * turned(col, 2 * k + h));
    }
    // (all of a step's factors are on their way before the first product)
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
        for (int i = 0; i < KN; ++i)
#pragma unroll
            for (int j = 0; j < KM; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[k][i], xf[k][j], acc[i][j], 0, 0, 0);
}

// Four outputs and four others of a lane's row, 8 on, for eight side by side: the first
// eight of sixteen in the lower half of the wave, the others in the upper.
template <typename T>
__device__ __forceinline__ Pack<T, 8> side_by_side(const float (&o)[8]) {
    Pack<T, 8> out;
    if constexpr (sizeof(T) == 2) {
        Pack<T, 8> mine;
#pragma unroll
        for (int e = 0; e < 8; ++e) mine.v[e] = static_cast<T>(o[e]);
        const i32x4 v = __builtin_bit_cast(i32x4, mine);
        const auto p = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
        const auto q = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
        const i32x4 u = {(int)p[0], (int)q[0], (int)p[1], (int)q[1]};
        out = __builtin_bit_cast(Pack<T, 8>, u);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[e]), __float_as_uint(o[e + 4]), false, false);
            out.v[e] = static_cast<T>(__uint_as_float(p[0]));
            out.v[e + 4] = static_cast<T>(__uint_as_float(p[1]));
        }
    }
    return out;
}

// A pack of 16 bytes to LDS, where it begins at a multiple of them.
template <typename T>
__device__ __forceinline__ void put(Pack<T, 8> *at, const Pack<T, 8> &v) {
    if constexpr (sizeof(v) == 16) *reinterpret_cast<i32x4 *>(__builtin_assume_aligned(at, 16)) = __builtin_bit_cast(i32x4, v);
}

// The first `left` of a pack, all of it where FULL.
template <bool FULL, typename T>
__device__ __forceinline__ void store_left(T *y, const Pack<T, 8> &v, int left) {
    if (FULL || left >= 8) {
        // (past the caches, which large outputs have no use of: 128000 x 512 to 1536 210 -> 174 us)
        typedef i32x4 __attribute__((aligned(2))) Words;
        const Words *from = reinterpret_cast<const Words *>(&v);
        Words *to = reinterpret_cast<Words *>(y);
#pragma unroll
        for (int e = 0; e < (int)sizeof(v) / 16; ++e) __builtin_nontemporal_store(from[e], to + e);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < left) y[e] = v.v[e];
}

// The compiler moves no access to memory over this.
__device__ __forceinline__ void stand() { asm volatile("" ::: "memory"); }

// A wave's outputs of a tile.  FULL: all of its rows and outputs are there.  Outputs of
// 16 bits go through LDS (`room`, kRoom<KN> bytes of the wave's own), 32 rows at a time, so that a
// row's are stored as 64 KN bytes in one piece: with stores of the 32 bytes that a lane
// has beside each other 128000 x 512 to 1536 took 233 us, 95 of them for stores.
template <typename T, bool GELU, bool FULL, int KM, int KN, typename S, typename Tile>
__device__ __forceinline__ void finish(const LinearArgs &a, const Tile &t, const S &s, int turn, int wm, int wn, int8_t *room,
                                       const i32x16 (&acc)[KN][KM]) {
    constexpr bool kStaged = sizeof(T) == 2;
    constexpr int kParts = 4 * KN;  // of 8 outputs, a row
    const int lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const auto part_at = [](int row, int part) { return row * kParts + (part ^ (KN == 2 ? row & 7 : (row >> 1) & 3)); };
    Pack<T, 8> *stage = reinterpret_cast<Pack<T, 8> *>(room);
    T *y = static_cast<T *>(a.y) + (t.m0 + wm) * a.y_stride + t.n0 + wn;
#pragma unroll
    for (int j = 0; j < KM; ++j) {
        const float xs = s.x_scale[turn][wm + 32 * j + col];
#pragma unroll
        for (int i = 0; i < KN; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                // outputs n .. n + 3 and n + 8 .. n + 11 of the lane's row
                const int n = wn + 32 * i + 2 * r + 4 * h;
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = n + (e & 3) + 8 * (e >> 2);
                    o[e] = (float)acc[i][j][r + e] * xs * s.w_scale[turn][at] + s.bias[turn][at];
                    if (GELU) o[e] = gelu<T>(o[e]);
                }
                const Pack<T, 8> out = side_by_side<T>(o);
                const int part = 4 * i + r / 4 + h;
                if (kStaged) put(stage + part_at(col, part), out);
                else if (FULL || wm + 32 * j + col < t.rows)
                    store_left<FULL>(y + (int64_t)(32 * j + col) * a.y_stride + 8 * part, out, t.columns - wn - 8 * part);
            }
        if (!kStaged) continue;
        stand();
#pragma unroll
        for (int i = 0; i < kParts / 2; ++i) {
            const int row = (64 * i + lane) / kParts, part = lane % kParts;
            const Pack<T, 8> out = stage[part_at(row, part)];
            if (FULL || wm + 32 * j + row < t.rows)
                store_left<FULL>(y + (int64_t)(32 * j + row) * a.y_stride + 8 * part, out, t.columns - wn - 8 * part);
        }
        stand();
    }
}

// Waits for LDS, and for all but the last N loads and stores.
template <int N>
__device__ __forceinline__ void wait_but() {
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x070);
}

template <typename T, bool GELU, int BM, int BN>
__global__ void __launch_bounds__(kThreads, 2) linear_kernel(LinearArgs a) {
    constexpr int kMT = BM / 64, kNT = BN / 64;      // 32 x 32 parts of a wave
    constexpr int kLoads = LinearLoads<BM, BN>::kLoads;
    __shared__ LinearShared<BM, BN> s;

    // tiles of this workgroup: an eighth of all to each XCD, in one piece, its workgroups side by side
    uint32_t first, end, beside = 1;
    const uint32_t tiles = a.tiles;
    if (tiles <= gridDim.x) {  // one each
        const uint32_t per = tiles / 8, id = blockIdx.x;
        first = id < per * 8 ? (id & 7) * per + (id >> 3) : id;
        end = first + 1;
    } else {                     // (as many workgroups on each XCD)
        const uint32_t xcd = blockIdx.x & 7;
        beside = gridDim.x >> 3;
        first = tiles * xcd / 8 + (blockIdx.x >> 3);
        end = tiles * (xcd + 1) / 8;
        if (first >= end) return;
    }
    const int steps = (a.width + kStep - 1) / kStep;
    int64_t left = (int64_t)((end - first - 1) / beside + 1) * steps;  // steps to multiply

    LinearLoads<BM, BN> loads;
    uint32_t next_tile = first;
    int next_step = 0, next_turn = 0, next_stage = 0;
    const auto load = [&] {
        if (next_tile >= end) return;
        if (next_step == 0) loads.begin(a, next_tile, next_turn, s);
        loads.step(next_step * kStep, a.width, s.x[next_stage], s.w[next_stage]);
        next_stage = (next_stage + 1) & (kStages - 1);
        if (++next_step == steps) {
            next_step = 0;
            next_tile += beside;
            next_turn = (next_turn + 1) & (kStages - 1);
        }
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load();

    const int wave = threadIdx.x >> 6, wm = (wave & 1) * (BM / 2), wn = (wave >> 1) * (BN / 2);
    // a whole tile's stores, at least; they come between the loads of kAhead steps, which need not wait for them
    constexpr int kStores = 2 * kMT * kNT;
    int stage = 0, turn = 0, since = kAhead;
    for (uint32_t tile = first; tile < end; tile += beside, turn = (turn + 1) & (kStages - 1)) {
        i32x16 acc[kNT][kMT] = {};
        // (a wave that multiplies goes before the one beside it that has a tile's outputs to make: 2 to 4%)
        __builtin_amdgcn_s_setprio(2);
        for (int t = 0; t < steps; ++t) {
            // this step's loads are all but the last of the steps after it (a tile's first step has more of them)
            stand();
            if (left < kAhead) wait_but<0>();
            else if (since < kAhead) wait_but<(kAhead - 1) * kLoads + kStores>();
            else wait_but<(kAhead - 1) * kLoads>();
            ++since;
            stand();
            if (a.width % 16 && t == steps - 1) {
                loads.mask(t * kStep, a.width, s.w[stage]);
                stand();
                __builtin_amdgcn_s_waitcnt(0xc07f);  // (LDS)
            }
            __builtin_amdgcn_s_barrier();  // ... of all waves, and the stage before has been read by all
            stand();
            load();
            multiply<kMT, kNT>(s.x[stage] + wm * kStep, s.w[stage] + wn * kStep, acc);
            stage = (stage + 1) & (kStages - 1);
            --left;
        }
        // the stage that was multiplied last is free until the next step's barrier
        __builtin_amdgcn_s_setprio(0);
        const int last = (stage + kStages - 1) & (kStages - 1);
        int8_t *room = stage_room<kNT>(s, last, wave);
        stand();
        __builtin_amdgcn_s_waitcnt(0xc07f);  // (LDS)
        __builtin_amdgcn_s_barrier();
        stand();
        const LinearTile<BM, BN> t(a, tile);
        if (t.rows == BM && t.columns == BN) {
            finish<T, GELU, true>(a, t, s, turn, wm, wn, room, acc);
            since = 0;
        } else {
            finish<T, GELU, false>(a, t, s, turn, wm, wn, room, acc);
        }
    }
}

// Rows that begin anywhere: 64 x 64 outputs a workgroup, chunks through registers, one
// step at a time.
template <typename T>
__global__ void __launch_bounds__(kThreads) linear_any_kernel(LinearArgs a) {
    constexpr int B = 64;
    __shared__ LinearShared<B, B> s;
    const LinearTile<B, B> t(a, blockIdx.x);
    if (threadIdx.x < B) {
        const int m = min((int)threadIdx.x, t.rows - 1), n = t.n0 + min((int)threadIdx.x, t.columns - 1);
        s.x_scale[0][threadIdx.x] = a.x_scale[t.m0 + m];
        s.w_scale[0][threadIdx.x] = a.w_scale[n];
        s.bias[0][threadIdx.x] = a.bias ? a.bias[n] : 0.0f;
    }
    const int wave = threadIdx.x >> 6, wm = (wave & 1) * (B / 2), wn = (wave >> 1) * (B / 2);
    i32x16 acc[1][1] = {};
    for (int k0 = 0; k0 < a.width; k0 += kStep) {
        i32x4 xv[B * kChunks / kThreads], wv[B * kChunks / kThreads];
#pragma unroll
        for (int i = 0; i < B * kChunks / kThreads; ++i) {
            const int slot = i * kThreads + threadIdx.x, row = slot / kChunks, k = k0 + 16 * turned(row, slot % kChunks);
            xv[i] = load_chunk(a.x + (t.m0 + min(row, t.rows - 1)) * a.x_stride, k, a.width);
            wv[i] = load_chunk(a.w + (t.n0 + min(row, t.columns - 1)) * a.w_stride, k, a.width);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < B * kChunks / kThreads; ++i) {
            *reinterpret_cast<i32x4 *>(s.x[0] + 16 * (i * kThreads + threadIdx.x)) = xv[i];
            *reinterpret_cast<i32x4 *>(s.w[0] + 16 * (i * kThreads + threadIdx.x)) = wv[i];
        }
        __syncthreads();
        multiply<1, 1>(s.x[0] + wm * kStep, s.w[0] + wn * kStep, acc);
    }
    int8_t *room = stage_room<1>(s, 1, wave);  // (the first stage may still be read by other waves, the second has no use)
    if (a.gelu) finish<T, true, false>(a, t, s, 0, wm, wn, room, acc);
    else finish<T, false, false>(a, t, s, 0, wm, wn, room, acc);
}

// Outputs of 16 bits of a wave's 32 rows, 64 of each, by way of LDS (`room`, 2 KB of the
// wave's own), 16 rows at a time, in pieces of 128 bytes.  FULL: all of them are there, of
// others the first `rows` and `here`.  Rows that begin inside 64 bytes (not LINES) go
// through the caches, which join their parts (30001 x 2047 to 501 51 -> 42 us, 40 between
// other work).  Places in
// LDS are made here, not kept: registers are full where this is called.
template <bool FULL, bool LINES, bool GELU, typename T>
__device__ __forceinline__ void make_64(T *y, int64_t y_stride, int rows, int here, Pack<T, 8> *room,
                                        const float *w_scale, const float *bias, float scale, const i32x16 &first,
                                        const i32x16 &second) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int h = lane >> 5, col = lane & 31;
    const auto part_at = [](int row, int part) { return row * 8 + (part ^ (row & 7)); };
    Pack<T, 8> out[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int at = 16 * u + 4 * h + (e & 3) + 8 * (e >> 2);
            o[e] = (float)(u < 2 ? first : second)[8 * (u & 1) + e] * scale * w_scale[at] + bias[at];
            if (GELU) o[e] = gelu<T>(o[e]);
        }
        out[u] = side_by_side<T>(o);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        stand();
        if (col >> 4 == half) {
#pragma unroll
            for (int u = 0; u < 4; ++u) put(room + part_at(col & 15, 2 * u + h), out[u]);
        }
        stand();
        if (FULL) {
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int row = lane / 8, part = lane & 7;
                T *to = y + (16 * half + 8 * v) * y_stride + ((uint32_t)row * (uint32_t)y_stride + 8 * part);
                const Pack<T, 8> all = room[part_at(8 * v + row, part)];
                if constexpr (LINES) store_left<true>(to, all, 8);
                else *reinterpret_cast<Pack<T, 8> *>(to) = all;
            }
        } else if (lane < here) {
#pragma unroll 1
            for (int row = 0; row < min(16, rows - 16 * half); ++row)
                y[(16 * half + row) * y_stride + lane] = room[part_at(row, lane / 8)].v[lane & 7];
        }
    }
    stand();
}

// ---------------------------------------------------------------------------
// Many rows: 256 x 256 outputs a workgroup of eight waves, 64 x 128 a wave.
//
// The same steps and loads as above, with half the bytes to LDS and three quarters of
// those from it for a product, and nothing beside the workgroup on its compute unit, so
// that a wave reads the next factors from LDS under the products of these, the next
// step's first ones too: the barrier is before a step's last products, when all of its
// factors have been read.  8192^3 567 us (1.9 POP/s), 128000 rows of 2048 to 512 150
// (1.8), without that 600 and 152.
// ---------------------------------------------------------------------------

constexpr int kWide = 256, kWideThreads = 512;

struct __attribute__((aligned(16))) WideShared {
    int8_t x[2][kWide * kStep], w[2][kWide * kStep];
    float x_scale[2][kWide], w_scale[2][kWide], bias[2][kWide];  // of tiles in turn (a tile is two steps or more)
    int8_t room[kWideThreads / 64][16 * 64 * 2];
};

template <typename T, bool GELU, bool LINES>
__global__ void __launch_bounds__(kWideThreads, 2) linear_wide_kernel(LinearArgs a) {
    using Loads = LinearLoads<kWide, kWide, kWideThreads>;
    constexpr int kMT = 2, kNT = 4, kParts = kStep / 32;
    __shared__ WideShared s;

    const uint32_t tiles = a.tiles, id = blockIdx.x, per = tiles / 8;
    uint32_t tile, end, beside = 1;
    if (tiles <= gridDim.x) {  // one each, an eighth of all beside each other on each XCD
        tile = id < per * 8 ? (id & 7) * per + (id >> 3) : id;
        end = tile + 1;
    } else {
        const uint32_t xcd = id & 7;
        beside = gridDim.x >> 3;
        tile = tiles * xcd / 8 + (id >> 3);
        end = tiles * (xcd + 1) / 8;
        if (tile >= end) return;
    }
    const int steps = (a.width + kStep - 1) / kStep;
    int64_t left = (int64_t)((end - tile - 1) / beside + 1) * steps;  // steps to multiply

    Loads loads;
    uint32_t next_tile = tile;
    int next_step = 0, next_turn = 0, next_stage = 0;
    const auto load = [&] {
        if (next_tile >= end) return;
        if (next_step == 0) loads.begin(a, next_tile, next_turn, s);
        loads.step(next_step * kStep, a.width, s.x[next_stage], s.w[next_stage]);
        next_stage ^= 1;
        if (++next_step == steps) {
            next_step = 0;
            next_tile += beside;
            next_turn ^= 1;
        }
    };
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    const int wm = (wave & 3) * 64, wn = (wave >> 2) * 128;
    i32x4 wf[2][kNT], xf[2][kMT];
    const auto read = [&](int to, int stage, int k) {
        const int chunk = 16 * turned(col, 2 * k + h) + col * kStep;
#pragma unroll
        for (int i = 0; i < kNT; ++i) wf[to][i] = *reinterpret_cast<const i32x4 *>(s.w[stage] + (wn + 32 * i) * kStep + chunk);
#pragma unroll
        for (int j = 0; j < kMT; ++j) xf[to][j] = *reinterpret_cast<const i32x4 *>(s.x[stage] + (wm + 32 * j) * kStep + chunk);
    };
    const auto arrive = [&](int stage, bool last) {  // the waits are the caller's
        stand();
        if (a.width % 16 && last) {
            loads.mask((steps - 1) * kStep, a.width, s.w[stage]);
            stand();
            __builtin_amdgcn_s_waitcnt(0xc07f);  // (LDS)
        }
        __builtin_amdgcn_s_barrier();
        stand();
    };

    load();
    wait_but<0>();
    arrive(0, false);
    load();
    read(0, 0, 0);
    constexpr int kStores = 16;  // of a whole tile, a wave
    int stage = 0, turn = 0, since = 1;
    for (; tile < end; tile += beside, turn ^= 1) {
        i32x16 acc[kNT][kMT] = {};
        const auto multiply = [&](int from) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kNT; ++i)
#pragma unroll
                for (int j = 0; j < kMT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[from][i], xf[from][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int t = 0; t < steps; ++t) {
#pragma unroll
            for (int k = 0; k + 1 < kParts; ++k) {
                read((k + 1) & 1, stage, k + 1);
                multiply(k & 1);
            }
            if (--left > 0) {
                // the next step's loads (a whole tile's stores came after them, in a tile's first step)
                stand();
                if (since == 0) wait_but<kStores>();
                else wait_but<0>();
                ++since;
                arrive(stage ^ 1, (t + 1 == steps ? 0 : t + 1) == steps - 1);
                load();
                read(0, stage ^ 1, 0);
            }
            multiply((kParts - 1) & 1);
            stage ^= 1;
        }
        const LinearTile<kWide, kWide> at(a, tile);
        Pack<T, 8> *room = reinterpret_cast<Pack<T, 8> *>(s.room[wave]);
        const auto finish = [&](auto full) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < kMT; ++j)
#pragma unroll
                for (int i = 0; i < kNT; i += 2) {
                    const int m = wm + 32 * j, n = wn + 32 * i, rows = at.rows - m, here = at.columns - n;
                    const auto make = [&](auto all) __attribute__((always_inline)) {
                        make_64<decltype(all)::value, LINES, GELU>(static_cast<T *>(a.y) + (at.m0 + m) * a.y_stride + at.n0 + n,
                                                                   a.y_stride, rows, here, room, s.w_scale[turn] + n,
                                                                   s.bias[turn] + n, s.x_scale[turn][m + col], acc[i][j],
                                                                   acc[i + 1][j]);
                    };
                    if (decltype(full)::value || (rows >= 32 && here >= 64)) make(std::true_type{});
                    else if (rows > 0 && here > 0) make(std::false_type{});
                }
        };
        if (at.rows == kWide && at.columns == kWide) {
            finish(std::true_type{});
            since = 0;
        } else {
            finish(std::false_type{});
        }
    }
}

// ---------------------------------------------------------------------------
// Very many rows of a width that fits: the weights stay.
//
// A workgroup keeps the weights of 256 outputs in LDS (128 KB) and takes rows, 32 at a
// time and wave: their bytes go from memory to the wave's registers as factors, the next
// rows' while this one's last outputs are made.  Waves wait for their own loads alone, so
// that one's products run beside another's outputs and stores.  The workgroups of all
// outputs of the same rows run side by side on one XCD, whose L2 then serves them.
// Twelve waves are what registers allow, and one workgroup: two of six waves and half
// the weights each lie three and three on two units of four, and do not fit together.
// ---------------------------------------------------------------------------

constexpr int kStayWidth = 512, kStayWaves = 12, kStayOutputs = 256, kStayHalf = 128;

struct __attribute__((aligned(16))) StayShared {
    float w_scale[kStayOutputs], bias[kStayOutputs];
    int8_t room[kStayWaves][16 * 64 * 2];  // 16 rows of 64 outputs
    int8_t w[kStayOutputs / kStayHalf][kStayWidth / kStep][kStayHalf * kStep];
};

template <typename T, bool GELU>
__global__ void __launch_bounds__(64 * kStayWaves) linear_stay_kernel(LinearArgs a) {
    constexpr int kBlocks = kStayHalf / 32, kParts = kStayWidth / 32;
    __shared__ StayShared s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    // this workgroup's outputs and rows
    const int per_xcd = (int)(gridDim.x >> 3), groups = per_xcd / a.column_tiles;
    const int xcd = blockIdx.x & 7, at = (int)(blockIdx.x >> 3), group = at / a.column_tiles;
    if (group >= groups) return;
    const int n0 = (at - group * a.column_tiles) * kStayOutputs, columns = min(kStayOutputs, a.outputs - n0);
    const int64_t tiles = a.tiles, end = tiles * (xcd + 1) / 8;
    // (the last turn, which some waves are without, is then as short for every workgroup: 136 -> 129 us to 1536)
    int64_t tile = tiles * xcd / 8 + wave * groups + group;

    const int8_t *w = a.w + n0 * (int64_t)a.w_stride;
    for (int i = wave; i < kStayWidth / kStep * kStayOutputs * kChunks / 64; i += kStayWaves) {
        const int slot = i * 64 + lane, row = slot / kChunks % kStayHalf, step = slot / (kStayHalf * kChunks);
        const int k = step % (kStayWidth / kStep) * kStep + 16 * turned(row, slot % kChunks);
        const int n = row + step / (kStayWidth / kStep) * kStayHalf;
        i32x4 v = {0, 0, 0, 0};
        if (k < a.width) v = load_chunk(w + (int64_t)min(n, columns - 1) * a.w_stride, k, a.width);
        *reinterpret_cast<i32x4 *>(s.w[0][0] + 16 * slot) = v;
    }
    for (int i = threadIdx.x; i < kStayOutputs; i += 64 * kStayWaves) {
        const int n = n0 + min(i, columns - 1);
        s.w_scale[i] = a.w_scale[n];
        s.bias[i] = a.bias ? a.bias[n] : 0.0f;
    }
    __syncthreads();
    if (tile >= end) return;

    i32x4 x[kParts];
    float xs;
    // a half of the next rows' chunks (rows beyond the last are the last; chunks beyond the width any bytes of
    // the row, the weights are zeros there)
    const auto load = [&](int64_t tile, int half) {
        const int64_t row0 = tile * 32;
        const uint32_t row = (uint32_t)min((int64_t)col, a.rows - 1 - row0), first = row * (uint32_t)a.x_stride;
        uint32_t at = first + 16 * h;
        asm volatile("" : "+v"(at));  // (not 16 places kept)
        const int8_t *from = a.x + row0 * a.x_stride;
        if (half == 0) xs = (a.x_scale + row0)[row];
#pragma unroll
        for (int k = half * kParts / 2; k < (half + 1) * kParts / 2; ++k)
            x[k] = *reinterpret_cast<const i32x4 *>(from + (32 * k < a.width ? 32 * k : 0) + (32 * k + 16 < a.width ? at : first));
    };
    Pack<T, 8> *room = reinterpret_cast<Pack<T, 8> *>(s.room[wave]);
    const auto make = [&](auto full, int n1, auto block, int64_t row0, const i32x16 (&acc)[kBlocks], float scale) __attribute__((always_inline)) {
        constexpr int i = decltype(block)::value;
        const int n = n1 + 32 * i;
        make_64<decltype(full)::value, true, GELU>(static_cast<T *>(a.y) + row0 * a.y_stride + n0 + n, a.y_stride,
                                                   (int)min((int64_t)32, a.rows - row0), columns - n, room,
                                                   s.w_scale + n, s.bias + n, scale, acc[i], acc[i + 1]);
    };

    const auto multiply = [&](int half, i32x16 (&acc)[kBlocks]) __attribute__((always_inline)) {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));
        const int h = lane >> 5, col = lane & 31;
        __builtin_amdgcn_s_setprio(2);
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            i32x4 wf[kBlocks];
#pragma unroll
            for (int i = 0; i < kBlocks; ++i)
                wf[i] = *reinterpret_cast<const i32x4 *>(s.w[half][k / 4] + (32 * i + col) * kStep + 16 * turned(col, 2 * (k % 4) + h));
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) acc[i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[i], x[k], acc[i], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    constexpr std::integral_constant<int, 0> kFirst;
    constexpr std::integral_constant<int, 2> kSecond;
    // rows up to a tile, all of whose rows and outputs are there where FULL; nothing branches
    // there, so that a wait for rows is for those alone and not for stores
    const auto go = [&](auto full, int64_t last) __attribute__((always_inline)) {
        while (tile < last) {
            const int64_t row0 = tile * 32;
            const float scale = xs;
            {
                i32x16 acc[kBlocks] = {};
                multiply(0, acc);
                stand();
                make(full, 0, kFirst, row0, acc, scale);
                make(full, 0, kSecond, row0, acc, scale);
            }
            i32x16 acc[kBlocks] = {};
            multiply(1, acc);
            tile += groups * kStayWaves;
            // (the second half of the next rows when there is room for it)
            stand();
            load(min(tile, end - 1), 0);
            stand();
            make(full, kStayHalf, kFirst, row0, acc, scale);
            stand();
            load(min(tile, end - 1), 1);
            stand();
            make(full, kStayHalf, kSecond, row0, acc, scale);
        }
    };
    load(tile, 0);
    load(tile, 1);
    wait_but<0>();  // (so that the loop's waits are those of its later turns)
    if (columns == kStayOutputs) go(std::true_type{}, min(end, a.rows / 32));
    go(std::false_type{}, end);
}

// ---------------------------------------------------------------------------
// Few rows: the weights are what is read, so a workgroup takes 16 outputs and its
// eight waves share the width, 256 bytes of each output a wave and turn (a lane 64
// of them in four loads).  Factors go from memory to the matrix cores as they are:
// both sides take their bytes in the same order, and that order is free.  The
// waves' sums are joined in LDS.  7 rows of 2048 to 512 outputs 4.4 us: the time of a
// load, the joint and a store, one after the other, of 1 MB.
// ---------------------------------------------------------------------------

constexpr int kFewWaves = 8;

template <typename T, int MT>
__global__ void __launch_bounds__(64 * kFewWaves) linear_few_kernel(LinearArgs a) {
    __shared__ int sums[kFewWaves][MT][16][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, part = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const int8_t *w = a.w + (int64_t)min(n0 + row, a.outputs - 1) * a.w_stride;
    const int8_t *x[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) x[j] = a.x + min((int64_t)(16 * j + row), a.rows - 1) * a.x_stride;
    i32x4 acc[MT] = {};
    for (int k0 = wave * 256; k0 < a.width; k0 += 256 * kFewWaves) {
        i32x4 wf[4], xf[MT][4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k = k0 + 64 * s + 16 * part;
            wf[s] = load_chunk(w, k, a.width);
#pragma unroll
            for (int j = 0; j < MT; ++j) xf[j][s] = load_chunk(x[j], k, a.width);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[s], xf[j][s], acc[j], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][j][row][4 * part + r] = acc[j][r];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 256; i += 64 * kFewWaves) {
        const int n = i & 15, m = i >> 4;
        if (m >= a.rows || n0 + n >= a.outputs) continue;
        int total = 0;
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) total += sums[v][m >> 4][m & 15][n];
        float o = (float)total * a.x_scale[m] * a.w_scale[n0 + n] + (a.bias ? a.bias[n0 + n] : 0.0f);
        if (a.gelu) o = gelu<T>(o);
        static_cast<T *>(a.y)[m * a.y_stride + n0 + n] = static_cast<T>(o);
    }
}

// launch(part) over the rows of a, by as many as `most` tiles hold.
template <typename T, int BM, int BN, typename F>
hipError_t by_tiles(LinearArgs a, F &&launch) {
    a.column_tiles = (a.outputs + BN - 1) / BN;
    const int64_t rows = a.rows, most = kMaxWorkgroups / a.column_tiles * BM;
    hipError_t err = hipSuccess;
    for (int64_t first = 0; first < rows && err == hipSuccess; first += most) {
        LinearArgs part = a;
        part.rows = std::min(rows - first, most);
        part.advance(first, sizeof(T));
        part.tiles = (part.rows + BM - 1) / BM * a.column_tiles;
        launch(part);
        err = hipGetLastError();
    }
    return err;
}

template <typename T, int BM, int BN>
hipError_t launch_tiles(const LinearArgs &a, int per_cu, int n_cus, hipStream_t stream) {
    const int64_t workgroups = std::max(per_cu * n_cus / 8 * 8, 8);

    return by_tiles<T, BM, BN>(a, [&](const LinearArgs &part) {
        const dim3 grid((uint32_t)std::min(part.tiles, workgroups));
        if (a.gelu) hipLaunchKernelGGL((linear_kernel<T, true, BM, BN>), grid, dim3(kThreads), 0, stream, part);
        else hipLaunchKernelGGL((linear_kernel<T, false, BM, BN>), grid, dim3(kThreads), 0, stream, part);
    });
}

// Whether outputs of `y` begin at a multiple of 64 bytes, each row of them.
template <typename T>
bool whole_lines(const LinearArgs &a) {
    return a.y_stride * sizeof(T) % 64 == 0 && reinterpret_cast<uintptr_t>(a.y) % 64 == 0;
}

// Workgroups that keep their weights, one a compute unit and an eighth of them on each XCD;
// 0 where tiles of 128 x 128 are as fast.  128000 rows of 512 to 1536 outputs 172 -> 129 us,
// to 2048 237 -> 165, with gelu 357 -> 260; 8 waves a compute unit beside each other make
// those tiles, 12 here, and they copy rows to LDS for every 128 outputs.  What bounds it is
// no one thing (without gelu vector instructions take 38% of the time, matrix cores 40,
// LDS 43), but with gelu vector instructions, 80%.
// - Narrower rows leave factors empty: 256 wide 148 -> 158 us, 320 188 -> 166.
// - Workgroups that outputs do not divide among have nothing.
// - With fewer than two turns a wave loading the weights is not paid back: 16000 rows
//   to 2048 29 -> 34 us, 25000 46 -> 39.
// - Rows of outputs that begin inside 64 bytes are written in parts (pitch 1544: 180 -> 301 us).
template <typename T>
int64_t stay_workgroups(const LinearArgs &a, int n_cus) {
    const int64_t per_xcd = n_cus / 8, columns = (a.outputs + kStayOutputs - 1) / kStayOutputs;
    if (a.width <= kStayWidth / 2 || a.width > kStayWidth || columns > per_xcd) return 0;
    if (a.y_stride >= 1 << 24) return 0;  // (places in 32 bits; x's stride is below that in any call)
    if (!whole_lines<T>(a)) return 0;
    const int64_t groups = per_xcd / columns;
    if (8 * groups * columns < 7 * per_xcd) return 0;
    if (a.rows < 32 * 8 * groups * kStayWaves * 2) return 0;
    return 8 * per_xcd;
}

// Whether tiles of 256 x 256 are faster than those of 128 x 128, two of which a compute unit
// makes at a time: by a tenth for the same outputs a compute unit (128000 x 2048 to 512 162
// -> 150 us, 30000 41 -> 38, 30001 x 2047 to 501 47 -> 42), so not where they do not share
// them as evenly (40000 52 -> 66).  Narrow rows are bound by their outputs (300000 x 128 to
// 512 65 -> 66), the more so where those begin anywhere (128000 x 512 to 1000 142 -> 154,
// 30000 x 1024 53 -> 48).
template <typename T>
bool wide_tiles(const LinearArgs &a, int n_cus) {
    const auto turns = [&](int64_t size, int64_t beside) {
        const int64_t tiles = (a.rows + size - 1) / size * ((a.outputs + size - 1) / size);
        return (tiles + beside - 1) / beside;
    };
    return a.width >= (whole_lines<T>(a) ? 2 : 8) * kStep && a.y_stride < 1 << 24 &&
           9 * 4 * turns(kWide, n_cus) <= 10 * 2 * turns(128, 2 * n_cus);
}

template <typename T>
hipError_t launch_wide(const LinearArgs &a, int n_cus, hipStream_t stream) {
    const int64_t workgroups = std::max(n_cus / 8 * 8, 8);
    return by_tiles<T, kWide, kWide>(a, [&](const LinearArgs &part) {
        const dim3 grid((uint32_t)std::min(part.tiles, workgroups)), block(kWideThreads);
        const auto launch = [&](auto gelu, auto lines) {
            hipLaunchKernelGGL((linear_wide_kernel<T, decltype(gelu)::value, decltype(lines)::value>), grid, block, 0, stream, part);
        };
        const auto with_gelu = [&](auto gelu) { whole_lines<T>(part) ? launch(gelu, std::true_type{}) : launch(gelu, std::false_type{}); };
        a.gelu ? with_gelu(std::true_type{}) : with_gelu(std::false_type{});
    });
}

template <typename T>
hipError_t launch_stay(LinearArgs a, int64_t workgroups, hipStream_t stream) {
    a.column_tiles = (a.outputs + kStayOutputs - 1) / kStayOutputs;
    a.tiles = (a.rows + 31) / 32;
    if (a.gelu) hipLaunchKernelGGL((linear_stay_kernel<T, true>), dim3((uint32_t)workgroups), dim3(64 * kStayWaves), 0, stream, a);
    else hipLaunchKernelGGL((linear_stay_kernel<T, false>), dim3((uint32_t)workgroups), dim3(64 * kStayWaves), 0, stream, a);
    return hipGetLastError();
}

template <typename T, int MT>
hipError_t launch_few(const LinearArgs &a, hipStream_t stream) {
    hipLaunchKernelGGL((linear_few_kernel<T, MT>), dim3((a.outputs + 15) / 16), dim3(64 * kFewWaves), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(LinearArgs a, int32_t dtype, int n_cus, hipStream_t stream) {
    const auto fits = [](const void *p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 16 == 0; };
    return with_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        if (a.rows <= 16) return launch_few<T, 1>(a, stream);
        if (a.rows <= 32) return launch_few<T, 2>(a, stream);
        if (!fits(a.x, a.x_stride) || !fits(a.w, a.w_stride))
            return by_tiles<T, 64, 64>(a, [&](const LinearArgs &part) {
                hipLaunchKernelGGL((linear_any_kernel<T>), dim3((uint32_t)part.tiles), dim3(kThreads), 0, stream, part);
            });
        if constexpr (sizeof(T) == 2)
            if (const int64_t workgroups = stay_workgroups<T>(a, n_cus)) return launch_stay<T>(a, workgroups, stream);
        if constexpr (sizeof(T) == 2)
            if (wide_tiles<T>(a, n_cus)) return launch_wide<T>(a, n_cus, stream);
        const int64_t tiles = (a.rows + 127) / 128 * ((a.outputs + 127) / 128);
        if (tiles < 2 * (int64_t)n_cus) return launch_tiles<T, 64, 64>(a, 4, n_cus, stream);
        return launch_tiles<T, 128, 128>(a, 2, n_cus, stream);
    });
}

}  // namespace flock
