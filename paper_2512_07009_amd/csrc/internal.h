// internal.h - declarations shared by the library's own translation units
// (host API and kernel launchers).  Not part of the public C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace flock {

// ----------------------------------------------------------------------------
// Clustering
// ----------------------------------------------------------------------------
struct ClusterArgs {
    const int32_t *xy;        // [total][2] 1/16 px
    const int32_t *offsets;   // [n_frames + 1]
    int32_t n_frames;
    int32_t total;
    int32_t eps_q;            // radius in quanta
    int32_t min_pts;
    int32_t cell_side;        // largest s >= 1 with 2 s^2 <= eps_q^2
    int32_t cap_points;       // frames with more points leave the on-chip kernel
    int32_t cap_cells;        // cell-table entries available on chip
    int32_t big_path;         // 1: frames above cap_points go to the multi-workgroup
                              // path; 0: the on-chip kernel clusters them in place
    int32_t big_all;          // 1: the multi-workgroup path takes every frame and also
                              // writes the counts of empty and inconsistent frames
                              // (the on-chip kernel is not launched)
    int32_t union_regs;       // 1: the on-chip unions keep up to 3072 core cells'
                              // edges in registers; 0: always re-read them from LDS
    // Neighbour-cell tables for cells of side cell_side (as the on-chip
    // kernel's build_stencil makes them), packed 6 bits per cell offset
    // ((dx + 2) | (dy + 2) << 3), five per word:
    uint32_t sten_all[5];     // the whole stencil, nearest cells first
    uint32_t sten_fwd[3];     // its forward half, adjacent cells first
    uint32_t sten_meta;       // nsten | nadj << 8 | nfwd << 16 | dxmax[k] << (24 + 2 k)
    int32_t *labels;          // [total]
    uint8_t *kind;            // [total]
    int32_t *n_clusters;      // [n_frames] or nullptr
};

// Bytes of dynamic LDS the resident clustering kernel needs for these caps.
size_t cluster_lds_bytes(int32_t cap_points, int32_t cap_cells);
// Largest point capacity that fits the device's LDS with a cell table of
// at least min_cells entries.
int32_t cluster_max_cap_points(size_t lds_limit);

// Static shared memory of the compact clustering kernel (bytes).
size_t cluster_compact_static_lds();
// Largest frame the compact kernel holds (points per thread x threads).
constexpr int32_t kClusterCompactCap = 5120;
// compact: the two-workgroups-per-compute-unit kernel (frames of at most
// kClusterCompactCap points, lds_bytes at most half a compute unit's LDS
// less its static shared memory).
hipError_t launch_cluster_resident(const ClusterArgs &a, size_t lds_bytes, bool compact, hipStream_t stream);

// Multi-workgroup path for frames above cap_points (cluster_big.hip).
size_t cluster_big_workspace(int32_t n_frames, int32_t total);
hipError_t launch_cluster_big(const ClusterArgs &a, void *workspace, hipStream_t stream);

// ----------------------------------------------------------------------------
// Density
// ----------------------------------------------------------------------------
struct DensityArgs {
    const int32_t *xy;
    const int32_t *offsets;
    int32_t n_frames;
    int32_t total;
    int32_t width_px, height_px;
    int32_t grid_w, grid_h;
    float sigma_px;
    float *density;           // [n_frames][grid_h][grid_w]
};

struct DensityPlan {
    bool tables;              // factors from tables, else evaluated (density.hip)
    int rm, rn;               // region height and width in tiles of 16 x 16 cells
    int regions_y, regions_x; // regions per frame
    int split;                // bird slices per (frame, region); > 1 adds partial grids afterwards
    int waves;                // waves sharing one (frame, region, slice)
    long long blocks;         // workgroups of the main kernel
    int resident;             // of them per compute unit
    size_t lds_bytes;         // of each
};

// `room`: bytes there are for partial grids (SIZE_MAX: as many as a plan takes).
DensityPlan plan_density(const DensityArgs &a, int n_cus, size_t room);
// Workspace for the partial grids of a split launch (0 if none); depends on the
// batch shape and grid only, and bounds every plan for that shape.
size_t density_workspace_bytes(int32_t n_frames, int32_t total, int32_t grid_w, int32_t grid_h, int n_cus);
hipError_t launch_density(const DensityArgs &a, const DensityPlan &p, float *partial, hipStream_t stream);
// The allocation-free entry point's scratch: a file-scope device array of
// kDensityScratchBytes per device (the partial grids of split launches).
// Returns its address on the current device (looked up once per device).
constexpr size_t kDensityScratchBytes = (size_t)16 << 20;
hipError_t density_static_scratch(void **ptr);

// ----------------------------------------------------------------------------
// Heatmap analytics
// ----------------------------------------------------------------------------
struct HeatArgs {
    const float *density;     // [n_frames][grid_h][grid_w]
    int32_t n_frames;
    int32_t grid_w, grid_h;
    int32_t tiles_x, tiles_y; // set by launch_heatmap
    double cell_area;
    float threshold;
    int32_t connectivity;     // 4 or 8
    int32_t *labels;          // [n_frames][grid_h][grid_w]
    int32_t *n_components;    // [n_frames]
    double *entropy;          // [n_frames]
    double *degree;           // [n_frames]
    int32_t *comp_cells;      // [n_frames][grid_h][grid_w]
    double *comp_mass;        // [n_frames][grid_h][grid_w]
};

size_t heatmap_workspace_bytes(int32_t n_frames, int32_t grid_w, int32_t grid_h);
// Launch plan: component slots of the frame-resident kernel (one workgroup per
// frame, no workspace), 0 for the tiled kernels, which use the workspace.
struct HeatPlan {
    int slots;
    bool spill;  // the frame's bit words wait in comp_mass
};
HeatPlan plan_heatmap(int32_t grid_w, int32_t grid_h, size_t lds_limit);
hipError_t launch_heatmap(HeatArgs a, void *workspace, const HeatPlan &plan, int n_cus, size_t lds_per_cu, hipStream_t stream);

// ----------------------------------------------------------------------------
// Region of interest
// ----------------------------------------------------------------------------
constexpr int kRoiMaxVertices = 64;
constexpr int kRoiBlock = 2048;  // birds per block of the ROI kernels

struct RoiArgs {
    const int32_t *xy;        // [total][2]
    const int32_t *offsets;   // [n_frames + 1]
    int32_t n_frames;
    int32_t total;
    int32_t n_vertices;       // 3 .. kRoiMaxVertices
    int32_t vx[kRoiMaxVertices], vy[kRoiMaxVertices];  // polygon, quanta
    int32_t bx0, by0, bx1, by1;                          // its bounding box
    int32_t *counts;          // [n_frames]
    int32_t *out_xy;          // [total][2] capacity
    int32_t *out_offsets;     // [n_frames + 1]
    int32_t *out_index;       // [total] capacity, or nullptr
};

size_t roi_workspace_bytes(int32_t total);
hipError_t launch_roi(const RoiArgs &a, void *workspace, hipStream_t stream);

// ----------------------------------------------------------------------------
// Drinker-line proximity
// ----------------------------------------------------------------------------
constexpr int kDrinkMaxLines = 64;

struct DrinkArgs {
    const int32_t *xy;        // [total][2]
    const int32_t *offsets;   // [n_frames + 1]
    int32_t n_frames;
    int32_t total;
    int32_t n_lines;          // 1 .. kDrinkMaxLines
    int32_t threshold;        // quanta, 0 .. 2^24
    int32_t ax[kDrinkMaxLines], ay[kDrinkMaxLines], bx[kDrinkMaxLines], by[kDrinkMaxLines];
    uint8_t *drinking;        // [total], 16-byte aligned
    int32_t *line;            // [total] or nullptr
    int32_t *counts;          // [n_frames]
};

size_t drink_workspace_bytes(int32_t total);
hipError_t launch_drinkers(const DrinkArgs &a, void *workspace, hipStream_t stream);

// Detection post-processing (mask components with statistics)
constexpr int kMaskTile = 64;  // tile side in pixels

struct MaskArgs {
    const float *prob;         // [n_frames][height][width]
    int32_t n_frames, width, height;
    float threshold;
    int32_t connectivity;
    int32_t tiles_x, tiles_y;  // set by launch_mask
    int64_t n_tiles;
    int64_t frame_slots, band_slots;
    int32_t *labels;           // optional
    int32_t *n_components;     // [n_frames]
    int32_t *comp_offsets;     // [n_frames + 1]
    int64_t capacity;
    int32_t *comp_label, *comp_area, *comp_box;  // each optional
    double *comp_centroid;
    int32_t *comp_xy;
    float *comp_score;
};
size_t mask_workspace_bytes(int32_t n_frames, int32_t width, int32_t height, int32_t connectivity);
hipError_t launch_mask(MaskArgs a, void *workspace, hipStream_t stream);

// ----------------------------------------------------------------------------
// Per-bird encoder: layer norm, rotary positions, attention
// ----------------------------------------------------------------------------
// Threads of a launch are numbered in 32 bits: workgroups of 256 that one holds.
constexpr int64_t kMaxWorkgroups = (1 << 24) - 1;

// p, n elements of `size` bytes on; nullptr stays.
template <typename P>
inline void move_on(P *&p, int64_t n, size_t size) {
    if (p) p = reinterpret_cast<P *>(reinterpret_cast<uintptr_t>(p) + n * size);
}

struct NormArgs {
    const void *x, *residual;          // [rows][width], strides in elements; residual may be nullptr
    int64_t x_stride, residual_stride;
    int64_t rows;
    int32_t width;
    const float *weight, *bias;        // [width] or nullptr
    float eps;
    void *y, *sum;                     // sum only with residual
    int64_t y_stride, sum_stride;
    float *mean, *rstd;                // [rows] or nullptr

    void advance(int64_t first, size_t size) {
        move_on(x, first * x_stride, size);
        move_on(residual, first * residual_stride, size);
        move_on(y, first * y_stride, size);
        move_on(sum, first * sum_stride, size);
        move_on(mean, first, sizeof(float));
        move_on(rstd, first, sizeof(float));
    }
};
hipError_t launch_norm(const NormArgs &a, int32_t dtype, hipStream_t stream);

struct NormBackwardArgs {
    const void *grad_y, *grad_sum, *x;  // grad_sum may be nullptr
    int64_t grad_y_stride, grad_sum_stride, x_stride;
    int64_t rows;
    int32_t width;
    const float *weight;                // [width] or nullptr
    const float *mean, *rstd;           // [rows]
    void *grad_x;
    int64_t grad_x_stride;
    float *partial;                     // set by launch_norm_backward

    void advance(int64_t first, size_t size) {
        move_on(grad_y, first * grad_y_stride, size);
        move_on(grad_sum, first * grad_sum_stride, size);
        move_on(x, first * x_stride, size);
        move_on(grad_x, first * grad_x_stride, size);
        move_on(mean, first, sizeof(float));
        move_on(rstd, first, sizeof(float));
    }
};
size_t norm_backward_workspace_bytes(int64_t rows, int32_t width, int n_cus);
hipError_t launch_norm_backward(NormBackwardArgs a, int32_t dtype, void *workspace, int n_cus, float *grad_weight,
                                float *grad_bias, hipStream_t stream);

// Root-mean-square norm of rows, or rows as they are, in the features' type or in 8 bits.
struct RmsArgs {
    const void *x, *residual;          // [rows][width], strides in elements; residual may be nullptr
    int64_t x_stride, residual_stride;
    int64_t rows;
    int32_t width;
    const float *weight;               // [width] or nullptr
    float eps;
    void *y, *sum;                     // y is int8 where scale is given; sum only with residual
    int64_t y_stride, sum_stride;
    float *rstd, *scale;               // [rows] or nullptr
    int32_t as_is;                     // 1: no norm (with scale)

    void advance(int64_t first, size_t size) {
        move_on(x, first * x_stride, size);
        move_on(residual, first * residual_stride, size);
        move_on(y, first * y_stride, scale ? 1 : size);
        move_on(sum, first * sum_stride, size);
        move_on(rstd, first, sizeof(float));
        move_on(scale, first, sizeof(float));
    }
};
hipError_t launch_rms(const RmsArgs &a, int32_t dtype, hipStream_t stream);

struct RmsBackwardArgs {
    const void *grad_y, *grad_sum, *x;  // grad_sum may be nullptr
    int64_t grad_y_stride, grad_sum_stride, x_stride;
    int64_t rows;
    int32_t width;
    const float *weight;                // [width] or nullptr
    const float *rstd;                  // [rows]
    void *grad_x;
    int64_t grad_x_stride;
    float *partial;                     // set by launch_rms_backward

    void advance(int64_t first, size_t size) {
        move_on(grad_y, first * grad_y_stride, size);
        move_on(grad_sum, first * grad_sum_stride, size);
        move_on(x, first * x_stride, size);
        move_on(grad_x, first * grad_x_stride, size);
        move_on(rstd, first, sizeof(float));
    }
};
size_t rms_backward_workspace_bytes(int64_t rows, int32_t width, int n_cus);
hipError_t launch_rms_backward(RmsBackwardArgs a, int32_t dtype, void *workspace, int n_cus, float *grad_weight,
                               hipStream_t stream);

// Products of rows and weights in 8 bits.
constexpr int32_t kLinearMaxWidth = (1 << 17) - 1;   // sums stay within 32 bits
constexpr int64_t kLinearMaxStride = (1 << 24) - 16; // a tile's rows lie within 2^32 bytes

struct LinearArgs {
    const int8_t *x, *w;               // [rows][width], [outputs][width], strides in bytes
    int64_t x_stride, w_stride;
    int64_t rows;
    int32_t width, outputs;
    const float *x_scale, *w_scale;    // [rows], [outputs]
    const float *bias;                 // [outputs] or nullptr
    int32_t gelu;
    void *y;                           // [rows][outputs]
    int64_t y_stride;
    int32_t column_tiles;              // set by launch_linear: tiles of outputs, and of all
    int64_t tiles;

    void advance(int64_t first, size_t size) {
        move_on(x, first * x_stride, 1);
        move_on(x_scale, first, sizeof(float));
        move_on(y, first * y_stride, size);
    }
};
hipError_t launch_linear(LinearArgs a, int32_t dtype, int n_cus, hipStream_t stream);

constexpr int kRotaryMaxPairs = 128;

struct RotaryArgs {
    const void *q, *k;                 // [total][heads][head_dim], strides of birds in elements
    void *q_out, *k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
    const int32_t *xy;                 // [total][2], or nullptr without y and x pairs
    const int32_t *time;               // [total], or nullptr without time pairs
    int64_t total;
    int32_t q_heads, k_heads, head_dim;
    int32_t n_time, n_y, pairs;        // pairs = n_time + n_y + n_x
    int32_t interleaved, inverse;
    int32_t tail, birds_per_block;     // set by launch_rotary
    uint32_t chunk_reciprocal, head_reciprocal, pair_reciprocal;
    uint64_t step[kRotaryMaxPairs];    // 2^-64 turns per unit

    void advance(int64_t first, size_t size) {
        move_on(q, first * q_stride, size);
        move_on(k, first * k_stride, size);
        move_on(q_out, first * q_out_stride, size);
        move_on(k_out, first * k_out_stride, size);
        move_on(xy, 2 * first, sizeof(int32_t));
        move_on(time, first, sizeof(int32_t));
    }
};
hipError_t launch_rotary(RotaryArgs a, int32_t dtype, hipStream_t stream);

// Tracks: a paged cache of keys and values in 8 bits (layout: tracks_common.h).
constexpr int kTrackPage = 64;
constexpr int32_t kTrackMaxPages = 1 << 24;  // of a track: tokens are numbered in 31 bits

struct TrackCacheArgs {
    int8_t *k, *v;                     // [pages][kv_heads][64 * dim]
    float *k_scale, *v_scale;          // [pages][kv_heads]
    int32_t pages, kv_heads, dim;
};

struct TrackArgs {
    const int32_t *offsets;            // [n_tracks + 1]: rows of each track
    const int32_t *lengths;            // [n_tracks]: tokens, those of the rows among them
    const int32_t *table;              // [n_tracks][max_pages], rows table_stride apart
    int64_t table_stride;
    int32_t n_tracks, total, max_pages;
};

struct AppendArgs {
    TrackArgs tracks;
    TrackCacheArgs cache;
    const void *k, *v;                 // [total][kv_heads][dim], strides of rows in elements
    int64_t k_stride, v_stride;
    const int32_t *xy, *time;
    int32_t n_time, n_y, pairs, interleaved;
    int32_t pack_shift, pair_shift;    // set by launch_append
    uint64_t step[kRotaryMaxPairs];
};
int64_t append_workgroups(int32_t n_tracks, int32_t total, int32_t kv_heads);
hipError_t launch_append(AppendArgs a, int32_t dtype, hipStream_t stream);

struct TrackAttentionArgs {
    TrackArgs tracks;
    TrackCacheArgs cache;
    const void *q;                     // [total][q_heads][dim]
    void *out;
    int64_t q_stride, out_stride;
    int32_t q_heads, window;
    float scale, cap;
    int32_t group, tile_shift, gathered, splits, split_pages;  // set by launch_track_attention
    float *part_out, *part_stat;
};

// How the pages of a row are dealt out.
struct TrackPlan {
    int32_t tile_rows;    // rows of a workgroup
    int32_t waves;        // ... and its waves, which share their pages
    int64_t slots;        // numbers of row tiles
    int32_t splits;       // workgroups that may share a row's pages ...
    int32_t split_pages;  // ... and how many pages each takes
};
TrackPlan plan_track_attention(int32_t n_tracks, int32_t total, int32_t max_pages, int32_t q_heads, int32_t kv_heads,
                               int n_cus);
size_t track_attention_workspace_bytes(const TrackPlan &p, int32_t total, int32_t q_heads, int32_t dim);
hipError_t launch_track_attention(TrackAttentionArgs a, int32_t dtype, const TrackPlan &p, void *workspace,
                                  hipStream_t stream);

constexpr int kAttentionMaxDim = 128;
// 64 rows lie within 2^31 bytes: a tile's loads go through resources of 64 rows at most
constexpr int64_t kAttentionMaxStride = (1 << 24) - 8;

struct AttentionArgs {
    const void *q, *k, *v;             // [total][heads][dim], strides of birds in elements
    void *out;
    int64_t q_stride, k_stride, v_stride, out_stride;
    const int32_t *q_offsets, *k_offsets;  // [n_frames + 1]
    int32_t n_frames, total_q, total_k;
    int32_t q_heads, kv_heads, group, dim;  // group = q_heads / kv_heads
    uint32_t group_reciprocal;         // set by the launches
    const int32_t *q_xy, *k_xy;        // 1/16 px, with slopes
    const float *slopes;               // [q_heads] or nullptr
    const uint8_t *keep;               // [total_k] or nullptr
    const int32_t *prefix;             // [n_frames] or nullptr
    int32_t causal;
    float scale, cap;                  // cap = 0: none
    double *lse;                       // [total_q][q_heads] or nullptr
    int64_t slots;                     // set by the launches: numbers of row tiles
    int32_t splits;
    float *part_out, *part_stat;
};

// How the rows of a forward launch are dealt out.
struct AttentionPlan {
    bool split;      // 32 rows a workgroup and a quarter of the keys a wave
    int32_t splits;  // workgroups that share a row's keys
    int64_t slots;
};
AttentionPlan plan_attention(int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads, int32_t kv_heads,
                             int n_cus);
size_t attention_workspace_bytes(const AttentionPlan &p, int32_t total_q, int32_t q_heads, int32_t dim);
hipError_t launch_attention(AttentionArgs a, int32_t dtype, const AttentionPlan &p, void *workspace,
                            hipStream_t stream);

struct AttentionBackwardArgs {
    AttentionArgs fwd;
    const void *grad_out;
    void *grad_q, *grad_k, *grad_v;
    int64_t grad_out_stride, grad_q_stride, grad_k_stride, grad_v_stride;
    float *delta, *slope_shares;       // set by launch_attention_backward: [total_q][q_heads], [slots][q_heads]
    int64_t key_slots;
};
// Workgroups of the largest launch, for kMaxWorkgroups.
int64_t attention_workgroups(const AttentionPlan &p, int32_t total_q, int32_t q_heads, int32_t kv_heads);
int64_t attention_backward_workgroups(int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads, int32_t kv_heads);
size_t attention_backward_workspace_bytes(int32_t n_frames, int32_t total_q, int32_t q_heads, int32_t kv_heads);
hipError_t launch_attention_backward(AttentionBackwardArgs b, int32_t dtype, void *workspace, float *grad_slopes,
                                     hipStream_t stream);

}  // namespace flock
