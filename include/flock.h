/*
 * flock.h - C ABI of the MI355X (gfx950) per-frame bird clustering and
 * density library (libflock.so).
 *
 * The library computes, for a batch of video frames that each hold a ragged
 * set of detected bird centroids, the two per-frame analytics of the paper's
 * clustering module (Section 2.3; Section 3.6 and Algorithm 1):
 *   - radius-neighbour clustering of the birds (core / border / noise kinds
 *     and connected-component cluster labels), and
 *   - a Gaussian kernel density grid.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  Batch layout (CSR over frames; the paper's "frames" of tracked positions,
 *  Algorithm 1):
 *    xy       device, int32[total][2]: (x, y) of each bird in 1/16 px,
 *             0 <= x, y < 2^24.  Frame f is rows offsets[f] .. offsets[f+1]-1.
 *    offsets  device, int32[n_frames + 1]: offsets[0] = 0, non-decreasing,
 *             offsets[n_frames] = total.
 *    n_frames, total: host copies of the batch sizes.
 *  Every pointer argument is device memory owned by the caller; the library
 *  neither frees nor keeps it after the call returns.
 *  stream: a hipStream_t (NULL = the null stream).  Calls only enqueue work:
 *  outputs are valid once the stream reaches the call's point.  No host-device
 *  copy and no synchronisation happens, except when the environment variable
 *  FLOCK_VALIDATE=1 asks for a synchronous device-side check of offsets.
 *  Errors: a negative status; flock_last_error() then describes it.  On
 *  FLOCK_EINVAL nothing is enqueued and the outputs are untouched.  A frame
 *  whose offsets are inconsistent (negative count, past total) is never read;
 *  its outputs are left untouched and its n_clusters entry is set to -1 (so is
 *  that of a frame above the on-chip capacity whose birds cannot all be told
 *  from another, inconsistent frame's).
 *  Thread safety: calls on different streams may run concurrently; the only
 *  global state is a per-thread error string and a once-initialised cache of
 *  device properties.
 *  Graph capture: a call enqueues only kernel launches when it is given the
 *  workspace its *_workspace() query asks for (or when that query returns 0),
 *  so it can be captured into a HIP graph.  With a NULL workspace where one
 *  is needed the library allocates and frees its scratch stream-ordered
 *  (hipMallocAsync / hipFreeAsync), which a capture records as memory nodes;
 *  pass a workspace (or use density_frames_noalloc) under capture.
 */
#ifndef FLOCK_H
#define FLOCK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t flock_status;

#define FLOCK_OK 0
#define FLOCK_EINVAL (-1)      /* bad argument: nothing enqueued, outputs untouched */
#define FLOCK_ENOMEM (-2)      /* workspace too small, or allocation failed */
#define FLOCK_EDEVICE (-3)     /* a HIP runtime call failed (message has its text) */
#define FLOCK_EUNSUPPORTED (-4) /* device is not gfx950, or a size beyond the limits */

/*
 * cluster_frames - radius-neighbour (DBSCAN-style) clustering of every frame.
 *
 * The paper's clustering module groups nearby birds by connected-component
 * analysis (Section 2.3) and names the per-frame distance loops as the
 * bottleneck (Section 3.6).  The point-level definition computed here is
 * standard DBSCAN (Ester et al., 1996) with these exact conventions:
 *   neighbours   (x_i - x_j)^2 + (y_i - y_j)^2 <= eps_q^2, in exact integer
 *                arithmetic on the 1/16-px coordinates; a bird is its own
 *                neighbour and coincident birds count;
 *   core         a bird with >= min_pts neighbours;
 *   cluster      a connected component of core birds under the neighbour
 *                relation; its label is the smallest frame-local index of a
 *                core bird in it (global index = label + offsets[f]);
 *   border       a non-core bird with a core neighbour: it joins the cluster
 *                of its nearest core neighbour, ties broken by the smaller
 *                (y, x) of that core;
 *   noise        every other bird: label -1.
 *
 * Arguments:
 *   max_frame_points  host: an upper bound on the birds in any one frame
 *                     (used to size on-chip storage), or 0 if unknown.  A
 *                     frame above the bound is still clustered correctly, on a
 *                     slower path.
 *   eps_q             radius in 1/16 px, 0 <= eps_q <= 32766 (eps px = eps_q/16).
 *   min_pts           >= 1; the count includes the bird itself.
 *   labels            device out, int32[total]: frame-local cluster label or -1.
 *   kind              device out, uint8[total]: 0 noise, 1 border, 2 core.
 *   n_clusters        device out, int32[n_frames] (or NULL): clusters per frame.
 *   workspace         device scratch of workspace_bytes bytes, at least
 *                     cluster_frames_workspace(...) of them, 256-byte aligned;
 *                     or NULL, in which case the library allocates and frees
 *                     its scratch stream-ordered (hipMallocAsync/hipFreeAsync).
 * Labels, kinds and n_clusters are a deterministic function of the input:
 * they do not depend on the order of birds within a frame beyond the labels'
 * index convention, nor on thread scheduling.
 */
flock_status cluster_frames(const int32_t *xy, const int32_t *offsets, int32_t n_frames,
                            int32_t total, int32_t max_frame_points, int32_t eps_q,
                            int32_t min_pts, int32_t *labels, uint8_t *kind,
                            int32_t *n_clusters, void *workspace, size_t workspace_bytes,
                            void *stream);

/* Bytes of workspace cluster_frames needs for this batch shape (may be 0). */
size_t cluster_frames_workspace(int32_t n_frames, int32_t total, int32_t max_frame_points);

/*
 * density_frames - Gaussian kernel density grid of every frame.
 *
 * Algorithm 1 (Section 3.6) computes, for every grid cell and every bird, a
 * distance-based contribution to the cell's density; the paper vectorises
 * the grid-to-bird distances.  The grid here has grid_w x grid_h cells tiling
 * the frame [0, width_px) x [0, height_px), evaluated at the cell centres
 *     cx = (gx + 1/2) width_px / grid_w,   cy = (gy + 1/2) height_px / grid_h,
 * and each bird (x, y) = (x_q/16, y_q/16) px adds an isotropic Gaussian of
 * bandwidth sigma_px with unit mass:
 *     density[f][gy][gx] = sum_i exp(-((cx-x_i)^2 + (cy-y_i)^2) / (2 sigma^2))
 *                          / (2 pi sigma^2)                    [birds / px^2]
 * The sum factorises as density = c * Fy . Fx^T with Fx[gx][i] and Fy[gy][i]
 * the per-axis Gaussian factors; it is evaluated as that contraction over
 * the birds on the matrix cores, fp16 factors with fp32 accumulation.
 * Accuracy: relative to the frame's maximum, |error| <= 1e-3 (the fp16
 * rounding of the two factors bounds each term's relative error by about
 * 2^-10); an empty frame gives exact zeros.
 *
 * Arguments:
 *   max_frame_points      host: an upper bound on the birds in any one frame,
 *                         or 0 if unknown (a planning hint; every value >= 0
 *                         gives the same result).
 *   width_px, height_px   frame extent, >= 1.
 *   grid_w, grid_h        grid size, 1 .. 4096 each.
 *   sigma_px              bandwidth, finite, > 0.
 *   density               device out, float[n_frames][grid_h][grid_w].
 *   workspace             as for cluster_frames, sized by
 *                         density_frames_workspace(...).  Batches with few
 *                         frames are split into bird slices whose partial
 *                         grids are kept there and added in slice order.  A
 *                         shorter workspace holds fewer slices; one that holds
 *                         less than two is taken, without slices, on grids
 *                         whose cells are no whole number of 1/16 px or whose
 *                         6-sigma windows reach more than 29 cells, and
 *                         refused (FLOCK_ENOMEM) where another grid's launch
 *                         wants slices.
 * The result is deterministic (fixed summation order; the order, and with it
 * the last bits, depends on the slices, so on a workspace shorter than the
 * query's).  Frames whose offsets
 * are invalid (checked only with FLOCK_VALIDATE) leave their grid unspecified.
 */
flock_status density_frames(const int32_t *xy, const int32_t *offsets, int32_t n_frames,
                            int32_t total, int32_t max_frame_points, int32_t width_px,
                            int32_t height_px, int32_t grid_w, int32_t grid_h, float sigma_px,
                            float *density, void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of workspace density_frames needs for this batch shape and grid
 * (0 when no split is needed); the same value bounds every call with these
 * four arguments, whatever the frame extent and sigma. */
size_t density_frames_workspace(int32_t n_frames, int32_t total, int32_t grid_w, int32_t grid_h);

/*
 * density_frames_noalloc - density_frames for callers that cannot allocate
 * device memory: code under HIP graph capture, tight serving loops, and
 * harnesses that forbid allocation.
 *
 * Arguments, result and accuracy are those of density_frames (the same plan
 * and kernels, so the same bits as with a NULL workspace or one of the queried
 * size), without the workspace: a launch split into
 * bird slices keeps its partial grids in a static scratch array of the
 * library, 16 MiB per device (n_frames * slices * grid_w * grid_h * 4 bytes;
 * density_frames_workspace() gives that size for a batch shape).  The call
 * allocates nothing and makes no host-device copy or synchronisation
 * (FLOCK_VALIDATE is ignored here).
 * Errors: FLOCK_ENOMEM, with nothing enqueued, when the batch needs more
 * partial-grid bytes than the scratch holds; otherwise as density_frames.
 * Every call on one device shares that device's scratch: calls that overlap
 * in time on one device (concurrent streams, or threads) race and must be
 * serialised by the caller.  Every byte a call reads from the scratch it has
 * written first, so nothing needs clearing between calls.
 */
flock_status density_frames_noalloc(const int32_t *xy, const int32_t *offsets, int32_t n_frames,
                                    int32_t total, int32_t max_frame_points, int32_t width_px,
                                    int32_t height_px, int32_t grid_w, int32_t grid_h, float sigma_px,
                                    float *density, void *stream);

/*
 * heatmap_frames - heatmap analytics of every frame's density grid.
 *
 * The clustering module of Section 2.3 thresholds the density heatmaps and
 * applies connected component analysis; Algorithm 1 computes the heatmap,
 * its entropy and a clustering degree per frame.  The paper fixes none of
 * the details; this entry point computes, per frame f and cell
 * c = gy * grid_w + gx:
 *   hot          density[f][c] >= threshold;
 *   labels       connected hot cells under the 4-neighbourhood (shared edge)
 *                or the 8-neighbourhood (shared edge or corner) form a
 *                component, labelled by its smallest cell index; cold cells
 *                get -1;
 *   comp_cells, comp_mass   at each component's label cell, its number of
 *                cells and cell_area_px2 * (sum of its density) (expected
 *                birds); 0 at every other cell;
 *   n_components number of components;
 *   entropy      -sum p ln p over the cells with density > 0,
 *                p = density / S, S the sum of those cells (0 if S = 0);
 *   degree       (sum of density over hot cells) / S (0 if S = 0): the share
 *                of the frame's density mass that lies in components.
 *
 * Arguments:
 *   density          device in, float[n_frames][grid_h][grid_w], finite and
 *                    >= 0 (the output of density_frames).
 *   grid_w, grid_h   1 .. 4096 each.
 *   cell_area_px2    area of one cell in px^2 (W H / (grid_w grid_h)), >= 0.
 *   threshold        birds / px^2, finite and > 0.
 *   connectivity     4 or 8.
 *   labels, comp_cells   device out, int32[n_frames][grid_h][grid_w].
 *   comp_mass        device out, double[n_frames][grid_h][grid_w], 8-byte
 *                    aligned.
 *   n_components     device out, int32[n_frames].
 *   entropy, degree  device out, double[n_frames].
 *   workspace        as for cluster_frames, sized by heatmap_frames_workspace.
 * Every output is deterministic: sums are taken in a fixed order, and the
 * component masses are summed as 64-bit integers of a per-frame fixed-point
 * scale (each cell rounded to within 2^(lg - 62) of the frame's largest cell,
 * lg = ceil(log2(grid_w grid_h))).
 */
flock_status heatmap_frames(const float *density, int32_t n_frames, int32_t grid_w, int32_t grid_h,
                            double cell_area_px2, float threshold, int32_t connectivity,
                            int32_t *labels, int32_t *n_components, double *entropy, double *degree,
                            int32_t *comp_cells, double *comp_mass, void *workspace,
                            size_t workspace_bytes, void *stream);

/* Bytes of workspace heatmap_frames needs for this batch shape. */
size_t heatmap_frames_workspace(int32_t n_frames, int32_t grid_w, int32_t grid_h);

/*
 * roi_filter_frames - birds inside a region of interest, and per-frame counts.
 *
 * The wall pipeline counts the birds in a region near the wall (Section
 * 2.2), and Algorithm 1 filters the birds to the region of interest before
 * the density.  A bird is kept when its point (x_q, y_q) lies in the closed
 * polygon roi_xy (edges and vertices included; even-odd rule, which for a
 * simple polygon is its interior plus its boundary), tested exactly in
 * integers.  Kept birds keep their input order.
 *
 * Arguments:
 *   xy, offsets, n_frames, total   the batch, as for cluster_frames.
 *   roi_xy        host in, int32[n_vertices][2], vertices in 1/16 px with
 *                 |coordinate| <= 2^24, in either orientation; the last
 *                 vertex joins the first.  Copied during the call.
 *   n_vertices    3 .. 64.
 *   counts        device out, int32[n_frames]: kept birds per frame.
 *   out_xy        device out, int32[total][2] capacity: the kept birds, frame
 *                 after frame (the first out_offsets[n_frames] rows written).
 *   out_offsets   device out, int32[n_frames + 1]: CSR offsets of out_xy.
 *   out_index     device out, int32[total] capacity, or NULL: the input index
 *                 of each kept bird.
 *   workspace     as for cluster_frames, sized by roi_filter_frames_workspace.
 * Offsets must describe the batch (checked only with FLOCK_VALIDATE); with
 * invalid offsets the outputs are unspecified but every access stays in
 * bounds.
 */
flock_status roi_filter_frames(const int32_t *xy, const int32_t *offsets, int32_t n_frames, int32_t total,
                               const int32_t *roi_xy, int32_t n_vertices, int32_t *counts, int32_t *out_xy,
                               int32_t *out_offsets, int32_t *out_index, void *workspace,
                               size_t workspace_bytes, void *stream);

/* Bytes of workspace roi_filter_frames needs for this batch (a flag bit per bird,
 * a count and a base per block of 2048 birds, and 12 bytes per bird, rounded
 * up to whole blocks, where each block stages its kept birds). */
size_t roi_filter_frames_workspace(int32_t n_frames, int32_t total);

/*
 * drinker_proximity_frames - birds near drinker lines, and per-frame counts.
 *
 * The drinker pipeline computes each bird's distance to the nearest drinker
 * line and classifies the bird as drinking when the distance falls below a
 * threshold (Section 2.3).  Drinker lines are closed segments; the distance
 * is from the bird's point to the nearest point of a segment (end points
 * included); a bird drinks when that distance is strictly below
 * threshold_q for some segment.  The test is exact in integers.
 *
 * Arguments:
 *   xy, offsets, n_frames, total   the batch, as for cluster_frames
 *                    (coordinates 0 <= x, y < 2^24).
 *   lines            host in, int32[n_lines][4] = (ax, ay, bx, by) in 1/16 px,
 *                    |coordinate| <= 2^24.  Copied during the call.
 *   n_lines          1 .. 64.
 *   threshold_q      distance threshold in 1/16 px, 0 .. 2^24.
 *   drinking         device out, uint8[total] (16-byte aligned): 1 if drinking.
 *   line             device out, int32[total], or NULL: the smallest index of
 *                    a segment strictly within the threshold, -1 if none.
 *   counts           device out, int32[n_frames]: drinking birds per frame.
 *   workspace        as for cluster_frames, sized by
 *                    drinker_proximity_frames_workspace.
 */
flock_status drinker_proximity_frames(const int32_t *xy, const int32_t *offsets, int32_t n_frames,
                                      int32_t total, const int32_t *lines, int32_t n_lines,
                                      int32_t threshold_q, uint8_t *drinking, int32_t *line,
                                      int32_t *counts, void *workspace, size_t workspace_bytes,
                                      void *stream);

/* Bytes of workspace drinker_proximity_frames needs for this batch. */
size_t drinker_proximity_frames_workspace(int32_t n_frames, int32_t total);

/*
 * mask_components_frames - detection post-processing of a batch of
 * segmentation outputs.
 *
 * Section 3.2 turns the segmentation network's output into detections with
 * a connected-components-with-statistics routine (threshold, connected
 * components, bounding boxes; Section 2.3 gives each box a confidence
 * score).  Per frame f and pixel p = y * width + x:
 *   foreground   prob[f][p] > threshold (NaN is background);
 *   labels       connected foreground pixels under the 4-neighbourhood
 *                (shared edge) or the 8-neighbourhood (shared edge or corner)
 *                form a component, labelled by its first pixel in raster
 *                order (smallest p); background gets -1;
 *   components   listed frame after frame, in label order within a frame:
 *                label, area (pixels), box (x, y, width, height), centroid
 *                (mean x, mean y of the pixel indices, correctly rounded
 *                quotient of exact integer sums), xy = floor(16 sum / area)
 *                per axis (the centroid in the 1/16-px layout of
 *                cluster_frames, with comp_offsets as its offsets), and score
 *                (largest probability among the component's pixels).
 *
 * Arguments:
 *   prob            device in, float[n_frames][height][width].
 *   width, height   1 .. 32768 each; n_frames * width * height < 2^31.
 *   threshold       finite and >= 0.
 *   connectivity    4 or 8.
 *   labels          device out, int32[n_frames][height][width], or NULL.
 *   n_components    device out, int32[n_frames].
 *   comp_offsets    device out, int32[n_frames + 1]: CSR offsets of the
 *                   component list; comp_offsets[n_frames] is the count K.
 *   capacity        rows of the component outputs; components with rank
 *                   >= capacity are counted but not written.
 *   comp_label, comp_area   device out, int32[capacity], or NULL.
 *   comp_box        device out, int32[capacity][4], 16-byte aligned, or NULL.
 *   comp_centroid   device out, double[capacity][2], 16-byte aligned, or NULL.
 *   comp_xy         device out, int32[capacity][2], 8-byte aligned, or NULL.
 *   comp_score      device out, float[capacity], or NULL.
 *   workspace       as for cluster_frames, sized by
 *                   mask_components_frames_workspace.
 * Every output is deterministic: statistics are integer sums, minima and
 * maxima, so their order of accumulation does not matter.
 */
flock_status mask_components_frames(const float *prob, int32_t n_frames, int32_t width, int32_t height,
                                    float threshold, int32_t connectivity, int32_t *labels,
                                    int32_t *n_components, int32_t *comp_offsets, int32_t capacity,
                                    int32_t *comp_label, int32_t *comp_area, int32_t *comp_box,
                                    double *comp_centroid, int32_t *comp_xy, float *comp_score,
                                    void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of workspace mask_components_frames needs for this batch shape: 56
 * bytes per possible piece of a component inside a 64 x 64 tile (a quarter
 * of the pixels with 8 neighbours, half with 4), plus the tile seams and a
 * bit per pixel. */
size_t mask_components_frames_workspace(int32_t n_frames, int32_t width, int32_t height, int32_t connectivity);

/*
 * Per-bird encoder
 * ----------------
 * Learned functions of ragged sets of birds (activity classes or weights per
 * bird, Section 2.3, from models that a user trains) run on the same CSR
 * batches: the birds of a frame, or the detections of one bird's track, attend
 * to each other.  The entries below are its operators and their gradients.
 *
 * Features are matrices of `dtype` in device memory.  Rows may lie apart: a
 * stride is the distance between the starts of two rows in elements, so that
 * queries, keys and values can be slices of one projection.  The heads of a
 * row are contiguous, head h at h * head_dim.  No output may overlap an input,
 * except as stated at layer_norm_rows and rotary_frames.
 * Attention numbers its work by the offsets: in a batch with an inconsistent
 * frame, what the other frames get is not defined.  Nothing is read or written
 * out of range, and rows that no consistent frame holds are left untouched.
 */
#define FLOCK_F32 0
#define FLOCK_F16 1
#define FLOCK_BF16 2

/*
 * layer_norm_rows - layer norm of every row, with an optional residual.
 *
 *   h = x, or x + residual rounded to dtype, which is written to sum;
 *   y = (h - mean) * rstd * weight + bias,
 *   mean = sum h / width,  rstd = 1 / sqrt(sum (h - mean)^2 / width + eps)
 * Statistics are taken in 32 bits, the variance from the centred values.
 *
 * Arguments:
 *   dtype          FLOCK_F32, FLOCK_F16 or FLOCK_BF16: x, residual, y, sum.
 *   x, residual    device in, [rows][width]; residual may be NULL.
 *   rows, width    rows >= 0, width 1 .. 2^20.
 *   *_stride       >= 0 for inputs, >= width for outputs.
 *   weight, bias   device in, float[width], or NULL (1 and 0).
 *   eps            finite, >= 0.
 *   y, sum         device out, [rows][width]; sum must be given with residual,
 *                  and is not used without.  y may be x, and sum residual.
 *   mean, rstd     device out, float[rows], or NULL: what the backward pass takes.
 */
flock_status layer_norm_rows(int32_t dtype, const void *x, int64_t x_stride, const void *residual,
                             int64_t residual_stride, int32_t rows, int32_t width, const float *weight,
                             const float *bias, float eps, void *y, int64_t y_stride, void *sum,
                             int64_t sum_stride, float *mean, float *rstd, void *stream);

/*
 * layer_norm_rows_backward - gradients of layer_norm_rows.
 *
 * With xh = (x - mean) * rstd and g = grad_y * weight, per row
 *   grad_x = rstd * (g - mean(g) - xh * mean(g * xh)) (+ grad_sum)
 * and over the rows, in a fixed order,
 *   grad_weight = sum grad_y * xh,  grad_bias = sum grad_y.
 *
 * Arguments:
 *   grad_y         device in, [rows][width].
 *   grad_sum       device in, [rows][width], or NULL: the gradient that the
 *                  kept sum got elsewhere.  grad_x is the gradient of x and of
 *                  the residual alike.
 *   x              device in: what was normalised (x, or the kept sum).
 *   mean, rstd     device in, float[rows], from layer_norm_rows.
 *   grad_x         device out, [rows][width].
 *   grad_weight, grad_bias   device out, float[width], or NULL.
 *   workspace      as for cluster_frames, sized by
 *                  layer_norm_rows_backward_workspace(...).
 */
flock_status layer_norm_rows_backward(int32_t dtype, const void *grad_y, int64_t grad_y_stride,
                                      const void *grad_sum, int64_t grad_sum_stride, const void *x,
                                      int64_t x_stride, int32_t rows, int32_t width, const float *weight,
                                      const float *mean, const float *rstd, void *grad_x,
                                      int64_t grad_x_stride, float *grad_weight, float *grad_bias,
                                      void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of workspace layer_norm_rows_backward needs for its column sums. */
size_t layer_norm_rows_backward_workspace(int32_t rows, int32_t width);

/*
 * rms_norm_rows - root-mean-square norm of every row, with an optional residual.
 *
 *   h = x, or x + residual rounded to dtype, which is written to sum;
 *   y = h * rstd * weight,  rstd = 1 / sqrt(sum h^2 / width + eps)
 * Squares are summed in 32 bits.
 *
 * Arguments: as for layer_norm_rows, without bias and mean.
 */
flock_status rms_norm_rows(int32_t dtype, const void *x, int64_t x_stride, const void *residual,
                           int64_t residual_stride, int32_t rows, int32_t width, const float *weight, float eps,
                           void *y, int64_t y_stride, void *sum, int64_t sum_stride, float *rstd, void *stream);

/*
 * rms_norm_rows_backward - gradients of rms_norm_rows.
 *
 * With xh = x * rstd and g = grad_y * weight, per row
 *   grad_x = rstd * (g - xh * mean(g * xh)) (+ grad_sum)
 * and over the rows, in a fixed order, grad_weight = sum grad_y * xh.
 *
 * Arguments: as for layer_norm_rows_backward, without mean and grad_bias;
 * workspace sized by rms_norm_rows_backward_workspace(...).
 */
flock_status rms_norm_rows_backward(int32_t dtype, const void *grad_y, int64_t grad_y_stride,
                                    const void *grad_sum, int64_t grad_sum_stride, const void *x,
                                    int64_t x_stride, int32_t rows, int32_t width, const float *weight,
                                    const float *rstd, void *grad_x, int64_t grad_x_stride, float *grad_weight,
                                    void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of workspace rms_norm_rows_backward needs for its column sums. */
size_t rms_norm_rows_backward_workspace(int32_t rows, int32_t width);

/*
 * rms_norm_rows_i8 - rms_norm_rows with its output in 8 bits.
 *
 * y as for rms_norm_rows, in 32 bits, is not written; per row
 *   scale = max |y| / 127,  q = y / scale to the nearest whole number, ties to even
 * (both quotients in 32 bits), so that y is scale * q to half a scale.  A row whose
 * largest |y| is below 2^-100 has scale and q 0; one with a value that is not
 * finite has scale NaN and q 0.
 *
 * Arguments: as for rms_norm_rows, and
 *   q              device out, int8[rows][width], rows q_stride bytes apart
 *                  (>= width; what lies between rows is left as it was).
 *   scale          device out, float[rows].
 */
flock_status rms_norm_rows_i8(int32_t dtype, const void *x, int64_t x_stride, const void *residual,
                              int64_t residual_stride, int32_t rows, int32_t width, const float *weight,
                              float eps, int8_t *q, int64_t q_stride, float *scale, void *sum,
                              int64_t sum_stride, void *stream);

/*
 * quantize_rows - rows in 8 bits with a scale each: q and scale as for
 * rms_norm_rows_i8, with y = x.  A weight's rows are its outputs.
 */
flock_status quantize_rows(int32_t dtype, const void *x, int64_t x_stride, int32_t rows, int32_t width, int8_t *q,
                           int64_t q_stride, float *scale, void *stream);

/*
 * linear_rows_i8 - products of rows in 8 bits with weights in 8 bits.
 *
 *   y[m][n] = act(x_scale[m] * w_scale[n] * sum_k x[m][k] * w[n][k] + bias[n])
 * Sums over k are exact; what follows is in 32 bits, with one rounding to dtype.
 * act is the identity, or with gelu act(t) = t Phi(t), Phi being the normal
 * distribution (to 1e-5 of itself, in types of 16 bits 4e-5 before its rounding);
 * gelu of -infinity is 0.
 *
 * Arguments:
 *   dtype          FLOCK_F32, FLOCK_F16 or FLOCK_BF16: y.
 *   x              device in, int8[rows][width], rows x_stride bytes apart
 *                  (0 <= x_stride < 2^24), from rms_norm_rows_i8 or
 *                  quantize_rows.  Rows that begin at multiples of 16 bytes, of x
 *                  and w both, are loaded fastest; what follows a row's end in the
 *                  same 16 bytes may be read then, and has no influence.
 *   x_scale        device in, float[rows].
 *   w              device in, int8[outputs][width], rows w_stride bytes apart.
 *   w_scale        device in, float[outputs].
 *   rows           >= 0.
 *   width          1 .. 2^17 - 1.
 *   outputs        1 .. 2^20.
 *   bias           device in, float[outputs], or NULL (0).
 *   gelu           0 or 1.
 *   y              device out, [rows][outputs]; rows that begin at multiples of 64
 *                  bytes are written fastest.
 */
flock_status linear_rows_i8(int32_t dtype, const int8_t *x, int64_t x_stride, const float *x_scale,
                            const int8_t *w, int64_t w_stride, const float *w_scale, int32_t rows, int32_t width,
                            int32_t outputs, const float *bias, int32_t gelu, void *y, int64_t y_stride,
                            void *stream);

/*
 * rotary_frames - rotary positions of queries and keys from time, y and x.
 *
 * Pair p of a head's dimensions is turned by angle_p = position * freq[p]:
 * the bird's time for the first n_time pairs, its y in px for the next n_y,
 * its x in px for the next n_x:
 *   (a, b) -> (a cos - b sin, a sin + b cos).
 * With P pairs in all, pair p is dimensions (p, p + P), or (2 p, 2 p + 1) where
 * interleaved; dimensions from 2 P on are copied.  inverse turns back, which is
 * the gradient of the turn.  Phases are integer products of position and
 * frequency (64-bit fractions of a turn), so far birds lose no digits.
 *
 * Arguments:
 *   dtype          FLOCK_F32, FLOCK_F16 or FLOCK_BF16.
 *   q, k           device in, [total][q_heads][head_dim], [total][k_heads][head_dim].
 *   q_heads, k_heads   0 .. 256 each (0: that tensor is not used), one at least.
 *   head_dim       1 .. 256.
 *   xy             device in, as for cluster_frames; NULL if n_y = n_x = 0.
 *   time           device in, int32[total]; NULL if n_time = 0.
 *   freq           host in, double[n_time + n_y + n_x], finite: radians per
 *                  unit of time, then per px.  Copied during the call.
 *   n_time, n_y, n_x   >= 0, 1 <= sum, 2 * sum <= head_dim.
 *   q_out, k_out   device out; may be q and k with the same strides (in place).
 */
flock_status rotary_frames(int32_t dtype, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                           int32_t total, int32_t q_heads, int32_t k_heads, int32_t head_dim,
                           const int32_t *xy, const int32_t *time, const double *freq, int32_t n_time,
                           int32_t n_y, int32_t n_x, int32_t interleaved, int32_t inverse, void *q_out,
                           int64_t q_out_stride, void *k_out, int64_t k_out_stride, void *stream);

/*
 * attention_frames - attention of queries over the keys of their frame.
 *
 * For query i and key j of frame f (indices within the frame, n_q queries and
 * n_k keys), query head h and its kv head h / (q_heads / kv_heads):
 *   t = scale * q_i . k_j;  with cap > 0: t = cap * tanh(t / cap)
 *   s = t - slopes[h] * |place_i - place_j|^2          (px^2, with slopes)
 *   seen: keep[j] != 0, and in causal frames j < prefix[f] or j <= i + n_k - n_q
 *   out_i = sum over the keys seen of softmax_j(s) v_j;  lse_i = log sum exp(s)
 * A query that sees no key gets zeros and lse -infinity.  Hidden keys' (keep =
 * 0) features are not read.  What order alone hides must be finite.
 * slopes = 1 / (2 sigma^2) weighs keys by the Gaussian that density_frames
 * adds per bird.  Products take 16-bit factors with 32-bit sums; the softmax
 * is in 32 bits, its weights rounded to dtype for the product with v.  A score's
 * distance may be a product of bfloat16 parts (without lse, and for the
 * gradients of k and v): that leaves a weight off by at most 7e-4 of itself in
 * bfloat16 and 2.5e-4 in float16, below its rounding.  With lse, and for the
 * gradient of q, distances are differences in 32 bits.
 *
 * Arguments:
 *   dtype          FLOCK_F16 or FLOCK_BF16.
 *   q, k, v        device in, [total_q][q_heads][head_dim] and
 *                  [total_k][kv_heads][head_dim], 16-byte aligned, strides
 *                  multiples of 8 below 2^24.
 *   n_frames       frames of both batches.  A batch whose tiles (of 32 or 128 rows
 *                  or keys of a frame and kv head) are 2^24 or more may be refused
 *                  (FLOCK_EUNSUPPORTED).
 *   q_offsets, k_offsets   device in, int32[n_frames + 1] each; the same array
 *                  where the birds of a frame attend to each other.
 *   q_heads, kv_heads      1 .. 256, q_heads a multiple of kv_heads.
 *   head_dim       8 .. 128, a multiple of 8.
 *   q_xy, k_xy     device in, int32[total][2], 1/16 px, with slopes.
 *   slopes         device in, float[q_heads], finite, or NULL.
 *   keep           device in, uint8[total_k], or NULL (all kept).
 *   causal         0 or 1.
 *   prefix         device in, int32[n_frames], or NULL (0); used when causal.
 *   scale, cap     finite; scale > 0, cap >= 0 (none: 0, or 2^96 and more).
 *   out            device out, [total_q][q_heads][head_dim].
 *   lse            device out, double[total_q][q_heads], or NULL: what the
 *                  backward pass takes.
 *   workspace      as for cluster_frames, sized by
 *                  attention_frames_workspace(...).
 */
flock_status attention_frames(int32_t dtype, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                              const void *v, int64_t v_stride, const int32_t *q_offsets,
                              const int32_t *k_offsets, int32_t n_frames, int32_t total_q, int32_t total_k,
                              int32_t q_heads, int32_t kv_heads, int32_t head_dim, const int32_t *q_xy,
                              const int32_t *k_xy, const float *slopes, const uint8_t *keep, int32_t causal,
                              const int32_t *prefix, float scale, float cap, void *out, int64_t out_stride,
                              double *lse, void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of workspace attention_frames needs for this batch shape (may be 0):
 * partial results where several workgroups share a query's keys. */
size_t attention_frames_workspace(int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads,
                                  int32_t kv_heads, int32_t head_dim);

/*
 * attention_frames_backward - gradients of attention_frames.
 *
 * Takes the forward call's arguments with its out and lse, and grad_out
 * [total_q][q_heads][head_dim]; writes grad_q, grad_k and grad_v (shaped as q,
 * k and v; the query heads of a kv head are summed), and with slopes
 * grad_slopes, float[q_heads] or NULL.  Hidden keys and queries without keys
 * get zeros.  Every sum has a fixed order: no atomics.
 * workspace: as for cluster_frames, sized by
 * attention_frames_backward_workspace(...).
 */
flock_status attention_frames_backward(
    int32_t dtype, const void *grad_out, int64_t grad_out_stride, const void *q, int64_t q_stride,
    const void *k, int64_t k_stride, const void *v, int64_t v_stride, const void *out, int64_t out_stride,
    const double *lse, const int32_t *q_offsets, const int32_t *k_offsets, int32_t n_frames, int32_t total_q,
    int32_t total_k, int32_t q_heads, int32_t kv_heads, int32_t head_dim, const int32_t *q_xy,
    const int32_t *k_xy, const float *slopes, const uint8_t *keep, int32_t causal, const int32_t *prefix,
    float scale, float cap, void *grad_q, int64_t grad_q_stride, void *grad_k, int64_t grad_k_stride,
    void *grad_v, int64_t grad_v_stride, float *grad_slopes, void *workspace, size_t workspace_bytes,
    void *stream);

/* Bytes of workspace attention_frames_backward needs for this batch shape. */
size_t attention_frames_backward_workspace(int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads,
                                           int32_t kv_heads, int32_t head_dim);

/*
 * Tracks: a paged cache of keys and values in 8 bits
 * --------------------------------------------------
 * What a bird's earlier detections leave for its later ones.  A cache is a pool of
 * pages of FLOCK_TRACK_PAGE tokens, of any track each:
 *   k          int8[pages][kv_heads][64][head_dim]
 *   v          int8[pages][kv_heads][head_dim][64], token t of the page at place
 *              16 * (t % 16 / 4) + 4 * (t / 16) + t % 4 of a dimension
 *   k_scale, v_scale   float[pages][kv_heads]: keys and values are the whole
 *              numbers times their page's and head's scale
 * k and v are 16-byte aligned; a new pool may hold anything.  A table says which
 * page holds which 64 tokens of a track:
 *   table      device in, int32[n_tracks][max_pages], rows table_stride apart:
 *              token t of track i is in page table[i][t / 64].  Numbers outside
 *              0 .. pages - 1 stand for no page: what would go there is not kept,
 *              and its tokens are not seen.
 *   lengths    device in, int32[n_tracks]: the tokens of each track, the batch's
 *              own among them, 0 .. 64 * max_pages.
 *   offsets    device in, int32[n_tracks + 1]: the batch's rows of each track,
 *              which are its last tokens, oldest first; none is allowed.
 * A track whose offsets or length are out of range is passed over: nothing is
 * appended, and its rows of outputs are left as they were.
 */
#define FLOCK_TRACK_PAGE 64

/*
 * append_tracks - keys and values of new detections into their tracks' pages.
 *
 * Keys are turned as by rotary_frames (in 32 bits, not rounded in between), and per
 * page and head, for keys and values alike,
 *   scale = max(the scale it has, if it holds earlier tokens; max |new| / 127)
 *   new tokens:  value / scale, to the nearest whole number, ties to even
 *   held tokens, where the scale grew:  whole number * (old scale / scale), likewise
 * with quotients in 32 bits.  A page's first token begins it anew, whatever its scale
 * was.  Places of tokens to come are left as they are.  A page that gets a value that is
 * not finite has scale NaN and zeros from then on; new tokens below 2^-100 are zeros.
 * Rows of one call must not meet in a page: where the table names a page for two
 * tracks, or twice for one, what it holds after both were appended to is undefined.
 * (Pages that tracks share may be read by all.)
 *
 * Arguments:
 *   dtype          FLOCK_F32, FLOCK_F16 or FLOCK_BF16: new_k, new_v.
 *   new_k, new_v   device in, [total][kv_heads][head_dim], strides >= 0.
 *   total          rows of all tracks; a track with more rows than `lengths`
 *                  has tokens is passed over.
 *   xy, time, freq, n_time, n_y, n_x, interleaved   as for rotary_frames, the
 *                  positions of the rows; without pairs (n_time + n_y + n_x = 0)
 *                  keys are not turned.
 *   k, v, k_scale, v_scale   device in and out: the cache.
 *   pages          >= 0.
 *   kv_heads       1 .. 256.
 *   head_dim       16 .. 128, a multiple of 16.
 *   max_pages      0 .. 2^24.
 */
flock_status append_tracks(int32_t dtype, const void *new_k, int64_t new_k_stride, const void *new_v,
                           int64_t new_v_stride, const int32_t *offsets, int32_t n_tracks, int32_t total,
                           const int32_t *table, int64_t table_stride, int32_t max_pages, const int32_t *lengths,
                           const int32_t *xy, const int32_t *time, const double *freq, int32_t n_time, int32_t n_y,
                           int32_t n_x, int32_t interleaved, int8_t *k, int8_t *v, float *k_scale, float *v_scale,
                           int32_t pages, int32_t kv_heads, int32_t head_dim, void *stream);

/*
 * attention_tracks - attention of the newest detections of tracks over their pages.
 *
 * For query i of n of a track (its last n of `length` tokens, p_i = length - n + i)
 * and token j, query head h and its kv head h / (q_heads / kv_heads):
 *   t = scale * q_i . k_j;  with cap > 0: t = cap * tanh(t / cap)
 *   seen: j <= p_i, and with window > 0: j > p_i - window
 *   out_i = sum over the tokens seen of softmax_j(t) v_j
 * A query that sees no token gets zeros.  Keys and values are taken as the whole
 * numbers they are, with products in 32-bit sums and a softmax in 32 bits.  A query's
 * dimension is rounded by at most 1/64000 of its head's largest (a head whose largest is
 * below 2^-100 is zeros, one that is not finite gives NaN), and weights are rounded to 11
 * bits for the product with v, those below 2^-17 of their row's largest to 2^-28 of it,
 * whatever the scales of other pages (up to 2^100 apart).  Weights times values are summed
 * before they are divided by the weights' sum, so those sums have to be below 2^128.
 * Scales are >= 0, or NaN: then what sees the page is NaN.
 *
 * Arguments:
 *   dtype          FLOCK_F16 or FLOCK_BF16: q, out.
 *   q              device in, [total][q_heads][head_dim], stride >= 0; turned by
 *                  rotary_frames where keys were.
 *   window         >= 0; 0: all tokens up to the query's own.
 *   scale, cap     finite; scale > 0, cap >= 0 (none: 0, or 2^96 and more).
 *   out            device out, [total][q_heads][head_dim].
 *   workspace      as for cluster_frames, sized by attention_tracks_workspace(...).
 * Others as for append_tracks; q_heads is 1 .. 256, a multiple of kv_heads.  A batch
 * of more workgroups than a launch holds is refused (FLOCK_EUNSUPPORTED).
 */
flock_status attention_tracks(int32_t dtype, const void *q, int64_t q_stride, const int32_t *offsets,
                              int32_t n_tracks, int32_t total, const int32_t *table, int64_t table_stride,
                              int32_t max_pages, const int32_t *lengths, const int8_t *k, const int8_t *v,
                              const float *k_scale, const float *v_scale, int32_t pages, int32_t q_heads,
                              int32_t kv_heads, int32_t head_dim, int32_t window, float scale, float cap, void *out,
                              int64_t out_stride, void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of workspace attention_tracks needs for this batch shape (may be 0):
 * partial results where several workgroups share a row's pages. */
size_t attention_tracks_workspace(int32_t n_tracks, int32_t total, int32_t max_pages, int32_t q_heads,
                                  int32_t kv_heads, int32_t head_dim);

/* Text of the last error on this thread ("" if none); valid until the next
 * library call on this thread. */
const char *flock_last_error(void);

/* Library version string, e.g. "flock 0.1.0 gfx950". */
const char *flock_version(void);

#ifdef __cplusplus
}
#endif

#endif /* FLOCK_H */
