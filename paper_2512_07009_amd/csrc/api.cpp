// api.cpp - the C ABI of libflock (declared in include/flock.h): argument
// validation, launch planning and error reporting.  No computation happens
// here; every step of the path runs in the HIP kernels.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <memory>
#include <mutex>
#include <new>
#include <string>
#include <vector>

#include "flock.h"
#include "internal.h"

namespace {

thread_local char g_error[512];

flock_status fail(flock_status st, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof g_error, fmt, ap);
    va_end(ap);
    return st;
}

flock_status hip_fail(hipError_t err, const char *what) {
    return fail(FLOCK_EDEVICE, "%s: %s", what, hipGetErrorString(err));
}

struct DeviceInfo {
    bool valid = false;
    bool gfx950 = false;
    int n_cus = 0;
    size_t lds_per_block = 0;
    size_t lds_per_cu = 0;
    char arch[64] = {0};
};

constexpr int kMaxDevices = 64;
DeviceInfo g_devices[kMaxDevices];
std::once_flag g_device_once[kMaxDevices];

flock_status device_info(const DeviceInfo **out) {
    int dev = 0;
    hipError_t err = hipGetDevice(&dev);
    if (err != hipSuccess) return hip_fail(err, "hipGetDevice");
    if (dev < 0 || dev >= kMaxDevices) return fail(FLOCK_EUNSUPPORTED, "device index %d", dev);
    std::call_once(g_device_once[dev], [dev] {
        hipDeviceProp_t prop;
        if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return;
        DeviceInfo &d = g_devices[dev];
        std::snprintf(d.arch, sizeof d.arch, "%s", prop.gcnArchName);
        d.gfx950 = std::strncmp(prop.gcnArchName, "gfx950", 6) == 0;
        d.n_cus = prop.multiProcessorCount;
        d.lds_per_block = prop.sharedMemPerBlock;
        d.lds_per_cu = prop.maxSharedMemoryPerMultiProcessor;
        d.valid = true;
    });
    const DeviceInfo &d = g_devices[dev];
    if (!d.valid) return fail(FLOCK_EDEVICE, "could not read properties of device %d", dev);
    if (!d.gfx950) return fail(FLOCK_EUNSUPPORTED, "device %d is %s; this library is built for gfx950", dev, d.arch);
    *out = &d;
    return FLOCK_OK;
}

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

bool validate_requested() {
    const char *v = std::getenv("FLOCK_VALIDATE");
    return v && v[0] == '1';
}

// Debug mode: copy offsets (and coordinates) to the host and check them.
flock_status validate_batch(const int32_t *xy, const int32_t *offsets, int32_t n_frames, int32_t total,
                            hipStream_t stream) {
    std::vector<int32_t> off((size_t)n_frames + 1);
    hipError_t err = hipMemcpyAsync(off.data(), offsets, off.size() * sizeof(int32_t),
                                    hipMemcpyDeviceToHost, stream);
    if (err == hipSuccess) err = hipStreamSynchronize(stream);
    if (err != hipSuccess) return hip_fail(err, "FLOCK_VALIDATE offsets copy");
    if (off[0] != 0) return fail(FLOCK_EINVAL, "offsets[0] = %d, expected 0", off[0]);
    for (int32_t f = 0; f < n_frames; ++f)
        if (off[f + 1] < off[f]) return fail(FLOCK_EINVAL, "offsets decrease at frame %d", f);
    if (off[n_frames] != total)
        return fail(FLOCK_EINVAL, "offsets[n_frames] = %d but total = %d", off[n_frames], total);
    if (total > 0) {
        std::vector<int32_t> h((size_t)total * 2);
        err = hipMemcpyAsync(h.data(), xy, h.size() * sizeof(int32_t), hipMemcpyDeviceToHost, stream);
        if (err == hipSuccess) err = hipStreamSynchronize(stream);
        if (err != hipSuccess) return hip_fail(err, "FLOCK_VALIDATE xy copy");
        for (size_t i = 0; i < h.size(); ++i)
            if (h[i] < 0 || h[i] >= (1 << 24))
                return fail(FLOCK_EINVAL, "coordinate %d of bird %zu outside [0, 2^24)", h[i], i / 2);
    }
    return FLOCK_OK;
}

// Largest s >= 1 with 2 s^2 <= e^2 (cell side whose diagonal is <= e).
int32_t diagonal_cell_side(int32_t e) {
    const int64_t half = (int64_t)e * e / 2;
    int64_t s = (int64_t)std::sqrt((double)half);
    while (s * s > half) --s;
    while ((s + 1) * (s + 1) <= half) ++s;
    return s < 1 ? 1 : (int32_t)s;
}

// The on-chip kernel's neighbour-cell tables for cells of side `side`
// (offsets (dx, dy), |dx|, |dy| <= reach <= 2, whose cells can hold points
// within e: gap(|dx|)^2 + gap(|dy|)^2 <= e^2, gap(d) = (d - 1) side + 1 for
// d > 0).  Whole stencil by gap distance, ties in row-major order; forward
// half (dy > 0, or dy = 0 and dx > 0) with the adjacent cells first.
void pack_stencil(int32_t e, int32_t side, flock::ClusterArgs *a) {
    const int reach = e == 0 ? 0 : std::min(1 + (e - 1) / side, 7);
    auto gap = [side](int d) -> int64_t { d = d < 0 ? -d : d; return d == 0 ? 0 : (int64_t)(d - 1) * side + 1; };
    struct Off { int dx, dy; int64_t key; int idx; };
    std::vector<Off> all, adj, far;
    int rowcnt[3] = {0, 0, 0};
    for (int idx = 0; idx < 25; ++idx) {
        const int dx = idx % 5 - 2, dy = idx / 5 - 2;
        if (std::abs(dx) > reach || std::abs(dy) > reach) continue;
        const int64_t d = gap(dx) * gap(dx) + gap(dy) * gap(dy);
        if (d > (int64_t)e * e) continue;
        all.push_back({dx, dy, d, idx});
        if (dy >= 0) rowcnt[dy]++;
        if (dy > 0 || (dy == 0 && dx > 0)) (std::abs(dx) <= 1 && std::abs(dy) <= 1 ? adj : far).push_back({dx, dy, d, idx});
    }
    std::stable_sort(all.begin(), all.end(), [](const Off &x, const Off &y) { return x.key < y.key; });
    auto code = [](const Off &o) { return (uint32_t)((o.dx + 2) | ((o.dy + 2) << 3)); };
    for (uint32_t &w : a->sten_all) w = 0;
    for (uint32_t &w : a->sten_fwd) w = 0;
    for (size_t i = 0; i < all.size(); ++i) a->sten_all[i / 5] |= code(all[i]) << (6 * (i % 5));
    std::vector<Off> fwd = adj;
    fwd.insert(fwd.end(), far.begin(), far.end());
    for (size_t i = 0; i < fwd.size(); ++i) a->sten_fwd[i / 5] |= code(fwd[i]) << (6 * (i % 5));
    uint32_t meta = (uint32_t)all.size() | ((uint32_t)adj.size() << 8) | ((uint32_t)fwd.size() << 16);
    for (int k = 0; k < 3; ++k) meta |= (uint32_t)(rowcnt[k] > 0 ? (rowcnt[k] - 1) / 2 : 0) << (24 + 2 * k);
    a->sten_meta = meta;
}

struct ClusterPlan {
    int32_t cap_points;
    int32_t cap_cells;
    size_t lds_bytes;
    bool compact = false;  // two workgroups per compute unit
};

ClusterPlan plan_cluster(int32_t max_frame_points, size_t lds_limit) {
    ClusterPlan p;
    int32_t limit = flock::cluster_max_cap_points(lds_limit);
    // FLOCK_CLUSTER_CAP lowers the on-chip capacity (for tuning the split
    // between the on-chip and the multi-workgroup paths)
    const char *cap = std::getenv("FLOCK_CLUSTER_CAP");
    if (cap && std::atoi(cap) > 0) limit = std::min(limit, std::atoi(cap));
    p.cap_points = (max_frame_points > 0 && max_frame_points < limit) ? max_frame_points : limit;
    const size_t reserve = 1024;  // static shared variables
    const int64_t avail = (int64_t)lds_limit - (int64_t)reserve - 13 * (int64_t)p.cap_points - 4;
    int64_t cells = std::max<int64_t>(4096, 2 * (int64_t)p.cap_points);
    cells = std::min<int64_t>(cells, avail / 6);
    p.cap_cells = (int32_t)cells;
    p.lds_bytes = flock::cluster_lds_bytes(p.cap_points, p.cap_cells);
    return p;
}

// With more frames than compute units and frames of at most
// kClusterCompactCap points, two workgroups share a compute unit when half
// its LDS holds the frame with a cell table of at least kCompactMinCells
// entries (a 1080p frame at eps 40 px needs 2652).  A frame whose grid has
// more cells than the table runs on a coarsened grid (correct, slower).
// FLOCK_CLUSTER_COMPACT=0 turns this off.
constexpr int64_t kCompactMinCells = 2048;

void plan_compact(ClusterPlan *p, int32_t max_frame_points, int32_t n_frames, const DeviceInfo &dev) {
    const char *env = std::getenv("FLOCK_CLUSTER_COMPACT");
    if (env && std::strcmp(env, "0") == 0) return;
    if (n_frames <= dev.n_cus || max_frame_points <= 0 || max_frame_points > flock::kClusterCompactCap) return;
    if (max_frame_points > p->cap_points) return;
    const size_t half = (dev.lds_per_cu ? dev.lds_per_cu : dev.lds_per_block) / 2;
    const size_t fixed = flock::cluster_compact_static_lds() + 16;  // static variables, alignment
    const int64_t avail = (int64_t)half - (int64_t)fixed - 13 * (int64_t)max_frame_points - 4;
    const int64_t cells = std::min<int64_t>(avail / 6, 2 * (int64_t)max_frame_points + 4096);
    if (cells < kCompactMinCells) return;
    const size_t bytes = flock::cluster_lds_bytes(max_frame_points, (int32_t)cells);
    if (bytes + fixed > half) return;
    p->cap_points = max_frame_points;
    p->cap_cells = (int32_t)cells;
    p->lds_bytes = bytes;
    p->compact = true;
}

}  // namespace

extern "C" {

const char *flock_last_error(void) { return g_error; }

const char *flock_version(void) { return "flock 0.1.0 gfx950"; }

size_t cluster_frames_workspace(int32_t n_frames, int32_t total, int32_t max_frame_points) {
    if (n_frames <= 0 || total <= 0 || max_frame_points < 0) return 0;
    const DeviceInfo *dev = nullptr;
    size_t lds = 160 * 1024;
    if (device_info(&dev) == FLOCK_OK) lds = dev->lds_per_block;
    g_error[0] = '\0';
    const ClusterPlan plan = plan_cluster(max_frame_points, lds);
    const bool big = max_frame_points == 0 || max_frame_points > plan.cap_points;
    return big ? flock::cluster_big_workspace(n_frames, total) : 0;
}

size_t density_frames_workspace(int32_t n_frames, int32_t total, int32_t grid_w, int32_t grid_h) {
    const DeviceInfo *dev = nullptr;
    int n_cus = 256;
    if (device_info(&dev) == FLOCK_OK) n_cus = dev->n_cus;
    g_error[0] = '\0';
    return flock::density_workspace_bytes(n_frames, total, grid_w, grid_h, n_cus);
}

flock_status cluster_frames(const int32_t *xy, const int32_t *offsets, int32_t n_frames, int32_t total,
                            int32_t max_frame_points, int32_t eps_q, int32_t min_pts, int32_t *labels,
                            uint8_t *kind, int32_t *n_clusters, void *workspace, size_t workspace_bytes,
                            void *stream) {
    g_error[0] = '\0';
    if (n_frames < 0) return fail(FLOCK_EINVAL, "n_frames = %d < 0", n_frames);
    if (total < 0) return fail(FLOCK_EINVAL, "total = %d < 0", total);
    if (max_frame_points < 0) return fail(FLOCK_EINVAL, "max_frame_points = %d < 0", max_frame_points);
    if (eps_q < 0 || eps_q > 32766) return fail(FLOCK_EINVAL, "eps_q = %d outside [0, 32766]", eps_q);
    if (min_pts < 1) return fail(FLOCK_EINVAL, "min_pts = %d < 1", min_pts);
    if (n_frames == 0) return FLOCK_OK;
    if (!offsets) return fail(FLOCK_EINVAL, "offsets is NULL");
    if (total > 0 && (!xy || !labels || !kind))
        return fail(FLOCK_EINVAL, "xy, labels and kind must be non-NULL when total > 0");
    if (!aligned(xy, 8)) return fail(FLOCK_EINVAL, "xy must be 8-byte aligned");
    if (!aligned(offsets, 4) || !aligned(labels, 4) || !aligned(n_clusters, 4))
        return fail(FLOCK_EINVAL, "offsets, labels and n_clusters must be 4-byte aligned");
    if (total == 0 && !n_clusters) return FLOCK_OK;

    const DeviceInfo *dev = nullptr;
    flock_status st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (validate_requested()) {
        st = validate_batch(xy, offsets, n_frames, total, s);
        if (st != FLOCK_OK) return st;
    }

    ClusterPlan plan = plan_cluster(max_frame_points, dev->lds_per_block);
    const bool big = max_frame_points == 0 || max_frame_points > plan.cap_points;
    if (!big) plan_compact(&plan, max_frame_points, n_frames, *dev);
    const size_t ws_need = big ? flock::cluster_big_workspace(n_frames, total) : 0;
    if (workspace && workspace_bytes < ws_need)
        return fail(FLOCK_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, ws_need);
    if (workspace && !aligned(workspace, 256)) return fail(FLOCK_EINVAL, "workspace must be 256-byte aligned");
    flock::ClusterArgs a{};
    a.xy = xy;
    a.offsets = offsets;
    a.n_frames = n_frames;
    a.total = total;
    a.eps_q = eps_q;
    a.min_pts = min_pts;
    a.cell_side = diagonal_cell_side(eps_q);
    pack_stencil(eps_q, a.cell_side, &a);
    a.cap_points = plan.cap_points;
    a.cap_cells = plan.cap_cells;
    a.labels = labels;
    a.kind = kind;
    a.n_clusters = n_clusters;
    a.big_path = big ? 1 : 0;
    {
        // FLOCK_CLUSTER_UNION=lds takes the general union stage for every
        // frame (for tests of that path)
        const char *u = std::getenv("FLOCK_CLUSTER_UNION");
        a.union_regs = (u && std::strcmp(u, "lds") == 0) ? 0 : 1;
    }
    // one frame above the on-chip capacity (offsets[1] = total): the
    // multi-workgroup path alone, without an on-chip launch that would only
    // return
    a.big_all = big && n_frames == 1 && total > plan.cap_points ? 1 : 0;
    hipError_t err = hipSuccess;
    if (!a.big_all) {
        err = flock::launch_cluster_resident(a, plan.lds_bytes, plan.compact, s);
        if (err != hipSuccess) return hip_fail(err, "cluster kernel launch");
    }
    if (big && total > 0) {
        void *ws = workspace;
        if (!ws) {
            err = hipMallocAsync(&ws, ws_need, s);
            if (err != hipSuccess) return fail(FLOCK_ENOMEM, "hipMallocAsync(%zu): %s", ws_need,
                                               hipGetErrorString(err));
        }
        err = flock::launch_cluster_big(a, ws, s);
        if (!workspace) {
            const hipError_t ferr = hipFreeAsync(ws, s);
            if (err == hipSuccess) err = ferr;
        }
        if (err != hipSuccess) return hip_fail(err, "large-frame cluster kernels");
    }
    return FLOCK_OK;
}

}  // extern "C"

namespace {

// density_frames and density_frames_noalloc: the same checks, plan and
// kernels; they differ only in where a split launch keeps its partial grids
// (the caller's workspace or a library allocation, or the static scratch).
flock_status density_run(const int32_t *xy, const int32_t *offsets, int32_t n_frames, int32_t total,
                         int32_t max_frame_points, int32_t width_px, int32_t height_px, int32_t grid_w,
                         int32_t grid_h, float sigma_px, float *density, void *workspace,
                         size_t workspace_bytes, bool noalloc, void *stream) {
    g_error[0] = '\0';
    if (n_frames < 0) return fail(FLOCK_EINVAL, "n_frames = %d < 0", n_frames);
    if (total < 0) return fail(FLOCK_EINVAL, "total = %d < 0", total);
    if (max_frame_points < 0) return fail(FLOCK_EINVAL, "max_frame_points = %d < 0", max_frame_points);
    if (width_px < 1 || height_px < 1)
        return fail(FLOCK_EINVAL, "frame extent %d x %d px must be >= 1", width_px, height_px);
    if (grid_w < 1 || grid_h < 1 || grid_w > 4096 || grid_h > 4096)
        return fail(FLOCK_EINVAL, "grid %d x %d outside 1..4096", grid_w, grid_h);
    if (!std::isfinite(sigma_px) || !(sigma_px > 0.0f))
        return fail(FLOCK_EINVAL, "sigma_px must be finite and > 0");
    if (n_frames == 0) return FLOCK_OK;
    if (!offsets || !density) return fail(FLOCK_EINVAL, "offsets and density must be non-NULL");
    if (total > 0 && !xy) return fail(FLOCK_EINVAL, "xy is NULL with total > 0");
    if (!aligned(xy, 8)) return fail(FLOCK_EINVAL, "xy must be 8-byte aligned");
    if (!aligned(offsets, 4) || !aligned(density, 4))
        return fail(FLOCK_EINVAL, "offsets and density must be 4-byte aligned");

    const DeviceInfo *dev = nullptr;
    flock_status st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    // the debug check copies to the host and synchronises: never on the
    // allocation-free entry point, which may run under graph capture
    if (!noalloc && validate_requested()) {
        st = validate_batch(xy, offsets, n_frames, total, s);
        if (st != FLOCK_OK) return st;
    }

    flock::DensityArgs a;
    a.xy = xy;
    a.offsets = offsets;
    a.n_frames = n_frames;
    a.total = total;
    a.width_px = width_px;
    a.height_px = height_px;
    a.grid_w = grid_w;
    a.grid_h = grid_h;
    a.sigma_px = sigma_px;
    a.density = density;
    const flock::DensityPlan plan = flock::plan_density(a, dev->n_cus, workspace ? workspace_bytes : SIZE_MAX);
    if (plan.blocks > 0x7fffffffLL) return fail(FLOCK_EUNSUPPORTED, "batch too large for one launch");
    if (plan.lds_bytes > dev->lds_per_block)
        return fail(FLOCK_EUNSUPPORTED, "density kernel needs %zu bytes of LDS, the device has %zu", plan.lds_bytes,
                    dev->lds_per_block);
    // a split launch keeps partial grids in the workspace
    const size_t need = plan.split > 1 ? (size_t)n_frames * plan.split * (size_t)grid_w * grid_h * sizeof(float) : 0;
    void *ws = workspace;
    hipError_t err = hipSuccess;
    if (noalloc) {
        if (need > flock::kDensityScratchBytes)
            return fail(FLOCK_ENOMEM,
                        "this batch needs %zu bytes of partial grids, beyond the %zu bytes of static scratch "
                        "of the allocation-free entry point (density_frames with a workspace takes it)",
                        need, flock::kDensityScratchBytes);
        ws = nullptr;
        if (need > 0) {
            err = flock::density_static_scratch(&ws);
            if (err != hipSuccess || !ws) return hip_fail(err, "static scratch address");
        }
    } else {
        if (workspace && workspace_bytes < need)
            return fail(FLOCK_ENOMEM, "workspace of %zu bytes < %zu needed", workspace_bytes, need);
        if (workspace && !aligned(workspace, 256)) return fail(FLOCK_EINVAL, "workspace must be 256-byte aligned");
        if (need > 0 && !ws) {
            err = hipMallocAsync(&ws, need, s);
            if (err != hipSuccess) return hip_fail(err, "workspace allocation");
        }
    }
    err = flock::launch_density(a, plan, static_cast<float *>(ws), s);
    if (!noalloc && need > 0 && !workspace) {
        const hipError_t ferr = hipFreeAsync(ws, s);
        if (err == hipSuccess) err = ferr;
    }
    if (err != hipSuccess) return hip_fail(err, "density kernel launch");
    return FLOCK_OK;
}

}  // namespace

extern "C" {

flock_status density_frames(const int32_t *xy, const int32_t *offsets, int32_t n_frames, int32_t total,
                            int32_t max_frame_points, int32_t width_px, int32_t height_px,
                            int32_t grid_w, int32_t grid_h,
                            float sigma_px, float *density, void *workspace, size_t workspace_bytes,
                            void *stream) {
    return density_run(xy, offsets, n_frames, total, max_frame_points, width_px, height_px, grid_w, grid_h,
                       sigma_px, density, workspace, workspace_bytes, false, stream);
}

flock_status density_frames_noalloc(const int32_t *xy, const int32_t *offsets, int32_t n_frames, int32_t total,
                                    int32_t max_frame_points, int32_t width_px, int32_t height_px,
                                    int32_t grid_w, int32_t grid_h, float sigma_px, float *density,
                                    void *stream) {
    return density_run(xy, offsets, n_frames, total, max_frame_points, width_px, height_px, grid_w, grid_h,
                       sigma_px, density, nullptr, 0, true, stream);
}

size_t roi_filter_frames_workspace(int32_t n_frames, int32_t total) {
    g_error[0] = '\0';
    return n_frames > 0 ? flock::roi_workspace_bytes(total) : 0;  // flags, block counts and bases, staging
}

flock_status roi_filter_frames(const int32_t *xy, const int32_t *offsets, int32_t n_frames, int32_t total,
                               const int32_t *roi_xy, int32_t n_vertices, int32_t *counts, int32_t *out_xy,
                               int32_t *out_offsets, int32_t *out_index, void *workspace,
                               size_t workspace_bytes, void *stream) {
    g_error[0] = '\0';
    if (n_frames < 0) return fail(FLOCK_EINVAL, "n_frames = %d < 0", n_frames);
    if (total < 0) return fail(FLOCK_EINVAL, "total = %d < 0", total);
    if (n_vertices < 3 || n_vertices > flock::kRoiMaxVertices)
        return fail(FLOCK_EINVAL, "n_vertices = %d outside 3..%d", n_vertices, flock::kRoiMaxVertices);
    if (!roi_xy) return fail(FLOCK_EINVAL, "roi_xy must be non-NULL");
    flock::RoiArgs a;
    for (int v = 0; v < n_vertices; ++v) {
        const int32_t x = roi_xy[2 * v], y = roi_xy[2 * v + 1];
        if (x < -(1 << 24) || x > (1 << 24) || y < -(1 << 24) || y > (1 << 24))
            return fail(FLOCK_EINVAL, "roi vertex %d = (%d, %d) outside |coordinate| <= 2^24", v, x, y);
        a.vx[v] = x;
        a.vy[v] = y;
    }
    for (int v = n_vertices; v < flock::kRoiMaxVertices; ++v) a.vx[v] = a.vy[v] = 0;
    a.bx0 = *std::min_element(a.vx, a.vx + n_vertices);
    a.bx1 = *std::max_element(a.vx, a.vx + n_vertices);
    a.by0 = *std::min_element(a.vy, a.vy + n_vertices);
    a.by1 = *std::max_element(a.vy, a.vy + n_vertices);
    if (n_frames == 0) return FLOCK_OK;
    if (!offsets || !counts || !out_offsets) return fail(FLOCK_EINVAL, "offsets, counts and out_offsets must be non-NULL");
    if ((long long)total / flock::kRoiBlock + 1 > 0x7fffffffLL / 64)
        return fail(FLOCK_EUNSUPPORTED, "batch too large for one launch");
    if (total > 0 && (!xy || !out_xy)) return fail(FLOCK_EINVAL, "xy and out_xy must be non-NULL with total > 0");
    if (!aligned(xy, 8) || !aligned(out_xy, 8)) return fail(FLOCK_EINVAL, "xy and out_xy must be 8-byte aligned");
    if (!aligned(offsets, 4) || !aligned(counts, 4) || !aligned(out_offsets, 4) || !aligned(out_index, 4))
        return fail(FLOCK_EINVAL, "offsets, counts, out_offsets and out_index must be 4-byte aligned");

    const DeviceInfo *dev = nullptr;
    flock_status st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (validate_requested()) {
        st = validate_batch(xy, offsets, n_frames, total, s);
        if (st != FLOCK_OK) return st;
    }
    const size_t need = flock::roi_workspace_bytes(total);
    if (workspace && workspace_bytes < need)
        return fail(FLOCK_ENOMEM, "workspace of %zu bytes < %zu needed", workspace_bytes, need);
    if (workspace && !aligned(workspace, 256)) return fail(FLOCK_EINVAL, "workspace must be 256-byte aligned");
    void *ws = workspace;
    hipError_t err = hipSuccess;
    if (!ws && need > 0) {
        err = hipMallocAsync(&ws, need, s);
        if (err != hipSuccess) return hip_fail(err, "workspace allocation");
    }
    a.xy = xy;
    a.offsets = offsets;
    a.n_frames = n_frames;
    a.total = total;
    a.n_vertices = n_vertices;
    a.counts = counts;
    a.out_xy = out_xy;
    a.out_offsets = out_offsets;
    a.out_index = out_index;
    err = flock::launch_roi(a, ws, s);
    if (!workspace && need > 0) {
        const hipError_t ferr = hipFreeAsync(ws, s);
        if (err == hipSuccess) err = ferr;
    }
    if (err != hipSuccess) return hip_fail(err, "roi kernels");
    return FLOCK_OK;
}

size_t drinker_proximity_frames_workspace(int32_t n_frames, int32_t total) {
    g_error[0] = '\0';
    return n_frames > 0 ? flock::drink_workspace_bytes(total) : 0;  // block counts and bases
}

flock_status drinker_proximity_frames(const int32_t *xy, const int32_t *offsets, int32_t n_frames, int32_t total,
                                      const int32_t *lines, int32_t n_lines, int32_t threshold_q,
                                      uint8_t *drinking, int32_t *line, int32_t *counts, void *workspace,
                                      size_t workspace_bytes, void *stream) {
    g_error[0] = '\0';
    if (n_frames < 0) return fail(FLOCK_EINVAL, "n_frames = %d < 0", n_frames);
    if (total < 0) return fail(FLOCK_EINVAL, "total = %d < 0", total);
    if (n_lines < 1 || n_lines > flock::kDrinkMaxLines)
        return fail(FLOCK_EINVAL, "n_lines = %d outside 1..%d", n_lines, flock::kDrinkMaxLines);
    if (!lines) return fail(FLOCK_EINVAL, "lines must be non-NULL");
    if (threshold_q < 0 || threshold_q > (1 << 24))
        return fail(FLOCK_EINVAL, "threshold_q = %d outside 0..2^24", threshold_q);
    flock::DrinkArgs a;
    for (int l = 0; l < flock::kDrinkMaxLines; ++l) {
        if (l >= n_lines) {
            a.ax[l] = a.ay[l] = a.bx[l] = a.by[l] = 0;
            continue;
        }
        for (int k = 0; k < 4; ++k) {
            const int32_t v = lines[4 * l + k];
            if (v < -(1 << 24) || v > (1 << 24))
                return fail(FLOCK_EINVAL, "line %d coordinate %d outside |coordinate| <= 2^24", l, v);
        }
        a.ax[l] = lines[4 * l];
        a.ay[l] = lines[4 * l + 1];
        a.bx[l] = lines[4 * l + 2];
        a.by[l] = lines[4 * l + 3];
    }
    if (n_frames == 0) return FLOCK_OK;
    if (!offsets || !counts) return fail(FLOCK_EINVAL, "offsets and counts must be non-NULL");
    if (total > 0 && (!xy || !drinking)) return fail(FLOCK_EINVAL, "xy and drinking must be non-NULL with total > 0");
    if (!aligned(xy, 8)) return fail(FLOCK_EINVAL, "xy must be 8-byte aligned");
    if (!aligned(drinking, 16)) return fail(FLOCK_EINVAL, "drinking must be 16-byte aligned");
    if (!aligned(offsets, 4) || !aligned(counts, 4) || !aligned(line, 4))
        return fail(FLOCK_EINVAL, "offsets, counts and line must be 4-byte aligned");
    if ((long long)total / flock::kRoiBlock + 1 > 0x7fffffffLL / 64)
        return fail(FLOCK_EUNSUPPORTED, "batch too large for one launch");

    const DeviceInfo *dev = nullptr;
    flock_status st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (validate_requested()) {
        st = validate_batch(xy, offsets, n_frames, total, s);
        if (st != FLOCK_OK) return st;
    }
    const size_t need = flock::drink_workspace_bytes(total);
    if (workspace && workspace_bytes < need)
        return fail(FLOCK_ENOMEM, "workspace of %zu bytes < %zu needed", workspace_bytes, need);
    if (workspace && !aligned(workspace, 256)) return fail(FLOCK_EINVAL, "workspace must be 256-byte aligned");
    void *ws = workspace;
    hipError_t err = hipSuccess;
    if (!ws) {
        err = hipMallocAsync(&ws, need, s);
        if (err != hipSuccess) return hip_fail(err, "workspace allocation");
    }
    a.xy = xy;
    a.offsets = offsets;
    a.n_frames = n_frames;
    a.total = total;
    a.n_lines = n_lines;
    a.threshold = threshold_q;
    a.drinking = drinking;
    a.line = line;
    a.counts = counts;
    err = flock::launch_drinkers(a, ws, s);
    if (!workspace) {
        const hipError_t ferr = hipFreeAsync(ws, s);
        if (err == hipSuccess) err = ferr;
    }
    if (err != hipSuccess) return hip_fail(err, "drinker kernels");
    return FLOCK_OK;
}

}  // extern "C"

namespace {

// One workgroup per frame where the grid's forest fits in LDS, else the tiled
// kernels (FLOCK_HEATMAP_PATH=tiled takes them for every grid).
flock::HeatPlan heatmap_plan(int32_t grid_w, int32_t grid_h, const DeviceInfo &dev) {
    const char *hp = std::getenv("FLOCK_HEATMAP_PATH");
    if (hp && std::strcmp(hp, "tiled") == 0) return {0, false};
    return flock::plan_heatmap(grid_w, grid_h, dev.lds_per_block);
}

}  // namespace

extern "C" {

size_t heatmap_frames_workspace(int32_t n_frames, int32_t grid_w, int32_t grid_h) {
    const DeviceInfo *dev = nullptr;
    const bool known = device_info(&dev) == FLOCK_OK;
    g_error[0] = '\0';
    if (grid_w < 1 || grid_h < 1 || (known && heatmap_plan(grid_w, grid_h, *dev).slots > 0)) return 0;
    return flock::heatmap_workspace_bytes(n_frames, grid_w, grid_h);
}

flock_status heatmap_frames(const float *density, int32_t n_frames, int32_t grid_w, int32_t grid_h,
                            double cell_area_px2, float threshold, int32_t connectivity, int32_t *labels,
                            int32_t *n_components, double *entropy, double *degree, int32_t *comp_cells,
                            double *comp_mass, void *workspace, size_t workspace_bytes, void *stream) {
    g_error[0] = '\0';
    if (n_frames < 0) return fail(FLOCK_EINVAL, "n_frames = %d < 0", n_frames);
    if (grid_w < 1 || grid_h < 1 || grid_w > 4096 || grid_h > 4096)
        return fail(FLOCK_EINVAL, "grid %d x %d outside 1..4096", grid_w, grid_h);
    if (!std::isfinite(cell_area_px2) || cell_area_px2 < 0.0)
        return fail(FLOCK_EINVAL, "cell_area_px2 must be finite and >= 0");
    if (!std::isfinite(threshold) || !(threshold > 0.0f))
        return fail(FLOCK_EINVAL, "threshold must be finite and > 0");
    if (connectivity != 4 && connectivity != 8)
        return fail(FLOCK_EINVAL, "connectivity = %d, expected 4 or 8", connectivity);
    if (n_frames == 0) return FLOCK_OK;
    if (!density || !labels || !n_components || !entropy || !degree || !comp_cells || !comp_mass)
        return fail(FLOCK_EINVAL, "density and every output must be non-NULL");
    if (!aligned(density, 4) || !aligned(labels, 4) || !aligned(n_components, 4) || !aligned(comp_cells, 4))
        return fail(FLOCK_EINVAL, "density, labels, n_components and comp_cells must be 4-byte aligned");
    if (!aligned(entropy, 8) || !aligned(degree, 8) || !aligned(comp_mass, 8))
        return fail(FLOCK_EINVAL, "entropy, degree and comp_mass must be 8-byte aligned");
    const long long tiles = (long long)((grid_w + 31) / 32) * ((grid_h + 31) / 32) * n_frames;
    const long long cells = (long long)grid_w * grid_h * n_frames;
    if (tiles > 0x7fffffffLL || (cells + 255) / 256 > 0x7fffffffLL)
        return fail(FLOCK_EUNSUPPORTED, "batch too large for one launch");

    const DeviceInfo *dev = nullptr;
    flock_status st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const flock::HeatPlan plan = heatmap_plan(grid_w, grid_h, *dev);
    const size_t need = plan.slots > 0 ? 0 : flock::heatmap_workspace_bytes(n_frames, grid_w, grid_h);
    if (workspace && workspace_bytes < need)
        return fail(FLOCK_ENOMEM, "workspace of %zu bytes < %zu needed", workspace_bytes, need);
    if (workspace && !aligned(workspace, 256)) return fail(FLOCK_EINVAL, "workspace must be 256-byte aligned");
    void *ws = workspace;
    hipError_t err = hipSuccess;
    if (!ws && need > 0) {
        err = hipMallocAsync(&ws, need, s);
        if (err != hipSuccess) return hip_fail(err, "workspace allocation");
    }
    flock::HeatArgs a;
    a.density = density;
    a.n_frames = n_frames;
    a.grid_w = grid_w;
    a.grid_h = grid_h;
    a.tiles_x = a.tiles_y = 0;
    a.cell_area = cell_area_px2;
    a.threshold = threshold;
    a.connectivity = connectivity;
    a.labels = labels;
    a.n_components = n_components;
    a.entropy = entropy;
    a.degree = degree;
    a.comp_cells = comp_cells;
    a.comp_mass = comp_mass;
    err = flock::launch_heatmap(a, ws, plan, dev->n_cus, dev->lds_per_cu ? dev->lds_per_cu : dev->lds_per_block, s);
    if (!workspace && need > 0) {
        const hipError_t ferr = hipFreeAsync(ws, s);
        if (err == hipSuccess) err = ferr;
    }
    if (err != hipSuccess) return hip_fail(err, "heatmap kernels");
    return FLOCK_OK;
}

size_t mask_components_frames_workspace(int32_t n_frames, int32_t width, int32_t height, int32_t connectivity) {
    g_error[0] = '\0';
    return flock::mask_workspace_bytes(n_frames, width, height, connectivity);
}

flock_status mask_components_frames(const float *prob, int32_t n_frames, int32_t width, int32_t height,
                                    float threshold, int32_t connectivity, int32_t *labels,
                                    int32_t *n_components, int32_t *comp_offsets, int32_t capacity,
                                    int32_t *comp_label, int32_t *comp_area, int32_t *comp_box,
                                    double *comp_centroid, int32_t *comp_xy, float *comp_score, void *workspace,
                                    size_t workspace_bytes, void *stream) {
    g_error[0] = '\0';
    if (n_frames < 0) return fail(FLOCK_EINVAL, "n_frames = %d < 0", n_frames);
    if (width < 1 || height < 1 || width > 32768 || height > 32768)
        return fail(FLOCK_EINVAL, "frame %d x %d outside 1..32768", width, height);
    if (!std::isfinite(threshold) || !(threshold >= 0.0f))
        return fail(FLOCK_EINVAL, "threshold must be finite and >= 0");
    if (connectivity != 4 && connectivity != 8)
        return fail(FLOCK_EINVAL, "connectivity = %d, expected 4 or 8", connectivity);
    if (capacity < 0) return fail(FLOCK_EINVAL, "capacity = %d < 0", capacity);
    if ((long long)n_frames * width * height > 0x7fffffffLL)
        return fail(FLOCK_EUNSUPPORTED, "batch of %lld pixels above 2^31 - 1",
                    (long long)n_frames * width * height);
    if (n_frames == 0) return FLOCK_OK;
    if (!prob || !n_components || !comp_offsets)
        return fail(FLOCK_EINVAL, "prob, n_components and comp_offsets must be non-NULL");
    if (!aligned(prob, 4) || !aligned(labels, 4) || !aligned(n_components, 4) || !aligned(comp_offsets, 4) ||
        !aligned(comp_label, 4) || !aligned(comp_area, 4) || !aligned(comp_score, 4))
        return fail(FLOCK_EINVAL, "prob, labels, n_components, comp_offsets, comp_label, comp_area and "
                                  "comp_score must be 4-byte aligned");
    if (!aligned(comp_box, 16) || !aligned(comp_centroid, 16) || !aligned(comp_xy, 8))
        return fail(FLOCK_EINVAL, "comp_box and comp_centroid must be 16-byte aligned, comp_xy 8-byte aligned");

    const DeviceInfo *dev = nullptr;
    flock_status st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const size_t need = flock::mask_workspace_bytes(n_frames, width, height, connectivity);
    if (workspace && workspace_bytes < need)
        return fail(FLOCK_ENOMEM, "workspace of %zu bytes < %zu needed", workspace_bytes, need);
    if (workspace && !aligned(workspace, 256)) return fail(FLOCK_EINVAL, "workspace must be 256-byte aligned");
    void *ws = workspace;
    hipError_t err = hipSuccess;
    if (!ws) {
        err = hipMallocAsync(&ws, need, s);
        if (err != hipSuccess) return hip_fail(err, "workspace allocation");
    }
    flock::MaskArgs a{};
    a.prob = prob;
    a.n_frames = n_frames;
    a.width = width;
    a.height = height;
    a.threshold = threshold;
    a.connectivity = connectivity;
    a.labels = labels;
    a.n_components = n_components;
    a.comp_offsets = comp_offsets;
    a.capacity = capacity;
    a.comp_label = comp_label;
    a.comp_area = comp_area;
    a.comp_box = comp_box;
    a.comp_centroid = comp_centroid;
    a.comp_xy = comp_xy;
    a.comp_score = comp_score;
    err = flock::launch_mask(a, ws, s);
    if (!workspace) {
        const hipError_t ferr = hipFreeAsync(ws, s);
        if (err == hipSuccess) err = ferr;
    }
    if (err != hipSuccess) return hip_fail(err, "mask component kernels");
    return FLOCK_OK;
}

}  // extern "C"

// ----------------------------------------------------------------------------
// Per-bird encoder
// ----------------------------------------------------------------------------
namespace {

bool is_dtype(int32_t dtype) { return dtype == FLOCK_F32 || dtype == FLOCK_F16 || dtype == FLOCK_BF16; }

size_t dtype_size(int32_t dtype) { return dtype == FLOCK_F32 ? 4 : 2; }

// The caller's workspace, or a stream-ordered allocation that release() frees.
struct Workspace {
    void *ptr = nullptr;
    bool owned = false;

    flock_status take(void *workspace, size_t bytes, size_t need, hipStream_t s) {
        if (workspace && bytes < need) return fail(FLOCK_ENOMEM, "workspace of %zu bytes, %zu needed", bytes, need);
        if (workspace && !aligned(workspace, 256)) return fail(FLOCK_EINVAL, "workspace must be 256-byte aligned");
        ptr = workspace;
        if (!ptr && need > 0) {
            const hipError_t err = hipMallocAsync(&ptr, need, s);
            if (err != hipSuccess) return fail(FLOCK_ENOMEM, "hipMallocAsync(%zu): %s", need, hipGetErrorString(err));
            owned = true;
        }
        return FLOCK_OK;
    }
    hipError_t release(hipStream_t s) { return owned ? hipFreeAsync(ptr, s) : hipSuccess; }
};

int device_cus() {
    const DeviceInfo *dev = nullptr;
    const int n = device_info(&dev) == FLOCK_OK ? dev->n_cus : 256;
    g_error[0] = '\0';
    return n;
}

flock_status check_norm(int32_t dtype, int32_t rows, int32_t width) {
    if (!is_dtype(dtype)) return fail(FLOCK_EINVAL, "dtype = %d, expected FLOCK_F32, FLOCK_F16 or FLOCK_BF16", dtype);
    if (rows < 0) return fail(FLOCK_EINVAL, "rows = %d < 0", rows);
    if (width < 1 || width > (1 << 20)) return fail(FLOCK_EINVAL, "width = %d outside 1..2^20", width);
    return FLOCK_OK;
}

// The arguments that attention_frames and its backward pass share.
flock_status check_attention(int32_t dtype, const flock::AttentionArgs &a) {
    if (dtype != FLOCK_F16 && dtype != FLOCK_BF16)
        return fail(FLOCK_EINVAL, "dtype = %d, expected FLOCK_F16 or FLOCK_BF16", dtype);
    if (a.n_frames < 0) return fail(FLOCK_EINVAL, "n_frames = %d < 0", a.n_frames);
    if (a.total_q < 0 || a.total_k < 0)
        return fail(FLOCK_EINVAL, "total_q = %d, total_k = %d must be >= 0", a.total_q, a.total_k);
    if (a.kv_heads < 1 || a.kv_heads > 256 || a.q_heads < 1 || a.q_heads > 256)
        return fail(FLOCK_EINVAL, "q_heads = %d, kv_heads = %d outside 1..256", a.q_heads, a.kv_heads);
    if (a.q_heads % a.kv_heads)
        return fail(FLOCK_EINVAL, "q_heads = %d is not a multiple of kv_heads = %d", a.q_heads, a.kv_heads);
    if (a.dim < 8 || a.dim > flock::kAttentionMaxDim || a.dim % 8)
        return fail(FLOCK_EINVAL, "head_dim = %d is not a multiple of 8 in 8..%d", a.dim, flock::kAttentionMaxDim);
    if (a.causal != 0 && a.causal != 1) return fail(FLOCK_EINVAL, "causal = %d, expected 0 or 1", a.causal);
    if (!std::isfinite(a.scale) || !(a.scale > 0.0f)) return fail(FLOCK_EINVAL, "scale must be finite and > 0");
    if (!std::isfinite(a.cap) || !(a.cap >= 0.0f)) return fail(FLOCK_EINVAL, "cap must be finite and >= 0");
    if (a.q_stride < 0 || a.k_stride < 0 || a.v_stride < 0 || a.q_stride % 8 || a.k_stride % 8 || a.v_stride % 8)
        return fail(FLOCK_EINVAL, "strides of q, k and v must be multiples of 8, >= 0");
    if (a.q_stride > flock::kAttentionMaxStride || a.k_stride > flock::kAttentionMaxStride ||
        a.v_stride > flock::kAttentionMaxStride)
        return fail(FLOCK_EINVAL, "strides of q, k and v above %lld", (long long)flock::kAttentionMaxStride);
    if (a.out_stride < (int64_t)a.q_heads * a.dim || a.out_stride % 8)
        return fail(FLOCK_EINVAL, "out's stride must be a multiple of 8 that holds a row");
    return FLOCK_OK;
}

flock_status check_attention_pointers(const flock::AttentionArgs &a) {
    if (!a.q_offsets || !a.k_offsets) return fail(FLOCK_EINVAL, "q_offsets and k_offsets must be non-NULL");
    if (a.total_q > 0 && (!a.q || !a.out)) return fail(FLOCK_EINVAL, "q and out must be non-NULL when total_q > 0");
    if (a.total_k > 0 && (!a.k || !a.v)) return fail(FLOCK_EINVAL, "k and v must be non-NULL when total_k > 0");
    if (a.slopes && ((a.total_q > 0 && !a.q_xy) || (a.total_k > 0 && !a.k_xy)))
        return fail(FLOCK_EINVAL, "q_xy and k_xy must be non-NULL with slopes");
    if (!aligned(a.q, 16) || !aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.out, 16))
        return fail(FLOCK_EINVAL, "q, k, v and out must be 16-byte aligned");
    if (!aligned(a.q_xy, 8) || !aligned(a.k_xy, 8)) return fail(FLOCK_EINVAL, "q_xy and k_xy must be 8-byte aligned");
    if (!aligned(a.q_offsets, 4) || !aligned(a.k_offsets, 4) || !aligned(a.slopes, 4) || !aligned(a.prefix, 4))
        return fail(FLOCK_EINVAL, "q_offsets, k_offsets, slopes and prefix must be 4-byte aligned");
    if (!aligned(a.lse, 8)) return fail(FLOCK_EINVAL, "lse must be 8-byte aligned");
    // rows and keys are numbered in 31 bits, up to the end of the tile after the last
    if ((int64_t)a.total_q * a.group > 0x7fffff00LL || a.total_k > 0x7fffff00)
        return fail(FLOCK_EUNSUPPORTED, "batch of more than 2^31 - 256 keys, or rows of queries and shared heads");
    return FLOCK_OK;
}

flock_status check_workgroups(int64_t n) {
    if (n > flock::kMaxWorkgroups)
        return fail(FLOCK_EUNSUPPORTED, "batch of %lld workgroups, more than a launch's %lld: split its frames", (long long)n,
                    (long long)flock::kMaxWorkgroups);
    return FLOCK_OK;
}

flock_status validate_offsets(const char *name, const int32_t *offsets, int32_t n_frames, int32_t total,
                              hipStream_t stream) {
    const size_t n = (size_t)n_frames + 1;
    const std::unique_ptr<int32_t[]> off(new (std::nothrow) int32_t[n]);
    if (!off) return fail(FLOCK_ENOMEM, "no host memory for FLOCK_VALIDATE's copy of %s", name);
    hipError_t err = hipMemcpyAsync(off.get(), offsets, n * sizeof(int32_t), hipMemcpyDeviceToHost, stream);
    if (err == hipSuccess) err = hipStreamSynchronize(stream);
    if (err != hipSuccess) return hip_fail(err, "FLOCK_VALIDATE offsets copy");
    if (off[0] != 0) return fail(FLOCK_EINVAL, "%s[0] = %d, expected 0", name, off[0]);
    for (int32_t f = 0; f < n_frames; ++f)
        if (off[f + 1] < off[f]) return fail(FLOCK_EINVAL, "%s decrease at frame %d", name, f);
    if (off[n_frames] != total) return fail(FLOCK_EINVAL, "%s[n_frames] = %d but its total is %d", name, off[n_frames], total);
    return FLOCK_OK;
}

void rotary_steps(const double *freq, int32_t n_time, int32_t pairs, uint64_t *steps) {
    for (int32_t p = 0; p < pairs; ++p) {
        // turns per unit, whole turns dropped, in 2^-64 turns (rounded down to the double's last digit)
        double turns = freq[p] / (2.0 * 3.14159265358979323846) / (p < n_time ? 1.0 : 16.0);
        const bool back = turns < 0.0;
        turns = std::fmod(std::fabs(turns), 1.0);
        const uint64_t step = (uint64_t)std::ldexp(turns, 64);
        steps[p] = back ? 0 - step : step;
    }
}

// What append_tracks and attention_tracks share.
flock_status check_tracks(const flock::TrackArgs &t, const flock::TrackCacheArgs &c) {
    if (t.n_tracks < 0) return fail(FLOCK_EINVAL, "n_tracks = %d < 0", t.n_tracks);
    if (t.total < 0) return fail(FLOCK_EINVAL, "total = %d < 0", t.total);
    if (c.pages < 0) return fail(FLOCK_EINVAL, "pages = %d < 0", c.pages);
    if (t.max_pages < 0 || t.max_pages > flock::kTrackMaxPages)
        return fail(FLOCK_EINVAL, "max_pages = %d outside 0..%d", t.max_pages, flock::kTrackMaxPages);
    if (t.table_stride < 0) return fail(FLOCK_EINVAL, "table_stride = %lld < 0", (long long)t.table_stride);
    if (c.kv_heads < 1 || c.kv_heads > 256) return fail(FLOCK_EINVAL, "kv_heads = %d outside 1..256", c.kv_heads);
    if (c.dim < 16 || c.dim > flock::kAttentionMaxDim || c.dim % 16)
        return fail(FLOCK_EINVAL, "head_dim = %d is not a multiple of 16 in 16..%d", c.dim, flock::kAttentionMaxDim);
    return FLOCK_OK;
}

flock_status check_tracks_pointers(const flock::TrackArgs &t, const flock::TrackCacheArgs &c) {
    if (!t.offsets || !t.lengths) return fail(FLOCK_EINVAL, "offsets and lengths must be non-NULL");
    if (t.max_pages > 0 && !t.table) return fail(FLOCK_EINVAL, "table must be non-NULL when max_pages > 0");
    if (c.pages > 0 && (!c.k || !c.v || !c.k_scale || !c.v_scale))
        return fail(FLOCK_EINVAL, "k, v, k_scale and v_scale must be non-NULL when pages > 0");
    if (!aligned(c.k, 16) || !aligned(c.v, 16)) return fail(FLOCK_EINVAL, "k and v must be 16-byte aligned");
    if (!aligned(t.offsets, 4) || !aligned(t.lengths, 4) || !aligned(t.table, 4) || !aligned(c.k_scale, 4) || !aligned(c.v_scale, 4))
        return fail(FLOCK_EINVAL, "offsets, lengths, table, k_scale and v_scale must be 4-byte aligned");
    return FLOCK_OK;
}

flock_status validate_attention(const flock::AttentionArgs &a, hipStream_t s) {
    flock_status st = validate_offsets("q_offsets", a.q_offsets, a.n_frames, a.total_q, s);
    if (st == FLOCK_OK && a.k_offsets != a.q_offsets)
        st = validate_offsets("k_offsets", a.k_offsets, a.n_frames, a.total_k, s);
    else if (st == FLOCK_OK && a.total_k != a.total_q)
        st = fail(FLOCK_EINVAL, "k_offsets[n_frames] = %d but its total is %d", a.total_q, a.total_k);
    return st;
}

}  // namespace

extern "C" {

flock_status layer_norm_rows(int32_t dtype, const void *x, int64_t x_stride, const void *residual,
                             int64_t residual_stride, int32_t rows, int32_t width, const float *weight,
                             const float *bias, float eps, void *y, int64_t y_stride, void *sum, int64_t sum_stride,
                             float *mean, float *rstd, void *stream) {
    g_error[0] = '\0';
    flock_status st = check_norm(dtype, rows, width);
    if (st != FLOCK_OK) return st;
    if (!std::isfinite(eps) || !(eps >= 0.0f)) return fail(FLOCK_EINVAL, "eps must be finite and >= 0");
    if (x_stride < 0 || (residual && residual_stride < 0)) return fail(FLOCK_EINVAL, "input strides must be >= 0");
    if (y_stride < width || (residual && sum_stride < width))
        return fail(FLOCK_EINVAL, "output strides must hold a row");
    if (rows == 0) return FLOCK_OK;
    if (!x || !y) return fail(FLOCK_EINVAL, "x and y must be non-NULL");
    if (residual && !sum) return fail(FLOCK_EINVAL, "sum must be non-NULL with residual");
    const size_t size = dtype_size(dtype);
    if (!aligned(x, size) || !aligned(y, size) || !aligned(residual, size) || !aligned(sum, size))
        return fail(FLOCK_EINVAL, "x, residual, y and sum must be aligned to their elements");
    if (!aligned(weight, 4) || !aligned(bias, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return fail(FLOCK_EINVAL, "weight, bias, mean and rstd must be 4-byte aligned");
    const DeviceInfo *dev = nullptr;
    st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    flock::NormArgs a{};
    a.x = x;
    a.x_stride = x_stride;
    a.residual = residual;
    a.residual_stride = residual ? residual_stride : 0;
    a.rows = rows;
    a.width = width;
    a.weight = weight;
    a.bias = bias;
    a.eps = eps;
    a.y = y;
    a.y_stride = y_stride;
    a.sum = residual ? sum : nullptr;
    a.sum_stride = residual ? sum_stride : 0;
    a.mean = mean;
    a.rstd = rstd;
    const hipError_t err = flock::launch_norm(a, dtype, reinterpret_cast<hipStream_t>(stream));
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "layer norm kernel launch");
}

size_t layer_norm_rows_backward_workspace(int32_t rows, int32_t width) {
    return flock::norm_backward_workspace_bytes(rows, width, device_cus());
}

flock_status layer_norm_rows_backward(int32_t dtype, const void *grad_y, int64_t grad_y_stride, const void *grad_sum,
                                      int64_t grad_sum_stride, const void *x, int64_t x_stride, int32_t rows,
                                      int32_t width, const float *weight, const float *mean, const float *rstd,
                                      void *grad_x, int64_t grad_x_stride, float *grad_weight, float *grad_bias,
                                      void *workspace, size_t workspace_bytes, void *stream) {
    g_error[0] = '\0';
    flock_status st = check_norm(dtype, rows, width);
    if (st != FLOCK_OK) return st;
    if (grad_y_stride < 0 || x_stride < 0 || (grad_sum && grad_sum_stride < 0))
        return fail(FLOCK_EINVAL, "input strides must be >= 0");
    if (grad_x_stride < width) return fail(FLOCK_EINVAL, "output strides must hold a row");
    if (rows > 0 && (!grad_y || !x || !mean || !rstd || !grad_x))
        return fail(FLOCK_EINVAL, "grad_y, x, mean, rstd and grad_x must be non-NULL");
    const size_t size = dtype_size(dtype);
    if (!aligned(grad_y, size) || !aligned(x, size) || !aligned(grad_sum, size) || !aligned(grad_x, size))
        return fail(FLOCK_EINVAL, "grad_y, grad_sum, x and grad_x must be aligned to their elements");
    if (!aligned(weight, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(grad_weight, 4) || !aligned(grad_bias, 4))
        return fail(FLOCK_EINVAL, "weight, mean, rstd, grad_weight and grad_bias must be 4-byte aligned");
    if (rows == 0 && !grad_weight && !grad_bias) return FLOCK_OK;
    const DeviceInfo *dev = nullptr;
    st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const bool columns = grad_weight || grad_bias;
    Workspace ws;
    st = ws.take(workspace, workspace_bytes,
                 columns ? flock::norm_backward_workspace_bytes(rows, width, dev->n_cus) : 0, s);
    if (st != FLOCK_OK) return st;
    flock::NormBackwardArgs a{};
    a.grad_y = grad_y;
    a.grad_y_stride = grad_y_stride;
    a.grad_sum = grad_sum;
    a.grad_sum_stride = grad_sum ? grad_sum_stride : 0;
    a.x = x;
    a.x_stride = x_stride;
    a.rows = rows;
    a.width = width;
    a.weight = weight;
    a.mean = mean;
    a.rstd = rstd;
    a.grad_x = grad_x;
    a.grad_x_stride = grad_x_stride;
    hipError_t err = flock::launch_norm_backward(a, dtype, ws.ptr, dev->n_cus, grad_weight, grad_bias, s);
    const hipError_t ferr = ws.release(s);
    if (err == hipSuccess) err = ferr;
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "layer norm backward kernels");
}

static flock_status rms_rows(int32_t dtype, flock::RmsArgs a, int32_t rows, void *stream) {
    g_error[0] = '\0';
    flock_status st = check_norm(dtype, rows, a.width);
    if (st != FLOCK_OK) return st;
    if (!std::isfinite(a.eps) || !(a.eps >= 0.0f)) return fail(FLOCK_EINVAL, "eps must be finite and >= 0");
    if (a.x_stride < 0 || (a.residual && a.residual_stride < 0)) return fail(FLOCK_EINVAL, "input strides must be >= 0");
    if (a.y_stride < a.width || (a.residual && a.sum_stride < a.width))
        return fail(FLOCK_EINVAL, "output strides must hold a row");
    if (rows == 0) return FLOCK_OK;
    if (!a.x || !a.y) return fail(FLOCK_EINVAL, "x and the output must be non-NULL");
    if (a.residual && !a.sum) return fail(FLOCK_EINVAL, "sum must be non-NULL with residual");
    const size_t size = dtype_size(dtype);
    if (!aligned(a.x, size) || (!a.scale && !aligned(a.y, size)) || !aligned(a.residual, size) || !aligned(a.sum, size))
        return fail(FLOCK_EINVAL, "x, residual, y and sum must be aligned to their elements");
    if (!aligned(a.weight, 4) || !aligned(a.rstd, 4) || !aligned(a.scale, 4))
        return fail(FLOCK_EINVAL, "weight, rstd and scale must be 4-byte aligned");
    const DeviceInfo *dev = nullptr;
    st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    a.rows = rows;
    if (!a.residual) {
        a.sum = nullptr;
        a.residual_stride = a.sum_stride = 0;
    }
    const hipError_t err = flock::launch_rms(a, dtype, reinterpret_cast<hipStream_t>(stream));
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "root-mean-square norm kernel launch");
}

flock_status rms_norm_rows(int32_t dtype, const void *x, int64_t x_stride, const void *residual,
                           int64_t residual_stride, int32_t rows, int32_t width, const float *weight, float eps,
                           void *y, int64_t y_stride, void *sum, int64_t sum_stride, float *rstd, void *stream) {
    flock::RmsArgs a{};
    a.x = x;
    a.x_stride = x_stride;
    a.residual = residual;
    a.residual_stride = residual_stride;
    a.width = width;
    a.weight = weight;
    a.eps = eps;
    a.y = y;
    a.y_stride = y_stride;
    a.sum = sum;
    a.sum_stride = sum_stride;
    a.rstd = rstd;
    return rms_rows(dtype, a, rows, stream);
}

flock_status rms_norm_rows_i8(int32_t dtype, const void *x, int64_t x_stride, const void *residual,
                              int64_t residual_stride, int32_t rows, int32_t width, const float *weight, float eps,
                              int8_t *q, int64_t q_stride, float *scale, void *sum, int64_t sum_stride, void *stream) {
    g_error[0] = '\0';
    if (rows > 0 && !scale) return fail(FLOCK_EINVAL, "scale must be non-NULL");
    flock::RmsArgs a{};
    a.x = x;
    a.x_stride = x_stride;
    a.residual = residual;
    a.residual_stride = residual_stride;
    a.width = width;
    a.weight = weight;
    a.eps = eps;
    a.y = q;
    a.y_stride = q_stride;
    a.sum = sum;
    a.sum_stride = sum_stride;
    a.scale = scale;
    return rms_rows(dtype, a, rows, stream);
}

flock_status quantize_rows(int32_t dtype, const void *x, int64_t x_stride, int32_t rows, int32_t width, int8_t *q,
                           int64_t q_stride, float *scale, void *stream) {
    g_error[0] = '\0';
    if (rows > 0 && !scale) return fail(FLOCK_EINVAL, "scale must be non-NULL");
    flock::RmsArgs a{};
    a.x = x;
    a.x_stride = x_stride;
    a.width = width;
    a.y = q;
    a.y_stride = q_stride;
    a.scale = scale;
    a.as_is = 1;
    return rms_rows(dtype, a, rows, stream);
}

size_t rms_norm_rows_backward_workspace(int32_t rows, int32_t width) {
    return flock::rms_backward_workspace_bytes(rows, width, device_cus());
}

flock_status rms_norm_rows_backward(int32_t dtype, const void *grad_y, int64_t grad_y_stride, const void *grad_sum,
                                    int64_t grad_sum_stride, const void *x, int64_t x_stride, int32_t rows, int32_t width,
                                    const float *weight, const float *rstd, void *grad_x, int64_t grad_x_stride,
                                    float *grad_weight, void *workspace, size_t workspace_bytes, void *stream) {
    g_error[0] = '\0';
    flock_status st = check_norm(dtype, rows, width);
    if (st != FLOCK_OK) return st;
    if (grad_y_stride < 0 || x_stride < 0 || (grad_sum && grad_sum_stride < 0))
        return fail(FLOCK_EINVAL, "input strides must be >= 0");
    if (grad_x_stride < width) return fail(FLOCK_EINVAL, "output strides must hold a row");
    if (rows > 0 && (!grad_y || !x || !rstd || !grad_x))
        return fail(FLOCK_EINVAL, "grad_y, x, rstd and grad_x must be non-NULL");
    const size_t size = dtype_size(dtype);
    if (!aligned(grad_y, size) || !aligned(x, size) || !aligned(grad_sum, size) || !aligned(grad_x, size))
        return fail(FLOCK_EINVAL, "grad_y, grad_sum, x and grad_x must be aligned to their elements");
    if (!aligned(weight, 4) || !aligned(rstd, 4) || !aligned(grad_weight, 4))
        return fail(FLOCK_EINVAL, "weight, rstd and grad_weight must be 4-byte aligned");
    if (rows == 0 && !grad_weight) return FLOCK_OK;
    const DeviceInfo *dev = nullptr;
    st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    Workspace ws;
    st = ws.take(workspace, workspace_bytes,
                 grad_weight ? flock::rms_backward_workspace_bytes(rows, width, dev->n_cus) : 0, s);
    if (st != FLOCK_OK) return st;
    flock::RmsBackwardArgs a{};
    a.grad_y = grad_y;
    a.grad_y_stride = grad_y_stride;
    a.grad_sum = grad_sum;
    a.grad_sum_stride = grad_sum ? grad_sum_stride : 0;
    a.x = x;
    a.x_stride = x_stride;
    a.rows = rows;
    a.width = width;
    a.weight = weight;
    a.rstd = rstd;
    a.grad_x = grad_x;
    a.grad_x_stride = grad_x_stride;
    hipError_t err = flock::launch_rms_backward(a, dtype, ws.ptr, dev->n_cus, grad_weight, s);
    const hipError_t ferr = ws.release(s);
    if (err == hipSuccess) err = ferr;
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "root-mean-square norm backward kernels");
}

flock_status linear_rows_i8(int32_t dtype, const int8_t *x, int64_t x_stride, const float *x_scale, const int8_t *w,
                            int64_t w_stride, const float *w_scale, int32_t rows, int32_t width, int32_t outputs,
                            const float *bias, int32_t gelu, void *y, int64_t y_stride, void *stream) {
    g_error[0] = '\0';
    if (!is_dtype(dtype)) return fail(FLOCK_EINVAL, "dtype = %d, expected FLOCK_F32, FLOCK_F16 or FLOCK_BF16", dtype);
    if (rows < 0) return fail(FLOCK_EINVAL, "rows = %d < 0", rows);
    if (width < 1 || width > flock::kLinearMaxWidth)
        return fail(FLOCK_EINVAL, "width = %d outside 1..%d", width, flock::kLinearMaxWidth);
    if (outputs < 1 || outputs > (1 << 20)) return fail(FLOCK_EINVAL, "outputs = %d outside 1..2^20", outputs);
    if (gelu != 0 && gelu != 1) return fail(FLOCK_EINVAL, "gelu = %d, expected 0 or 1", gelu);
    if (x_stride < 0 || w_stride < 0 || x_stride > flock::kLinearMaxStride || w_stride > flock::kLinearMaxStride)
        return fail(FLOCK_EINVAL, "strides of x and w outside 0..%lld", (long long)flock::kLinearMaxStride);
    if (y_stride < outputs) return fail(FLOCK_EINVAL, "y's stride must hold a row");
    if (rows == 0) return FLOCK_OK;
    if (!x || !x_scale || !w || !w_scale || !y)
        return fail(FLOCK_EINVAL, "x, x_scale, w, w_scale and y must be non-NULL");
    if (!aligned(y, dtype_size(dtype))) return fail(FLOCK_EINVAL, "y must be aligned to its elements");
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4))
        return fail(FLOCK_EINVAL, "x_scale, w_scale and bias must be 4-byte aligned");
    const DeviceInfo *dev = nullptr;
    const flock_status st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    flock::LinearArgs a{};
    a.x = x;
    a.w = w;
    a.x_stride = x_stride;
    a.w_stride = w_stride;
    a.rows = rows;
    a.width = width;
    a.outputs = outputs;
    a.x_scale = x_scale;
    a.w_scale = w_scale;
    a.bias = bias;
    a.gelu = gelu;
    a.y = y;
    a.y_stride = y_stride;
    const hipError_t err = flock::launch_linear(a, dtype, dev->n_cus, reinterpret_cast<hipStream_t>(stream));
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "linear kernel launch");
}

flock_status rotary_frames(int32_t dtype, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                           int32_t total, int32_t q_heads, int32_t k_heads, int32_t head_dim, const int32_t *xy,
                           const int32_t *time, const double *freq, int32_t n_time, int32_t n_y, int32_t n_x,
                           int32_t interleaved, int32_t inverse, void *q_out, int64_t q_out_stride, void *k_out,
                           int64_t k_out_stride, void *stream) {
    g_error[0] = '\0';
    if (!is_dtype(dtype)) return fail(FLOCK_EINVAL, "dtype = %d, expected FLOCK_F32, FLOCK_F16 or FLOCK_BF16", dtype);
    if (total < 0) return fail(FLOCK_EINVAL, "total = %d < 0", total);
    if (q_heads < 0 || q_heads > 256 || k_heads < 0 || k_heads > 256 || q_heads + k_heads < 1)
        return fail(FLOCK_EINVAL, "q_heads = %d, k_heads = %d outside 0..256, or none", q_heads, k_heads);
    if (head_dim < 1 || head_dim > 2 * flock::kRotaryMaxPairs)
        return fail(FLOCK_EINVAL, "head_dim = %d outside 1..%d", head_dim, 2 * flock::kRotaryMaxPairs);
    if (n_time < 0 || n_y < 0 || n_x < 0 || (int64_t)n_time + n_y + n_x < 1 ||
        2 * ((int64_t)n_time + n_y + n_x) > head_dim)
        return fail(FLOCK_EINVAL, "n_time = %d, n_y = %d, n_x = %d pairs do not fit head_dim = %d", n_time, n_y, n_x,
                    head_dim);
    if (!freq) return fail(FLOCK_EINVAL, "freq is NULL");
    const int32_t pairs = n_time + n_y + n_x;
    for (int32_t p = 0; p < pairs; ++p)
        if (!std::isfinite(freq[p])) return fail(FLOCK_EINVAL, "freq[%d] is not finite", p);
    if ((q_heads && (q_stride < 0 || q_out_stride < (int64_t)q_heads * head_dim)) ||
        (k_heads && (k_stride < 0 || k_out_stride < (int64_t)k_heads * head_dim)))
        return fail(FLOCK_EINVAL, "strides must be >= 0, and hold a row for outputs");
    if ((q_heads && q == q_out && q_stride != q_out_stride) || (k_heads && k == k_out && k_stride != k_out_stride))
        if (total > 0 && (q || k)) return fail(FLOCK_EINVAL, "an output in place has its input's stride");
    if (total == 0) return FLOCK_OK;
    if ((q_heads && (!q || !q_out)) || (k_heads && (!k || !k_out)))
        return fail(FLOCK_EINVAL, "q, k, q_out and k_out must be non-NULL where they have heads");
    if ((n_y || n_x) && !xy) return fail(FLOCK_EINVAL, "xy is NULL with y or x pairs");
    if (n_time && !time) return fail(FLOCK_EINVAL, "time is NULL with time pairs");
    const size_t size = dtype_size(dtype);
    if (!aligned(q, size) || !aligned(k, size) || !aligned(q_out, size) || !aligned(k_out, size))
        return fail(FLOCK_EINVAL, "q, k, q_out and k_out must be aligned to their elements");
    if (!aligned(xy, 8) || !aligned(time, 4))
        return fail(FLOCK_EINVAL, "xy must be 8-byte aligned, time 4-byte aligned");
    const DeviceInfo *dev = nullptr;
    const flock_status st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    flock::RotaryArgs a{};
    a.q = q_heads ? q : nullptr;
    a.k = k_heads ? k : nullptr;
    a.q_out = q_heads ? q_out : nullptr;
    a.k_out = k_heads ? k_out : nullptr;
    a.q_stride = q_heads ? q_stride : 0;
    a.k_stride = k_heads ? k_stride : 0;
    a.q_out_stride = q_heads ? q_out_stride : 0;
    a.k_out_stride = k_heads ? k_out_stride : 0;
    a.xy = xy;
    a.time = time;
    a.total = total;
    a.q_heads = q_heads;
    a.k_heads = k_heads;
    a.head_dim = head_dim;
    a.n_time = n_time;
    a.n_y = n_y;
    a.pairs = pairs;
    a.interleaved = interleaved != 0;
    a.inverse = inverse != 0;
    rotary_steps(freq, n_time, pairs, a.step);
    const hipError_t err = flock::launch_rotary(a, dtype, reinterpret_cast<hipStream_t>(stream));
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "rotary kernel launch");
}

size_t attention_frames_workspace(int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads,
                                  int32_t kv_heads, int32_t head_dim) {
    if (n_frames <= 0 || total_q <= 0 || total_k <= 0 || q_heads < 1 || kv_heads < 1 || head_dim < 1) return 0;
    const flock::AttentionPlan plan = flock::plan_attention(n_frames, total_q, total_k, q_heads, kv_heads, device_cus());
    return flock::attention_workspace_bytes(plan, total_q, q_heads, head_dim);
}

flock_status attention_frames(int32_t dtype, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                              const void *v, int64_t v_stride, const int32_t *q_offsets, const int32_t *k_offsets,
                              int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads, int32_t kv_heads,
                              int32_t head_dim, const int32_t *q_xy, const int32_t *k_xy, const float *slopes,
                              const uint8_t *keep, int32_t causal, const int32_t *prefix, float scale, float cap,
                              void *out, int64_t out_stride, double *lse, void *workspace, size_t workspace_bytes,
                              void *stream) {
    g_error[0] = '\0';
    flock::AttentionArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.out = out;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.out_stride = out_stride;
    a.q_offsets = q_offsets;
    a.k_offsets = k_offsets;
    a.n_frames = n_frames;
    a.total_q = total_q;
    a.total_k = total_k;
    a.q_heads = q_heads;
    a.kv_heads = kv_heads;
    a.dim = head_dim;
    a.q_xy = q_xy;
    a.k_xy = k_xy;
    a.slopes = slopes;
    a.keep = keep;
    a.prefix = prefix;
    a.causal = causal;
    a.scale = scale;
    a.cap = cap;
    a.lse = lse;
    flock_status st = check_attention(dtype, a);
    if (st != FLOCK_OK) return st;
    a.group = q_heads / kv_heads;
    if (n_frames == 0 || total_q == 0) return FLOCK_OK;
    st = check_attention_pointers(a);
    if (st != FLOCK_OK) return st;
    const flock::AttentionPlan plan = flock::plan_attention(n_frames, total_q, total_k, q_heads, kv_heads, device_cus());
    st = check_workgroups(flock::attention_workgroups(plan, total_q, q_heads, kv_heads));
    if (st != FLOCK_OK) return st;
    const DeviceInfo *dev = nullptr;
    st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (validate_requested()) {
        st = validate_attention(a, s);
        if (st != FLOCK_OK) return st;
    }
    Workspace ws;
    st = ws.take(workspace, workspace_bytes, flock::attention_workspace_bytes(plan, total_q, q_heads, head_dim), s);
    if (st != FLOCK_OK) return st;
    hipError_t err = flock::launch_attention(a, dtype, plan, ws.ptr, s);
    const hipError_t ferr = ws.release(s);
    if (err == hipSuccess) err = ferr;
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "attention kernels");
}

size_t attention_frames_backward_workspace(int32_t n_frames, int32_t total_q, int32_t total_k, int32_t q_heads,
                                           int32_t kv_heads, int32_t head_dim) {
    if (n_frames <= 0 || total_q < 0 || total_k < 0 || q_heads < 1 || kv_heads < 1 || head_dim < 1) return 0;
    return flock::attention_backward_workspace_bytes(n_frames, total_q, q_heads, kv_heads);
}

flock_status attention_frames_backward(
    int32_t dtype, const void *grad_out, int64_t grad_out_stride, const void *q, int64_t q_stride, const void *k,
    int64_t k_stride, const void *v, int64_t v_stride, const void *out, int64_t out_stride, const double *lse,
    const int32_t *q_offsets, const int32_t *k_offsets, int32_t n_frames, int32_t total_q, int32_t total_k,
    int32_t q_heads, int32_t kv_heads, int32_t head_dim, const int32_t *q_xy, const int32_t *k_xy,
    const float *slopes, const uint8_t *keep, int32_t causal, const int32_t *prefix, float scale, float cap,
    void *grad_q, int64_t grad_q_stride, void *grad_k, int64_t grad_k_stride, void *grad_v, int64_t grad_v_stride,
    float *grad_slopes, void *workspace, size_t workspace_bytes, void *stream) {
    g_error[0] = '\0';
    flock::AttentionBackwardArgs b{};
    flock::AttentionArgs &a = b.fwd;
    a.q = q;
    a.k = k;
    a.v = v;
    a.out = const_cast<void *>(out);  // read only
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.out_stride = out_stride;
    a.q_offsets = q_offsets;
    a.k_offsets = k_offsets;
    a.n_frames = n_frames;
    a.total_q = total_q;
    a.total_k = total_k;
    a.q_heads = q_heads;
    a.kv_heads = kv_heads;
    a.dim = head_dim;
    a.q_xy = q_xy;
    a.k_xy = k_xy;
    a.slopes = slopes;
    a.keep = keep;
    a.prefix = prefix;
    a.causal = causal;
    a.scale = scale;
    a.cap = cap;
    a.lse = const_cast<double *>(lse);  // read only
    b.grad_out = grad_out;
    b.grad_out_stride = grad_out_stride;
    b.grad_q = grad_q;
    b.grad_q_stride = grad_q_stride;
    b.grad_k = grad_k;
    b.grad_k_stride = grad_k_stride;
    b.grad_v = grad_v;
    b.grad_v_stride = grad_v_stride;
    flock_status st = check_attention(dtype, a);
    if (st != FLOCK_OK) return st;
    a.group = q_heads / kv_heads;
    const int64_t q_row = (int64_t)q_heads * head_dim, kv_row = (int64_t)kv_heads * head_dim;
    if (grad_out_stride < 0 || grad_out_stride % 8 || grad_out_stride > flock::kAttentionMaxStride)
        return fail(FLOCK_EINVAL, "grad_out's stride must be a multiple of 8 in 0..%lld",
                    (long long)flock::kAttentionMaxStride);
    if (grad_q_stride < q_row || grad_k_stride < kv_row || grad_v_stride < kv_row || grad_q_stride % 8 ||
        grad_k_stride % 8 || grad_v_stride % 8)
        return fail(FLOCK_EINVAL, "strides of grad_q, grad_k and grad_v must be multiples of 8 that hold a row");
    if (grad_slopes && !slopes) return fail(FLOCK_EINVAL, "grad_slopes without slopes");
    if (n_frames == 0 && !grad_slopes) return FLOCK_OK;  // (else they are zeros)
    st = check_attention_pointers(a);
    if (st != FLOCK_OK) return st;
    if (total_q > 0 && (!grad_out || !lse || !grad_q))
        return fail(FLOCK_EINVAL, "grad_out, lse and grad_q must be non-NULL when total_q > 0");
    if (total_k > 0 && (!grad_k || !grad_v))
        return fail(FLOCK_EINVAL, "grad_k and grad_v must be non-NULL when total_k > 0");
    if (!aligned(grad_out, 16) || !aligned(grad_q, 16) || !aligned(grad_k, 16) || !aligned(grad_v, 16))
        return fail(FLOCK_EINVAL, "grad_out, grad_q, grad_k and grad_v must be 16-byte aligned");
    if (!aligned(grad_slopes, 4)) return fail(FLOCK_EINVAL, "grad_slopes must be 4-byte aligned");
    st = check_workgroups(flock::attention_backward_workgroups(n_frames, total_q, total_k, q_heads, kv_heads));
    if (st != FLOCK_OK) return st;
    const DeviceInfo *dev = nullptr;
    st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (validate_requested()) {
        st = validate_attention(a, s);
        if (st != FLOCK_OK) return st;
    }
    Workspace ws;
    st = ws.take(workspace, workspace_bytes, flock::attention_backward_workspace_bytes(n_frames, total_q, q_heads, kv_heads), s);
    if (st != FLOCK_OK) return st;
    hipError_t err = flock::launch_attention_backward(b, dtype, ws.ptr, grad_slopes, s);
    const hipError_t ferr = ws.release(s);
    if (err == hipSuccess) err = ferr;
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "attention backward kernels");
}

flock_status append_tracks(int32_t dtype, const void *new_k, int64_t new_k_stride, const void *new_v, int64_t new_v_stride,
                           const int32_t *offsets, int32_t n_tracks, int32_t total, const int32_t *table,
                           int64_t table_stride, int32_t max_pages, const int32_t *lengths, const int32_t *xy,
                           const int32_t *time, const double *freq, int32_t n_time, int32_t n_y, int32_t n_x,
                           int32_t interleaved, int8_t *k, int8_t *v, float *k_scale, float *v_scale, int32_t pages,
                           int32_t kv_heads, int32_t head_dim, void *stream) {
    g_error[0] = '\0';
    flock::AppendArgs a{};
    a.tracks = {offsets, lengths, table, table_stride, n_tracks, total, max_pages};
    a.cache = {k, v, k_scale, v_scale, pages, kv_heads, head_dim};
    if (!is_dtype(dtype)) return fail(FLOCK_EINVAL, "dtype = %d, expected FLOCK_F32, FLOCK_F16 or FLOCK_BF16", dtype);
    flock_status st = check_tracks(a.tracks, a.cache);
    if (st != FLOCK_OK) return st;
    if (new_k_stride < 0 || new_v_stride < 0) return fail(FLOCK_EINVAL, "strides of new_k and new_v must be >= 0");
    if (n_time < 0 || n_y < 0 || n_x < 0 || 2 * ((int64_t)n_time + n_y + n_x) > head_dim)
        return fail(FLOCK_EINVAL, "n_time = %d, n_y = %d, n_x = %d pairs do not fit head_dim = %d", n_time, n_y, n_x,
                    head_dim);
    const int32_t pairs = n_time + n_y + n_x;
    if (pairs && !freq) return fail(FLOCK_EINVAL, "freq is NULL with pairs");
    for (int32_t p = 0; p < pairs; ++p)
        if (!std::isfinite(freq[p])) return fail(FLOCK_EINVAL, "freq[%d] is not finite", p);
    if (n_tracks == 0 || total == 0) return FLOCK_OK;
    st = check_tracks_pointers(a.tracks, a.cache);
    if (st != FLOCK_OK) return st;
    if (!new_k || !new_v) return fail(FLOCK_EINVAL, "new_k and new_v must be non-NULL when total > 0");
    const size_t size = dtype_size(dtype);
    if (!aligned(new_k, size) || !aligned(new_v, size))
        return fail(FLOCK_EINVAL, "new_k and new_v must be aligned to their elements");
    if ((n_y || n_x) && !xy) return fail(FLOCK_EINVAL, "xy is NULL with y or x pairs");
    if (n_time && !time) return fail(FLOCK_EINVAL, "time is NULL with time pairs");
    if (!aligned(xy, 8) || !aligned(time, 4))
        return fail(FLOCK_EINVAL, "xy must be 8-byte aligned, time 4-byte aligned");
    st = check_workgroups(flock::append_workgroups(n_tracks, total, kv_heads));
    if (st != FLOCK_OK) return st;
    if (pages == 0 || max_pages == 0) return FLOCK_OK;  // no page to go to
    const DeviceInfo *dev = nullptr;
    st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (validate_requested()) {
        st = validate_offsets("offsets", offsets, n_tracks, total, s);
        if (st != FLOCK_OK) return st;
    }
    a.k = new_k;
    a.v = new_v;
    a.k_stride = new_k_stride;
    a.v_stride = new_v_stride;
    a.xy = xy;
    a.time = time;
    a.n_time = n_time;
    a.n_y = n_y;
    a.pairs = pairs;
    a.interleaved = interleaved != 0;
    rotary_steps(freq, n_time, pairs, a.step);
    const hipError_t err = flock::launch_append(a, dtype, s);
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "append kernel launch");
}

size_t attention_tracks_workspace(int32_t n_tracks, int32_t total, int32_t max_pages, int32_t q_heads, int32_t kv_heads,
                                  int32_t head_dim) {
    if (n_tracks <= 0 || total <= 0 || max_pages < 0 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || head_dim < 1)
        return 0;
    return flock::track_attention_workspace_bytes(
            flock::plan_track_attention(n_tracks, total, max_pages, q_heads, kv_heads, device_cus()), total, q_heads, head_dim);
}

flock_status attention_tracks(int32_t dtype, const void *q, int64_t q_stride, const int32_t *offsets, int32_t n_tracks,
                              int32_t total, const int32_t *table, int64_t table_stride, int32_t max_pages,
                              const int32_t *lengths, const int8_t *k, const int8_t *v, const float *k_scale,
                              const float *v_scale, int32_t pages, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                              int32_t window, float scale, float cap, void *out, int64_t out_stride, void *workspace,
                              size_t workspace_bytes, void *stream) {
    g_error[0] = '\0';
    flock::TrackAttentionArgs a{};
    a.tracks = {offsets, lengths, table, table_stride, n_tracks, total, max_pages};
    // (the cache is only read)
    a.cache = {const_cast<int8_t *>(k), const_cast<int8_t *>(v), const_cast<float *>(k_scale),
               const_cast<float *>(v_scale), pages, kv_heads, head_dim};
    if (dtype != FLOCK_F16 && dtype != FLOCK_BF16)
        return fail(FLOCK_EINVAL, "dtype = %d, expected FLOCK_F16 or FLOCK_BF16", dtype);
    flock_status st = check_tracks(a.tracks, a.cache);
    if (st != FLOCK_OK) return st;
    if (q_heads < 1 || q_heads > 256 || q_heads % kv_heads)
        return fail(FLOCK_EINVAL, "q_heads = %d is not a multiple of kv_heads = %d in 1..256", q_heads, kv_heads);
    if (window < 0) return fail(FLOCK_EINVAL, "window = %d < 0", window);
    if (!std::isfinite(scale) || !(scale > 0.0f)) return fail(FLOCK_EINVAL, "scale must be finite and > 0");
    if (!std::isfinite(cap) || !(cap >= 0.0f)) return fail(FLOCK_EINVAL, "cap must be finite and >= 0");
    if (q_stride < 0 || out_stride < (int64_t)q_heads * head_dim)
        return fail(FLOCK_EINVAL, "q's stride must be >= 0, and out's hold a row");
    if (n_tracks == 0 || total == 0) return FLOCK_OK;
    st = check_tracks_pointers(a.tracks, a.cache);
    if (st != FLOCK_OK) return st;
    if (!q || !out) return fail(FLOCK_EINVAL, "q and out must be non-NULL when total > 0");
    if (!aligned(q, 2) || !aligned(out, 2)) return fail(FLOCK_EINVAL, "q and out must be aligned to their elements");
    // rows are numbered in 31 bits, up to the end of the tile after the last
    if ((int64_t)total * (q_heads / kv_heads) > 0x7fffff00LL)
        return fail(FLOCK_EUNSUPPORTED, "batch of more than 2^31 - 256 rows of queries and shared heads");
    const DeviceInfo *dev = nullptr;
    const flock::TrackPlan plan = flock::plan_track_attention(n_tracks, total, max_pages, q_heads, kv_heads, device_cus());
    st = check_workgroups(plan.slots * kv_heads * plan.splits);
    if (st != FLOCK_OK) return st;
    st = device_info(&dev);
    if (st != FLOCK_OK) return st;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (validate_requested()) {
        st = validate_offsets("offsets", offsets, n_tracks, total, s);
        if (st != FLOCK_OK) return st;
    }
    a.q = q;
    a.q_stride = q_stride;
    a.out = out;
    a.out_stride = out_stride;
    a.q_heads = q_heads;
    a.window = std::min(window, 1 << 30);  // (as long as any track)
    a.scale = scale;
    a.cap = cap;
    Workspace ws;
    st = ws.take(workspace, workspace_bytes, flock::track_attention_workspace_bytes(plan, total, q_heads, head_dim), s);
    if (st != FLOCK_OK) return st;
    hipError_t err = flock::launch_track_attention(a, dtype, plan, ws.ptr, s);
    const hipError_t ferr = ws.release(s);
    if (err == hipSuccess) err = ferr;
    return err == hipSuccess ? FLOCK_OK : hip_fail(err, "track attention kernels");
}

}  // extern "C"
