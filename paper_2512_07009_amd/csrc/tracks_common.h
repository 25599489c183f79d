// tracks_common.h - the paged cache of tracks in 8 bits: its layout, and how work
// on ragged tracks is numbered.
//
// A page holds kPage tokens of a track.  For each page and kv head there are
//   k  int8 [token][dim]
//   v  int8 [dim][place]: token t at place 16 * (t % 16 / 4) + 4 * (t / 16) + t % 4,
//      so that 16 bytes are the tokens that a lane multiplies with its weights
//   a scale each, float: what the whole numbers are times it.
#ifndef FLOCK_TRACKS_COMMON_H
#define FLOCK_TRACKS_COMMON_H

#include "encoder_common.h"

namespace flock {
namespace tracks {

constexpr int kPage = kTrackPage;

typedef int i32x4 __attribute__((ext_vector_type(4)));

// One track's part of the batch: `n` rows, which are the last of its `length` tokens.
struct Track {
    int32_t index, row0, n, length;
    bool ok;
};

__device__ __forceinline__ Track make_track(const TrackArgs &a, int index, int32_t row0, int32_t end, int32_t length) {
    Track s;
    s.index = index;
    s.row0 = row0;
    s.n = end - row0;
    s.length = length;
    s.ok = row0 >= 0 && end >= row0 && end <= a.total && length >= 0 && length <= (int64_t)a.max_pages * kPage;
    return s;
}

__device__ __forceinline__ Track track_of(const TrackArgs &a, int t) {
    return make_track(a, t, a.offsets[t], a.offsets[t + 1], a.lengths[t]);
}

// The track of work item `item` of `items`, and the item's number within it: items of
// track t begin at begin(offsets[t], t), which grows with t.
//
// Most workgroups live for a few trips to memory, so this is one: the lanes of a wave
// read 64 tracks around the place where the item is in an even batch, and the track's
// offsets and length come from them.  Where the track is not among those, a 64th of what
// is left is looked up each time.
template <typename F>
__device__ __forceinline__ Track find_track(const TrackArgs &a, int64_t item, int64_t items, F &&begin, int64_t *within) {
    const int lane = threadIdx.x & 63, n = a.n_tracks;
    const int middle = (int)((float)item / (float)items * (float)n);
    int lo = max(min(middle - 31, n - 63), 0);
    for (bool sought = false;; sought = true) {
        const int t = min(lo + lane, n);
        const int32_t offset = a.offsets[t], length = a.lengths[min(t, n - 1)];
        const uint64_t before = __ballot(lo + lane < n && begin(offset, t) <= item);
        int at = 63 - __builtin_clzll(before | 1);
        if (!sought && ((before & 1) == 0 ? lo > 0 : at == 63)) {
            lo = 0;
            for (int left = n; left > 1;) {
                const int step = (left + 63) >> 6, u = lo + step * lane;
                const bool early = u < lo + left && begin(a.offsets[min(u, n)], u) <= item;
                const int past = max(__builtin_popcountll(__ballot(early)), 1) - 1;
                left = min(step, left - past * step);
                lo += past * step;
            }
            continue;
        }
        if (sought) at = 0;
        at = __builtin_amdgcn_readfirstlane(at);
        const Track s = make_track(a, lo + at, __builtin_amdgcn_readlane(offset, at),
                                   __builtin_amdgcn_readlane(offset, at + 1), __builtin_amdgcn_readlane(length, at));
        *within = item - begin(s.row0, s.index);
        return s;
    }
}

}  // namespace tracks
}  // namespace flock

#endif  // FLOCK_TRACKS_COMMON_H
