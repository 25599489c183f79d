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

__device__ __forceinline__ constexpr int token_at(int place) { return 16 * (place % 16 / 4) + 4 * (place / 16) + place % 4; }

// One track's part of the batch: `n` rows, which are the last of its `length` tokens.
struct Track {
    int32_t row0, n, length;
    bool ok;
};

__device__ __forceinline__ Track track_of(const TrackArgs &a, int t) {
    Track s;
    s.row0 = a.offsets[t];
    const int32_t end = a.offsets[t + 1];
    s.length = a.lengths[t];
    s.ok = s.row0 >= 0 && end >= s.row0 && end <= a.total && s.length >= 0 && s.length <= (int64_t)a.max_pages * kPage;
    s.n = end - s.row0;
    return s;
}

// Track of a work item, and the item's number within the track: items of track t
// begin at begin(t), which grows with t.  All lanes of a wave look together, a 64th
// of what is left each time.
template <typename F>
__device__ __forceinline__ int find_track(int n_tracks, int64_t item, F &&begin, int64_t *within) {
    int lo = 0, left = n_tracks;
    while (left > 1) {
        const int step = (left + 63) >> 6, t = lo + step * (int)(threadIdx.x & 63);
        const bool before = t < lo + left && begin(t) <= item;
        const int at = max(__builtin_popcountll(__ballot(before)), 1) - 1;
        left = min(step, left - at * step);
        lo += at * step;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    *within = item - begin(lo);
    return lo;
}

}  // namespace tracks
}  // namespace flock

#endif  // FLOCK_TRACKS_COMMON_H
