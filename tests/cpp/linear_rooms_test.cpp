// Host test of where waves of the 8-bit products put their outputs in LDS: in a
// stage that is not the one that other waves may still multiply from, each wave's
// bytes apart from every other's, and all of them within the parts of that stage.
#include <cstdio>

#include "linear_common.h"

using namespace flock::linear;

static int failures = 0;

struct Bytes {
    const int8_t *from, *to;
    bool meets(const Bytes &o) const { return from < o.to && o.from < to; }
    bool within(const Bytes &o) const { return from >= o.from && to <= o.to; }
};

// Whether rooms of `size` bytes at at(stage, wave) meet neither each other nor what is read meanwhile.
template <int BM, int BN, typename F>
static bool apart(LinearShared<BM, BN> &s, int stage, int size, F &&at) {
    bool good = true;
    const Bytes x{s.x[stage], s.x[stage] + BM * kStep}, w{s.w[stage], s.w[stage] + BN * kStep};
    for (int wave = 0; wave < 4; ++wave) {
        const int8_t *p = at(stage, wave);
        const Bytes mine{p, p + size};
        good = good && (mine.within(x) || mine.within(w)) && (p - s.x[0]) % 16 == 0;
        for (int other = 0; other < kStages; ++other) {
            if (other == stage) continue;
            good = good && !mine.meets({s.x[other], s.x[other] + BM * kStep});
            good = good && !mine.meets({s.w[other], s.w[other] + BN * kStep});
        }
        for (int v = 0; v < wave; ++v) {
            const int8_t *q = at(stage, v);
            good = good && !mine.meets({q, q + size});
        }
    }
    return good;
}

template <int KN, int BM, int BN>
static void check() {
    static LinearShared<BM, BN> s;
    for (int stage = 0; stage < kStages; ++stage)
        if (!apart(s, stage, kRoom<KN>, [&](int t, int wave) { return stage_room<KN>(s, t, wave); })) {
            std::printf("tiles of %d x %d, stage %d: a room is in use\n", BM, BN, stage);
            ++failures;
        }
}

int main() {
    check<1, 64, 64>();
    check<2, 128, 128>();
    // rooms of half a stage's part one after the other run on into the weights of the first stage
    static LinearShared<64, 64> s;
    if (apart(s, 1, kRoom<1>, [&](int, int wave) { return s.x[1] + wave * (64 * kStep / 2); })) {
        std::printf("the check finds no fault in rooms that run on\n");
        ++failures;
    }
    if (failures) return 1;
    std::printf("rooms ok\n");
    return 0;
}
