// Which channels a lane of the gated recurrence has; plain arithmetic, compiled for the host too, where it is checked over all channel counts.
#pragma once
#include <cstdint>

namespace sig {

constexpr int kGatedGroup = 64;         // channels of a workgroup, two neighbouring ones a lane

// c and c1: channels that the lane reads, both below D (the same one where it has a single channel).  Lanes behind the last channel read those of the last
// lane and store nothing (not `on`).  even: it stores both.  pairs: D is even, and both channels are one access, so c is even as well.
struct GatedLane {
    int c, c1;
    bool on, even;
};
constexpr GatedLane gated_lane(uint32_t group, uint32_t lane, int D, bool pairs)
{
    const int c = (int)(group * kGatedGroup + lane * 2);
    GatedLane l{c, c + 1, c < D, true};
    if (c >= D) l.c = D - (pairs ? 2 : 1);
    l.even = pairs || l.c + 1 < D;
    l.c1 = l.even ? l.c + 1 : l.c;
    return l;
}

}  // namespace sig
