// Every lane's channels for every number of channels: argument 1 is the largest.  Prints what is wrong, and ends with 1 then.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "gated_lane.hpp"

int main(int, char** argv)
{
    const int most = std::atoi(argv[1]);
    long bad = 0;
    std::vector<int> stored;
    auto check = [&](bool good, const char* what, int D, bool pairs, int group, int lane, const sig::GatedLane& l) {
        if (!good && bad++ < 8) std::printf("%s: D %d pairs %d group %d lane %d: c %d c1 %d\n", what, D, pairs, group, lane, l.c, l.c1);
    };
    for (int D = 1; D <= most; D++)
        for (bool pairs : {false, true}) {
            if (pairs && D % 2) continue;
            stored.assign(D, 0);
            for (int group = 0; group < (D + sig::kGatedGroup - 1) / sig::kGatedGroup; group++)
                for (int lane = 0; lane < 32; lane++) {
                    const sig::GatedLane l = sig::gated_lane(group, lane, D, pairs);
                    check(l.c >= 0 && l.c < D && l.c1 >= 0 && l.c1 < D, "reads a channel that is not there", D, pairs, group, lane, l);
                    check(!pairs || (l.c % 2 == 0 && l.c1 == l.c + 1), "no pair", D, pairs, group, lane, l);
                    check(l.c1 == (l.even ? l.c + 1 : l.c), "not the next channel", D, pairs, group, lane, l);
                    if (!l.on) continue;
                    check(l.c == group * sig::kGatedGroup + lane * 2, "not its own channel", D, pairs, group, lane, l);
                    if (l.c < D) stored[l.c]++;
                    if (l.even && l.c1 < D) stored[l.c1]++;
                }
            for (int c = 0; c < D; c++)
                if (stored[c] != 1 && bad++ < 8) std::printf("D %d pairs %d: channel %d is stored %d times\n", D, pairs, c, stored[c]);
        }
    if (bad) std::printf("%ld in all\n", bad);
    return bad != 0;
}
