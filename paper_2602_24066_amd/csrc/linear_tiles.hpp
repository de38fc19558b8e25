// Tiles of a matrix product and splits of its contraction: what a launch is made of.  Plain arithmetic, compiled for the host alone too, where it is checked
// over the whole range of sizes.
#pragma once
#include <algorithm>
#include <cstdint>
#include <limits>

#include "launch.hpp"

namespace sig {

constexpr int kSlab = 128, kChunk = 16, kChunks = kSlab / kChunk;      // bytes; bytes; chunks of a slab
constexpr int kTile = 128;                                             // of rows of any alignment

// Tiles along m and n; slabs of a split; edge of a tile (few: in 16 tokens; 0: no launch numbers the threads of any); threads of a workgroup; what the launch's model says
struct Tiles {
    int64_t M, N, K;
    int m, n, splits;
    int64_t slabs;
    int tile, threads;
    bool few;
    double us;
    int64_t blocks() const { return (int64_t)m * n * splits; }
    int64_t joins() const { return splits > 1 ? (M * ((N + 3) / 4) + 255) / 256 : 0; }     // workgroups of 256 that add up the splits
    bool launchable() const { return tile && sig::launchable(blocks(), threads) && sig::launchable(joins(), 256); }
};

// ---- which tile, and how many splits.  A model of the launch, in us: `slab` is what a tile's slab costs a compute unit that is busy with as many
// as it holds, `alone` what it costs at least, `over` what a tile costs besides (first loads, outputs).  Measured on large squares (us a slab):
//   bfloat16 256: 8192^3 in 856 us, 128: 1,022 us     float32 128: 4096^3 in 998, 64: 1,040     e4m3 256: 8192^3 in 476, 128: 550
// and 16384 x 4096 x 1024 (16 slabs): 148 us with tiles of 256, 172 of 128; e4m3 16384 x 2048 x 2048: 72 and 79.
// Rows that are not whole chunks (product_kernel) take `rough` times the slab: bfloat16 16384 x 5460 to 1024 272 us, of 5456 189; float32 5000 x 1001 to 1001 139.
struct Cost { int tile; double slab, alone, over; };
constexpr double kRough[3] = {1.07, 1.5, 1.5};                                         // float32, bfloat16, e4m3
constexpr Cost kCosts[3][3] = {
    {{64, 0.51, 0.70, 1.0}, {128, 1.95, 1.95, 3.0}, {}},                               // float32: tiles of 256 gain 2 % at most
    {{64, 0.17, 0.50, 0.8}, {128, 0.50, 0.80, 2.4}, {256, 1.68, 1.68, 10.5}},          // bfloat16
    {{64, 0.18, 0.50, 0.8}, {128, 0.54, 0.80, 1.2}, {256, 1.86, 1.86, 6.3}},           // e4m3
};
constexpr int kUnits = 256;                                                            // compute units

// Up to 64 tokens: what few_kernel takes, in us, by the rate at which a compute unit's wavefronts get its operands (40 GB/s; 64 tokens bfloat16, the
// weight from the cache: 2048 to 1024 5.9 us with tiles of 16 x 16, 1024 to 4096 6.4 with 32 x 32; from memory 7.0 and 7.6, 8192 to 8192 36 with 64 x 32).
constexpr int kFew = 64, kFewThreads = 512;
struct FewPlan { int fm, fn; int64_t m, n; double us; };                                // fm 0: none
inline FewPlan few_plan(int64_t M, int64_t N, int64_t bytes)
{
    FewPlan best{};
    for (FewPlan p : {FewPlan{1, 1, 0, 0, 0.0}, FewPlan{2, 2, 0, 0, 0.0}, FewPlan{4, 2, 0, 0, 0.0}}) {
        p.m = (M + p.fm * 16 - 1) / (p.fm * 16);
        p.n = (N + p.fn * 16 - 1) / (p.fn * 16);
        if (!launchable(p.m * p.n, kFewThreads)) continue;
        p.us = 3.0 + (double)((p.m * p.n + kUnits - 1) / kUnits) * (p.fm + p.fn) * 16 * bytes / 40e3;
        if (best.fm == 0 || p.us < best.us) best = p;
    }
    return best;
}

inline Tiles tiles_of(int64_t M, int64_t N, int64_t K, int e, bool aligned, bool few = true)
{
    const int64_t slabs = std::max<int64_t>(1, (K * e + kSlab - 1) / kSlab);
    Tiles best{};
    best.us = std::numeric_limits<double>::infinity();
    for (const Cost& c : kCosts[e == 4 ? 0 : e == 2 ? 1 : 2]) {
        if (c.tile == 0 || (!aligned && c.tile != kTile)) continue;
        const int64_t m = (M + c.tile - 1) / c.tile, n = (N + c.tile - 1) / c.tile;
        for (int64_t want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            if (want > 1 && slabs / want < 4) break;
            const int64_t each = (slabs + want - 1) / want, splits = (slabs + each - 1) / each, rows = (m * n * splits + kUnits - 1) / kUnits;
            double us = (double)each * std::max(rows * c.slab, c.alone) * (aligned ? 1.0 : kRough[e == 4 ? 0 : e == 2 ? 1 : 2]) + rows * c.over;
            if (splits > 1) us += 4.0 + (double)M * N * 4.0 * (splits + 1) / 3e6;     // the sums, written and read again
            const Tiles t{M, N, K, (int)m, (int)n, (int)splits, each, c.tile, c.tile == 256 ? 512 : 256, false, us};
            if (us < best.us && t.launchable()) best = t;
        }
    }
    if (aligned && few && M <= kFew)
        if (const FewPlan p = few_plan(M, N, K * e); p.fm && p.us < 3.0 + best.us) return Tiles{M, N, K, (int)p.m, (int)p.n, 1, 0, p.fm, kFewThreads, true, p.us};
    return best;
}

}  // namespace sig
