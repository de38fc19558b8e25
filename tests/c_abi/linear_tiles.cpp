// The tiles of products of every size that memory holds (288 GB of operands and outputs): there are some, a launch numbers their threads, they cover the
// outputs, and the splits the contraction.  Prints what is wrong, and ends with 1 then.
#include <cstdio>
#include <initializer_list>

#include "linear_tiles.hpp"

int main()
{
    long bad = 0, seen = 0;
    const int64_t most = (1ll << 31) - 257, memory = 288ll << 30, small[] = {1, 2, 3, 4, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 300, 500, 513, 1000};
    auto check = [&](int64_t M, int64_t N, int64_t K, int e, bool aligned, bool few) {
        const int out = e == 4 ? 4 : 2;
        if (M * N > 1ll << 38 || M * K > 1ll << 38 || N * K > 1ll << 38 || M * N * out + (M + N) * K * e > memory) return;
        seen++;
        const sig::Tiles t = sig::tiles_of(M, N, K, e, aligned, few);
        const int64_t blocks = (int64_t)t.m * t.n * t.splits, threads = t.few || t.tile == 256 ? 512 : 256;
        const int64_t edge_m = t.few ? t.tile * 16 : t.tile, edge_n = t.few ? (t.tile == 1 ? 16 : 32) : t.tile, slabs = (K * e + sig::kSlab - 1) / sig::kSlab;
        const char* what = t.tile == 0 ? "no tile" : !sig::launchable(blocks, threads) ? "more threads than a launch numbers" :
                           t.splits > 1 && !sig::launchable((M * ((N + 3) / 4) + 255) / 256, 256) ? "more threads than the joining launch numbers" :
                           t.m * edge_m < M || t.n * edge_n < N || (t.m - 1) * edge_m >= M || (t.n - 1) * edge_n >= N ? "outputs not covered" :
                           !t.few && (t.splits * t.slabs < slabs || (t.splits - 1) * t.slabs >= slabs) ? "contraction not covered" : nullptr;
        if (what && bad++ < 8)
            std::printf("%s: %lld x %lld x %lld, %d bytes, aligned %d: tile %d, %d x %d x %d\n", what, (long long)M, (long long)N, (long long)K, e, aligned, t.tile, t.m, t.n, t.splits);
    };
    auto both = [&](int64_t M, int64_t N, int64_t K) {
        for (int e : {1, 2, 4})
            for (bool aligned : {false, true}) {
                check(M, N, K, e, aligned, true);
                if (aligned) check(M, N, K, e, aligned, false);
            }
    };
    for (int64_t N : small)
        for (int64_t K : small) {
            for (int64_t M : small) both(M, N, K);
            for (double f = 1000; f < 4e9; f *= 1.23) {
                const int64_t big = f < most ? (int64_t)f : most;
                both(big, N, K);
                both(N, big, K);
                both(N, K, big);
            }
        }
    for (double f = 300; f < 4e9; f *= 2.17)
        for (double g = 300; g < 4e9; g *= 2.17)
            for (int64_t s : {1, 8, 100, 1001, 5460}) {
                const int64_t a = f < most ? (int64_t)f : most, b = g < most ? (int64_t)g : most;
                both(a, b, s);
                both(a, s, b);
            }
    std::printf("%ld wrong of %ld\n", bad, seen);
    return bad != 0;
}
