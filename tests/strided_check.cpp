// Host-side check of the strided-row overlap rules (strided.h) against byte maps
// of random small layouts. Built and run by tests/test_strided.py on the CPU.
#include <cstdio>
#include <random>
#include <vector>

#include "strided.h"

using namespace sifar;

int main() {
    std::mt19937_64 rng(260708973);
    auto draw = [&](uint64_t lo, uint64_t hi) { return lo + rng() % (hi - lo + 1); };
    uint64_t met = 0, apart = 0, exact = 0;
    for (int n = 0; n < 300000; ++n) {
        Rows r[2];
        const uint64_t tokens = draw(1, 4), stride = draw(1, 24);
        for (Rows &x : r) {
            x.rows = tokens;
            x.stride = rng() % 3 ? stride : draw(1, 24);
            x.size = draw(1, 12);
            if (rng() % 2 && x.size > x.stride) x.size = x.stride;
            x.at = draw(1, 60);
        }
        std::vector<char> map(300, 0);
        for (uint64_t t = 0; t < r[0].rows; ++t)
            for (uint64_t i = 0; i < r[0].size; ++i) map[r[0].at + t * r[0].stride + i] = 1;
        bool meet = false;
        for (uint64_t t = 0; t < r[1].rows; ++t)
            for (uint64_t i = 0; i < r[1].size; ++i) meet |= map[r[1].at + t * r[1].stride + i];
        const bool may = may_overlap(r[0], r[1]);
        if (may != may_overlap(r[1], r[0])) return std::printf("asymmetric\n"), 1;
        if (meet && !may) return std::printf("overlap missed\n"), 1;
        met += meet;
        apart += !may;
        // at one stride, with rows that do not overlap themselves, inside the other's span:
        // interleaved views are told apart
        if (r[0].stride == r[1].stride && r[0].size <= r[0].stride && r[1].size <= r[1].stride &&
            tokens > 1 && r[1].at >= r[0].at && rows_end(r[1]) <= rows_end(r[0]) + stride - r[0].size) {
            if (may && !meet) return std::printf("interleaved rows refused\n"), 1;
            exact += !meet;
        }
        const bool same = same_rows(r[0], r[1]);
        if (same != (r[0].at == r[1].at && r[0].size == r[1].size &&
                     (tokens == 1 || r[0].stride == r[1].stride)))
            return std::printf("same rows\n"), 1;
    }
    const Rows none{}, some{64, 2, 8, 8};
    if (may_overlap(none, some) || may_overlap(some, none)) return std::printf("empty\n"), 1;
    if (met < 10000 || apart < 10000 || exact < 1000) return std::printf("thin\n"), 1;
    std::printf("ok %llu %llu %llu\n", (unsigned long long)met, (unsigned long long)apart,
                (unsigned long long)exact);
    return 0;
}
