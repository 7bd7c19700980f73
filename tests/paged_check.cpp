// Host-side check of the paged cache's strides (csrc/paged.h) against every element:
// extent() takes exactly the layouts whose elements are apart, and shares() finds exactly
// the offsets at which two caches of one layout meet. Built and run by
// tests/test_paged.py on the CPU.
#include <cstdint>
#include <cstdio>
#include <set>
#include <vector>

#include "paged.h"

using namespace sifar;

static std::vector<int64_t> elements(const int64_t (&n)[3], const int64_t (&s)[3], int64_t dim) {
    std::vector<int64_t> all;
    for (int64_t p = 0; p < n[0]; ++p)
        for (int64_t q = 0; q < n[1]; ++q)
            for (int64_t h = 0; h < n[2]; ++h)
                for (int64_t d = 0; d < dim; ++d) all.push_back(p * s[0] + q * s[1] + h * s[2] + d);
    return all;
}

int main() {
    const int64_t strides[] = {0, 4, 8, 16, 24, 32, 40, 48, 64, 96, 128, 200};
    const int64_t counts[][3] = {{1, 1, 1}, {2, 1, 3}, {3, 2, 2}, {1, 4, 2}, {2, 2, 1}, {3, 3, 2}};
    long layouts = 0, checked = 0;
    for (const auto &n : counts)
        for (int64_t a : strides)
            for (int64_t b : strides)
                for (int64_t c : strides)
                    for (int64_t dim : {8, 16}) {
                        const int64_t s[3] = {a, b, c};
                        const Paged p = paged(n[0], n[1], n[2], a, b, c, dim);
                        const int64_t e = extent(p);
                        int64_t used[3] = {n[0] > 1 ? a : 0, n[1] > 1 ? b : 0, n[2] > 1 ? c : 0};
                        const std::vector<int64_t> all = elements(n, used, dim);
                        const std::set<int64_t> own(all.begin(), all.end());
                        bool eights = true;
                        for (int64_t u : used) eights = eights && u % 8 == 0;
                        if (e == 0) {
                            // refused: elements meet, strides are odd, or loops interleave
                            continue;
                        }
                        if (!eights || own.size() != all.size() || e != *own.rbegin() + 1) {
                            std::printf("extent %ld of %ld,%ld,%ld x %ld,%ld,%ld\n", long(e), long(n[0]),
                                        long(n[1]), long(n[2]), long(s[0]), long(s[1]), long(s[2]));
                            return 1;
                        }
                        ++layouts;
                        for (int64_t d = -e - 8; d <= e + 8; ++d) {
                            bool meet = false;
                            for (int64_t x : own)
                                if (own.count(x + d)) {
                                    meet = true;
                                    break;
                                }
                            ++checked;
                            if (meet != shares(p, d)) {
                                std::printf("shares %ld of %ld,%ld,%ld x %ld,%ld,%ld\n", long(d),
                                            long(n[0]), long(n[1]), long(n[2]), long(s[0]), long(s[1]),
                                            long(s[2]));
                                return 1;
                            }
                        }
                    }
    // the usual layouts are all taken
    if (extent(paged(5, 16, 4, 16 * 4 * 64, 4 * 64, 64, 64)) != 5 * 16 * 4 * 64 ||
        extent(paged(5, 16, 4, 16 * 4 * 64, 64, 16 * 64, 64)) != 5 * 16 * 4 * 64 ||
        !extent(paged(5, 16, 4, 2 * 16 * 4 * 64, 4 * 64, 64, 64)) ||
        !extent(paged(1, 16, 1, 8, 64, 8, 64)) || extent(paged(2, 1, 1, int64_t{1} << 41, 0, 0, 8)) ||
        extent(paged(2147483647, 65536, 1024, int64_t{1} << 40, 1 << 18, 256, 256)) ||
        extent(paged(2, 2, 2, -4096, 1024, 64, 64))) {
        std::printf("usual layouts\n");
        return 1;
    }
    std::printf("ok %ld layouts %ld offsets\n", layouts, checked);
    return 0;
}
