// Host-side check of how sifar_paged_attention shares sequences (csrc/attend_plan.h): for
// random shapes, chunks that LDS has places for, no more of them than the grid has, and
// never more bytes of workspace than the call asks for. Built and run by
// tests/test_attend_plan.py on the CPU.
#include <cmath>
#include <cstdio>
#include <random>

#include "attend_plan.h"

using namespace sifar;

int main() {
    std::mt19937_64 rng(260708973);
    const auto spread = [&](int64_t most) {
        return static_cast<int64_t>(
            std::exp2(std::uniform_real_distribution<double>(0.0, std::log2(double(most)))(rng)));
    };
    const int64_t kvs[] = {1, 2, 3, 4, 8, 16, 32, 64, 128, 1024};
    const int64_t groups[] = {1, 2, 3, 5, 7, 8, 15, 16, 17, 33, 64, 1024};
    const int64_t dims[] = {8, 64, 80, 128, 136, 256};
    long shared = 0;
    for (int i = 0; i < 300000; ++i) {
        const int64_t tokens = spread(SIFAR_ATTENTION_MAX_TOKENS), kv = kvs[rng() % 10];
        const int64_t group = groups[rng() % 12], dim = dims[rng() % 6];
        if (kv * group > SIFAR_CACHE_MAX_HEADS) continue;
        const int64_t length = spread(SIFAR_ATTENTION_MAX_LENGTH);
        const int64_t reach = rng() % 2 ? length : 1 + length / int64_t(1 + rng() % 50);  // a window
        if (reach > length) continue;
        const int dtype = rng() % 2 ? SIFAR_BF16 : SIFAR_FP32;
        const int64_t splits = splits_of(dtype, tokens, kv * group, kv, dim, reach);
        const int64_t round = kWaves * tile_of(dtype, wide_of(dim));
        bool ok = splits >= 1 &&
                  used_bytes(tokens * kv * group, splits, dim) <=
                      asked_bytes(tokens, kv * group, kv, dim, length);
        for (int64_t count : {reach, reach - 1, reach / 2, reach / 3, int64_t{1}}) {
            if (count < 1) continue;
            int64_t chunk = ceil_div(ceil_div(count, splits), round) * round;  // as the kernel's
            chunk = chunk < kMinChunk ? kMinChunk : chunk;
            ok = ok && chunk <= kMaxChunk && ceil_div(count, chunk) <= splits;
        }
        if (!ok) {
            std::printf("FAIL tokens %ld heads %ld x %ld dim %ld length %ld reach %ld type %d: %ld\n",
                        long(tokens), long(kv), long(group), long(dim), long(length), long(reach),
                        dtype, long(splits));
            return 1;
        }
        shared += splits > 1;
    }
    std::printf("ok %ld shared\n", shared);
    return shared > 1000 ? 0 : 1;
}
