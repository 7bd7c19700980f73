// Host-side check of the chunks that sifar_paged_attention's kernels take (chunk_of() in
// csrc/attend_plan.h, which they call): on 300000 random shapes, of every length up to the
// most, no chunk is longer than LDS has places for, no sequence has more chunks than the
// grid, and no call uses more workspace than it asks for. Built and run by
// tests/test_attend_chunks.py on the CPU.
#include <cmath>
#include <cstdio>
#include <random>

#include "attend_plan.h"

using namespace sifar;

int main() {
    std::mt19937_64 rng(26070897);
    const auto spread = [&](int64_t most) {
        return static_cast<int64_t>(
            std::exp2(std::uniform_real_distribution<double>(0.0, std::log2(double(most)))(rng)));
    };
    long checked = 0, longest = 0, most = 0;
    while (checked < 300000) {
        const int64_t tokens = spread(SIFAR_ATTENTION_MAX_TOKENS), kv = spread(SIFAR_CACHE_MAX_HEADS);
        const int64_t group = spread(SIFAR_CACHE_MAX_HEADS), dim = 8 * (1 + rng() % 32);
        if (kv * group > SIFAR_CACHE_MAX_HEADS) continue;
        const int64_t length = spread(SIFAR_ATTENTION_MAX_LENGTH);
        const int64_t reach = rng() % 2 ? length : spread(length);  // the window
        const int types[] = {SIFAR_BF16, SIFAR_FP16, SIFAR_FP32};
        const int type = types[rng() % 3];
        const int64_t splits = splits_of(type, tokens, kv * group, kv, dim, reach);
        const int round = kWaves * tile_of(type, wide_of(dim));
        bool ok = kMaxChunk % round == 0 && splits >= 1 &&
                  used_bytes(tokens * kv * group, splits, dim) <=
                      asked_bytes(tokens, kv * group, kv, dim, length);
        for (int64_t count : {reach, reach - 1, reach / 2, spread(reach), spread(reach), int64_t{1}}) {
            if (count < 1) continue;
            const int chunk = chunk_of(static_cast<int>(ceil_div(count, splits)), round);
            ok = ok && chunk > 0 && chunk <= kMaxChunk && chunk % round == 0 &&
                 ceil_div(count, chunk) <= splits;
            longest = chunk > longest ? chunk : longest;
        }
        most = splits > most ? long(splits) : most;
        if (!ok) {
            std::printf("FAIL tokens %ld heads %ld x %ld dim %ld length %ld reach %ld type %d: %ld\n",
                        long(tokens), long(kv), long(group), long(dim), long(length), long(reach),
                        type, long(splits));
            return 1;
        }
        ++checked;
    }
    std::printf("checked %ld longest %ld most %ld\n", checked, longest, most);
    return longest == kMaxChunk && most > 1000 ? 0 : 1;
}
