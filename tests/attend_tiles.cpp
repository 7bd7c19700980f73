// Prints what sifar_paged_attention's plan (csrc/attend_plan.h) makes of shapes read from
// stdin as "type tokens q_heads kv_heads head_dim reach": the most tiles of a wave, and
// whether they are read past the caches. Built and run by tests/test_attend_tiles.py.
#include <cstdio>

#include "attend_plan.h"

using namespace sifar;

int main() {
    long type, tokens, q_heads, kv_heads, dim, reach;
    while (std::scanf("%ld %ld %ld %ld %ld %ld", &type, &tokens, &q_heads, &kv_heads, &dim, &reach) == 6) {
        const int64_t splits = splits_of(int(type), tokens, q_heads, kv_heads, dim, reach);
        const int64_t round = kWaves * tile_of(int(type), wide_of(dim));
        const int64_t tiles = ceil_div(ceil_div(reach, splits), round);
        const bool once = tiles_of(q_heads, kv_heads) == 1 && wide_of(dim) == dim &&
                          2 * reach * tokens * kv_heads * dim * (type == SIFAR_FP32 ? 4 : 2) >=
                              int64_t{1} << 27;
        std::printf("%ld %d\n", long(tiles), int(once));
    }
    return 0;
}
